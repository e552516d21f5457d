"""Accounts of shared pages where something is wrong, and with holders that are none of a call's requests."""
import numpy as np
import pytest
import torch

from tests import paged_ref as ref
from tests.test_gpu_operators import ea, i32  # noqa: F401  (ea: the fixture)

pytestmark = pytest.mark.gpu


# ---- compaction ---------------------------------------------------------------------------------------------------

def stack_after(free, count, pages):
    """What a compaction makes of a stack: its distinct pages in range, the lowest on top, and below them -1 for each other entry."""
    live = min(max(count, 0), pages)
    good = len({p for p in free[:live] if 0 <= p < pages})
    return [-1] * (live - good) + [pages - 1 - i for i in range(good)] + free[live:]


def test_no_page_in_use_is_on_the_stack_after_a_compaction(ea):  # noqa: F811
    # an id out of range on the stack; the pages that are free are granted first, then the entry is met and counted
    page, pages = 16, 8
    free = i32([99, 6, 7, 1, 0, 0, 0, 0])
    table = i32([[0, 2, 3, 4, 5], [-1] * 5])
    lens, count = i32([80, 0]), i32([4])
    out = ea.entmax_attn_cache_compact(lens, table, free, count, None, page)
    assert out[0].tolist() == [[0, 2, 3, 4, 1], [-1] * 5] and out[4].tolist() == [1, 5, 0, 1]
    assert out[1].tolist() == [-1, 7, 6, 5, 0, 0, 0, 0]
    step = ea.entmax_attn_cache_tables(lens, i32([80, 48]), out[0], out[1], count, page, 48)
    assert out[0].tolist() == [[0, 2, 3, 4, 1], [5, 6, 7, -1, -1]]
    assert step[-1].tolist()[3] == 0 and count.item() == 1
    step = ea.entmax_attn_cache_tables(i32([80, 48]), i32([80, 64]), out[0], out[1], count, page, 16)
    assert out[0].tolist()[1] == [5, 6, 7, -1, -1] and step[2].tolist() == [-1] * 16 and step[-1].tolist()[3] == 1


@pytest.mark.parametrize("free,count,lens,table", [
    ([4, 4, 11, -1, 5, 6, 2, 0, 0, 0], 7, [48, -1, 100], [[0, 5, 9], [3, 8, 1], [7, 7, 7]]),
    ([5, 6, 7, 8, 9, 5, 6, 7, 8, 9], 25, [48, 32, 0], [[0, 1, 2], [3, 4, 0], [0, 0, 0]]),       # (a count above the number of pages)
    ([5, 5, 5, 5, 5, 5, 5, 5, 5, 5], 10, [48, 0, 0], [[7, 8, 9], [0, 0, 0], [0, 0, 0]]),
    ([10, -1, 10, -1, 3, 2, 1, 0, 0, 0], 4, [48, 0, 0], [[7, 8, 9], [0, 0, 0], [0, 0, 0]]),
    ([6, 7, 3, 2, 1, 0, 9, 8, 5, 4], -3, [48, 0, 0], [[7, 8, 9], [0, 0, 0], [0, 0, 0]]),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_stacks_that_do_not_add_up(ea, free, count, lens, table, in_place):  # noqa: F811
    pages = len(free)
    t, f, c = i32(table), i32(free), i32([count])
    moves, status = torch.empty(pages // 2, 2, dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    out = ea.entmax_attn_cache_compact(i32(lens), t, f, c, None, 16, out=(t, f, None, moves, status) if in_place else None)
    live = min(max(count, 0), pages)
    want = stack_after(free, count, pages)
    assert out[1].tolist() == want and c.item() == count
    used = pages - len({p for p in free[:live] if 0 <= p < pages})
    assert out[4].tolist()[1] == used
    # every entry that can be popped is a page behind those in use, each once, or none at all
    popped = [p for p in out[1].tolist()[:live] if p != -1]
    assert sorted(popped) == list(range(used, pages))


def test_a_large_stack_that_does_not_add_up(ea):  # noqa: F811
    # (its bits are not made in LDS)
    pages = 600000
    free = list(range(pages - 1, 49, -1)) + [100, 70, 50, -9, pages] + [0] * 45
    table = i32([[49, 48, 47, 0], [1, 2, 3, 4]])
    out = ea.entmax_attn_cache_compact(i32([64, 64]), table, i32(free), i32([pages - 45]), None, 16)
    assert out[1].tolist() == stack_after(free, pages - 45, pages)
    assert out[4].tolist() == [0, 50, 0, 5] and torch.equal(out[0], table)


# ---- forks --------------------------------------------------------------------------------------------------------

PATHS = pytest.mark.parametrize("blocks", [5, 9000])            # (one launch, four launches)


def padded(rows, blocks):
    return i32([r + [-1] * (blocks - len(r)) for r in rows])


@PATHS
def test_pages_that_the_stack_has_no_room_for_are_counted(ea, blocks):  # noqa: F811
    # a count that says 7 of 8 pages are free while a request holds three: two of them find no place
    table, free, count, shares = padded([[0, 1, 2], [], []], blocks), i32([3, 4, 5, 6, 7, 3, 4, -5]), i32([7]), i32([0] * 8)
    out = ea.entmax_attn_cache_fork(i32([48, 0, 0]), i32([0, 1, 2]), i32([0, 0, 0]), table, free, count, shares, 16)
    assert out[2].tolist() == [0, 0, 0, 2] and out[0].tolist() == [0, 0, 0]
    assert count.item() == 8 and free.tolist() == [3, 4, 5, 6, 7, 3, 4, 2] and shares.tolist() == [0] * 8
    # beside ids out of range, which are met as well
    table, free, count, shares = padded([[0, 9, 2], [1], []], blocks), i32([3, 4, 5, 6, 7, 3, 4, -5]), i32([100]), i32([0] * 8)
    out = ea.entmax_attn_cache_fork(i32([48, 16, 0]), i32([0, 1, 2]), i32([0, 16, 0]), table, free, count, shares, 16)
    assert out[2].tolist() == [0, 0, 0, 3] and out[0].tolist() == [0, 16, 0]
    assert count.item() == 8 and free.tolist() == [3, 4, 5, 6, 7, 3, 4, -5]


@PATHS
@pytest.mark.parametrize("left", [0, 2])
def test_requests_with_arguments_out_of_range_stay_as_they_are(ea, blocks, left):  # noqa: F811
    # two or three requests end in one page; those with bad arguments keep it, and who else ends in it gets the copy, or ends before it
    rows = [[0, 1], [0, 1], [0, 1], [2]]
    lens = [20, 20, 20, 5]
    for parents, new, stay in (([0, 1, 2, 3], [20, 21, 0, 5], [1]), ([0, 4, 2, 3], [0, 20, 20, 5], [1]), ([0, -1, 2, 3], [20, 3, -1, 5], [1, 2]),
                               ([0, 0, 0, 3], [21, 21, 21, 6], [0, 1, 2, 3]), ([1, 1, 2, 3], [19, 21, 0, 0], [1]), ([7, 0, 0, 0], [1, 18, 0, 17], [0])):
        table, free, count = padded(rows, blocks), i32([6, 5, 4, 7, 3, -1, -1, -1]), i32([left])
        shares = i32([2, 2, 0, 0, 0, 0, 0, 0])
        out = ea.entmax_attn_cache_fork(i32(lens), i32(parents), i32(new), table, free, count, shares, 16)
        got, tables, stat = out[0].tolist(), table.tolist(), out[2].tolist()
        assert stat[2] == len(stay) and stat[3] == 0
        moves = [m for m in out[1].tolist() if m != [-1, -1]]
        assert stat[0] == len(moves)
        for r in range(4):
            if r in stay:
                assert got[r] == lens[r] and tables[r] == (rows[r] + [-1] * blocks)[:blocks], (parents, r)
            else:
                assert got[r] == new[r] or (stat[1] and got[r] == new[r] // 16 * 16), (parents, r)
        # accounts: every page's holders are counted, free pages are on the stack once, and who may write ends in a page of its own
        held = [tables[r][:-(-got[r] // 16)] for r in range(4)]
        live = free.tolist()[:count.item()]
        for p in range(3):
            k = sum(h.count(p) for h in held)
            assert shares.tolist()[p] == max(k - 1, 0) and live.count(p) == (k == 0), (parents, p)
        for r in range(4):
            if r not in stay and got[r] % 16:
                assert sum(h.count(held[r][-1]) for h in held) == 1, (parents, r)
        # a copy comes from the page that its request would have ended in
        for a, b in moves:
            assert a in (0, 1, 2) and sum(h.count(b) for h in held) == 1


class State:
    """The library's and the reference's tables, stack and holders, with holders that are none of the requests."""

    def __init__(self, lens, pages, blocks, page, rng, pinned):
        need = [-(-n // page) for n in lens]
        order, at, table = rng.permutation(pages).tolist(), 0, []
        for n in need:
            table.append(order[at:at + n] + [-1] * (blocks - n))
            at += n
        shares = [0] * pages
        for r, b in pinned:
            shares[table[r][b]] += 1
        self.want, self.lens, self.page = ref.Pages(table, order[at:], pages, page, shares), list(lens), page
        self.table, self.free, self.count, self.shares = i32(table), i32(self.want.stack), i32([pages - at]), i32(shares)

    def fork(self, ea, parents, new):  # noqa: F811
        out = ea.entmax_attn_cache_fork(i32(self.lens), i32(parents), i32(new), self.table, self.free, self.count, self.shares, self.page)
        lens, moves, status = self.want.fork(self.lens, parents, new)
        assert out[0].tolist() == lens and out[2].tolist() == status
        assert out[1].tolist() == [list(m) for m in moves] + [[-1, -1]] * (len(lens) - len(moves))
        assert self.count.item() == self.want.count and self.free[:self.want.count].tolist() == self.want.stack[:self.want.count]
        assert self.shares.tolist() == self.want.shares and torch.equal(self.table, i32(self.want.table))
        self.lens = lens


@pytest.mark.parametrize("blocks", [12, 9000])
def test_forks_of_pages_that_others_hold_too(ea, blocks):  # noqa: F811
    # a prefix that somebody outside the call holds, whole pages and the one in whose middle a request ends: it is copied, never
    # written to, and its pages stay off the stack when all requests have ended
    rng = np.random.default_rng(blocks)
    lens = [100, 40, 33, 0, 7, 16]
    pinned = [(0, b) for b in range(7)] + [(0, 6), (1, 0), (2, 2), (5, 0)]
    s = State(lens, 90, blocks, 16, rng, pinned)
    held = {s.want.table[r][b] for r, b in pinned}
    s.fork(ea, list(range(6)), lens)                             # everybody who ends in such a page gets one of its own
    assert all(s.want.table[r][s.lens[r] // 16] not in held for r in (0, 2))
    for _ in range(6):
        s.fork(ea, *ref.random_fork(rng, s.lens))
    s.fork(ea, list(range(6)), [0] * 6)
    assert not held & set(s.free[:s.count.item()].tolist())
    assert s.count.item() == 90 - len(held) and s.shares.sum().item() == len(pinned) - len(held)


def test_forks_of_more_entries_than_all_groups_take_at_a_time(ea):  # noqa: F811
    rng = np.random.default_rng(12)
    R, blocks, page, pages = 950, 300, 16, 5000
    s = State([blocks * page] + [0] * (R - 1), pages, blocks, page, rng, [])
    s.fork(ea, [0] * R, [blocks * page - (r % 3) * (r % 11) for r in range(R)])          # 284700 entries taken over
    assert sum(-(-n // page) for n in s.lens[1:]) > 262144 + 16384
    s.fork(ea, list(range(R)), [0] * R)                                                 # and left
    assert s.count.item() == pages and s.shares.sum().item() == 0
