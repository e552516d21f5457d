"""The 8-bit cache, the decode from it and pages that requests share, on the GPU against their definitions (tests/paged_ref.py)."""
import numpy as np
import pytest
import torch

from tests import operators_ref, paged_ref as ref
from tests.paged_ref import check_decode, part_bytes
from tests.test_gpu_operators import DT, U, ea, i32  # noqa: F401  (ea: the fixture)

pytestmark = pytest.mark.gpu


def garbage(pages, Hk, d, page, seed):
    """Any bytes, among them scales that are NaN, infinite and negative, and codes -128."""
    raw = np.random.default_rng(seed).integers(0, 256, (pages, Hk, part_bytes(d, page)), dtype=np.uint8)
    raw[:, :, ::5] = 128
    raw[0, :, 2 * page * d:] = 255
    return raw


def pair(pages, Hk, d, page, seed):
    raw = garbage(pages, Hk, d, page, seed)
    return torch.from_numpy(raw).cuda(), ref.Cache8(raw, d, page)


def same_rows(got, want, dtype):
    for a, b in zip(got, want):
        b = torch.from_numpy(b).float().to(dtype)                 # (a product of a code and a scale, rounded to fp32, then to dtype)
        assert torch.equal(torch.isnan(a.cpu()), torch.isnan(b)) and torch.equal(torch.nan_to_num(a.cpu()), torch.nan_to_num(b))


def rows_of(rng, T, Hk, d, dtype, spread=0.7):
    x = rng.standard_normal((T, Hk, d)) * np.exp(spread * rng.standard_normal((T, 1, d)))
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


# ---- rows ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("Hk,d,dtype,page", [(1, 64, "f32", 16), (3, 128, "bf16", 16), (2, 64, "bf16", 256), (5, 128, "f32", 64), (2, 128, "bf16", 32),
                                             (8, 64, "f32", 128)])
def test_rows_appended_chunk_by_chunk(ea, Hk, d, dtype, page):  # noqa: F811
    """Three requests grow by chunks of one to many tokens; after each call every byte of the cache is what the reference has."""
    rng = np.random.default_rng(Hk * d + page)
    pages = 3 * (300 // page + 1)
    cache, want = pair(pages, Hk, d, page, seed=page)
    order = rng.permutation(pages).reshape(3, -1)
    at = [0, 5 * 16, 0]
    for r in (1,):                                                # (its first blocks have been written before)
        pos = np.arange(at[r])
        slots = order[r][pos // page] * page + pos % page
        k, v = rows_of(rng, at[r], Hk, d, dtype), rows_of(rng, at[r], Hk, d, dtype)
        ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), i32(slots.tolist()), cache, page)
        want.write(k.float().numpy(), v.float().numpy(), slots)
    for chunk in ((1, 1, 1), (1, 3, 16), (2, 1, 17), (0, 33, 1), (15, 1, 30), (1, 1, 1), (40, 2, 64), (1, 1, 1)):
        pos = [np.arange(a, a + c) for a, c in zip(at, chunk)]
        slots = np.concatenate([order[r][p // page] * page + p % page for r, p in enumerate(pos)])
        at = [a + c for a, c in zip(at, chunk)]
        scale = float(np.exp(2 * rng.standard_normal()))
        k, v = rows_of(rng, len(slots), Hk, d, dtype) * scale, rows_of(rng, len(slots), Hk, d, dtype) / scale
        both = torch.cat([k, v], 1).cuda()                        # (views of one projection's rows)
        ea.entmax_attn_cache8_write(both[:, :Hk], both[:, Hk:], i32(slots.tolist()), cache, page)
        want.write(k.float().numpy(), v.float().numpy(), slots)
        np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes())
        for t in (DT["bf16"], DT["f32"]):
            same_rows(ea.entmax_attn_cache8_read(cache, i32(slots.tolist()), page, d, t), want.read(slots), t)


@pytest.mark.parametrize("T,Hk,d,dtype", [(5000, 4, 64, "bf16"), (3333, 8, 128, "f32")])
def test_rows_of_a_long_prompt(ea, T, Hk, d, dtype):  # noqa: F811
    # more rows than a wave each (the write) and items than a thread each (the read); the prompt begins inside a block
    rng = np.random.default_rng(T)
    page, start = 32, 7
    pages = (T + start) // page + 2
    cache, want = pair(pages, Hk, d, page, seed=T)
    pos = np.arange(start, start + T)
    slots = rng.permutation(pages)[pos // page] * page + pos % page
    k, v = rows_of(rng, T, Hk, d, dtype), rows_of(rng, T, Hk, d, dtype)
    assert T * 2 * Hk > 1 << 15 and T * 2 * Hk * d // 8 >= 1 << 18
    ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), i32(slots.tolist()), cache, page)
    want.write(k.float().numpy(), v.float().numpy(), slots)
    np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes())
    got = ea.entmax_attn_cache8_read(cache, i32(slots.tolist()), page, d, DT[dtype])
    same_rows(got, want.read(slots), DT[dtype])


def test_rows_of_many_requests(ea):  # noqa: F811
    # a few tokens each for some hundred requests (the write's middle variant), three times over: scales grow in most blocks
    Hk, d, page, R = 4, 64, 64, 300
    rng = np.random.default_rng(12)
    cache, want = pair(R * 2, Hk, d, page, seed=5)
    order = rng.permutation(R * 2).reshape(R, 2)
    at = np.zeros(R, np.int64)
    for step in range(3):
        chunk = rng.integers(0, 12, R)
        slots = np.concatenate([order[r][np.arange(a, a + c) // page] * page + np.arange(a, a + c) % page for r, (a, c) in enumerate(zip(at, chunk))])
        at += chunk
        k, v = rows_of(rng, len(slots), Hk, d, "bf16") * (1 + step), rows_of(rng, len(slots), Hk, d, "bf16") / (1 + step)
        assert 1 << 12 < len(slots) * 2 * Hk <= 1 << 15
        ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), i32(slots.tolist()), cache, page)
        want.write(k.float().numpy(), v.float().numpy(), slots)
        np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes())


def test_kept_rows_that_are_hard_to_round_again(ea):  # noqa: F811
    """A block of scale s with every code, and rows whose scale is s times what makes halves of many codes (2, 4, 2/3 ...) or nearly so."""
    d, page = 128, 32
    codes = torch.arange(-127, 129).clamp(max=127).float().view(2, 1, d)
    for s in (1.0, float(np.float32(1 / 3)), 2.0 ** -126, 1.7 * 2.0 ** -120, 1.9 * 2.0 ** 118):
        for ratio in (2.0, 4.0, 4 / 3, 2 / 1.5, 254.0, 8.0, 1.0000001, 1.5, 600.0, 2.0 ** 20):
            for step in (0, 1, -1):
                with np.errstate(over="ignore"):
                    top = np.float32(127) * np.float32(s) * np.float32(ratio)
                for _ in range(abs(step) * 60):
                    top = np.nextafter(top, np.float32(np.inf * step))
                if not np.isfinite(top):
                    continue
                cache, want = pair(1, 1, d, page, seed=3)
                k = codes * s
                v = torch.from_numpy(np.random.default_rng(4).standard_normal((2, 1, d)).astype(np.float32))
                row = torch.zeros(1, 1, d)
                row[0, 0, 77] = float(top)
                for a, b, slots in ((k, v, [16, 17]), (row, row, [18])):
                    ea.entmax_attn_cache8_write(a.cuda(), b.cuda(), i32(slots), cache, page)
                    want.write(a.numpy(), b.numpy(), slots)
                    np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes(), err_msg=str((s, ratio, step)))


def test_rows_that_are_hard_to_round(ea):  # noqa: F811
    """Quotients at and next to halves, zeros, the smallest and largest values, infinities and NaN; a block that grows past all of it."""
    d, page = 64, 16
    x = torch.zeros(10, 1, d)
    n = torch.arange(d) - 32.0
    x[0, 0] = n + 0.5
    x[0, 0, 0] = 127.0                                            # scale 1: ties
    x[1, 0] = torch.nextafter(n + 0.5, torch.full((d,), 1e9))
    x[2, 0] = torch.nextafter(n + 0.5, torch.full((d,), -1e9))
    x[3, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 126.5])
    rng = np.random.default_rng(1)
    for scale in (1.0, 1.3e-37, 2.0 ** -149, 2.6e36, 0.0, 1 / 3, 1e-3):
        cache, want = pair(2, 1, d, page, seed=2)
        k = (x * scale).nan_to_num(nan=float("nan")) if scale else torch.zeros_like(x)
        # x times odd scales: values that are near to, and of which many are, halves of the block's own scale
        s = np.float32(np.abs(k[:3].numpy()[np.isfinite(k[:3].numpy())]).max() / 127)
        k[4, 0] = torch.from_numpy((np.arange(d).astype(np.float32) + np.float32(0.5)) * s)
        v = torch.from_numpy(rng.standard_normal((10, 1, d)).astype(np.float32)) * (scale or 1)
        slots = list(range(16, 21))
        ea.entmax_attn_cache8_write(k[:5].cuda(), v[:5].cuda(), i32(slots), cache, page)
        want.write(k[:5].numpy(), v[:5].numpy(), slots)
        np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes())
        k2, v2 = k[5:7] + 3 * scale * 127, v[5:7] * 7
        ea.entmax_attn_cache8_write(k2.cuda(), v2.cuda(), i32([21, 22]), cache, page)
        want.write(k2.numpy(), v2.numpy(), [21, 22])
        np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes())
        same_rows(ea.entmax_attn_cache8_read(cache, i32(list(range(16, 23))), page, d, torch.float32), want.read(range(16, 23)), torch.float32)


def test_rows_skipped_and_out_of_order(ea):  # noqa: F811
    # slots that are negative or past the cache, in front of, between and behind others; rows of a block in falling order
    Hk, d, page = 2, 64, 32
    cache, want = pair(4, Hk, d, page, seed=8)
    rng = np.random.default_rng(9)
    slots = [-1, 4 * page, 40, 41, -7, 70, 71, 2 ** 31 - 1, 127, 126, 125, 112, 0, -2 ** 31, 99, 98]
    k, v = rows_of(rng, len(slots), Hk, d, "f32"), rows_of(rng, len(slots), Hk, d, "f32")
    ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), i32(slots), cache, page)
    want.write(k.numpy(), v.numpy(), slots)
    # (garbage that stood in front of a written row is a block's content like any other: only rows of clean blocks are compared)
    mine = [s for s in (0, 112, 125, 126, 127)]
    same_rows(ea.entmax_attn_cache8_read(cache, i32(mine), page, d, torch.float32), want.read(mine), torch.float32)
    out = [torch.full((3, Hk, d), 5.0, device="cuda") for _ in range(2)]
    ea.entmax_attn_cache8_read(cache, i32([-1, 112, 4 * page]), page, d, out=out)
    for t, w in zip(out, want.read([112])):
        assert (t[[0, 2]] == 5).all() and torch.equal(t[1].cpu(), torch.from_numpy(w[0]).float())     # (one rounding)
    untouched = cache.clone()
    ea.entmax_attn_cache8_write(k[:0].cuda(), v[:0].cuda(), i32([]), cache, page)
    ea.entmax_attn_cache8_write(k[:2].cuda(), v[:2].cuda(), i32([-1, 4 * page + 5]), cache, page)
    assert torch.equal(cache, untouched)


@pytest.mark.parametrize("T", [80, 5000])
def test_rows_of_one_slot_or_apart_leave_other_blocks_alone(ea, T):  # noqa: F811
    # what the header leaves undefined stays inside the blocks concerned: one slot forty times, rows of a block apart from each other
    Hk, d, page = 4, 64, 32
    rng = np.random.default_rng(T)
    pages = T // page + 4
    cache, want = pair(pages, Hk, d, page, seed=T)
    slots = list(range(2 * page, 2 * page + T))
    for i in range(40):
        slots[20 + i] = 5                                         # block 0
    slots[70], slots[75] = 17, 20                                 # block 1, apart, in the middle of other rows
    fine = [s if s >= 2 * page else -1 for s in slots]
    k, v = rows_of(rng, T, Hk, d, "bf16"), rows_of(rng, T, Hk, d, "bf16")
    ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), i32(slots), cache, page)
    want.write(k.float().numpy(), v.float().numpy(), fine)
    got, ref_bytes = cache.cpu().numpy(), want.bytes()
    hurt = {s // 16 for i, s in enumerate(slots) if s < 2 * page or any(0 <= j < T and slots[j] < 2 * page for j in (i - 1, i + 1))}
    hurt |= {(2 * page + i) // 16 for i in (20, 60, 70, 75)}
    n = page * d
    for b in range(pages * page // 16):
        if b in hurt:
            continue
        pg, at = b * 16 // page, b * 16 % page
        for o in (0, n):
            np.testing.assert_array_equal(got[pg, :, o + at * d:o + (at + 16) * d], ref_bytes[pg, :, o + at * d:o + (at + 16) * d])
        for o in (2 * n + 4 * (at // 16), 2 * n + 4 * (page // 16 + at // 16)):
            np.testing.assert_array_equal(got[pg, :, o:o + 4], ref_bytes[pg, :, o:o + 4])


def test_rows_of_any_stride(ea):  # noqa: F811
    Hk, d, page = 3, 64, 16
    rng = np.random.default_rng(4)
    slots = i32([3, 4, 5, 16, 17, 33])
    x = rows_of(rng, 6, Hk, d, "bf16").cuda()
    heads_first = x.transpose(0, 1).contiguous().transpose(0, 1)
    repeated = x[:1].expand(6, -1, -1)
    a, b = (ea.entmax_attn_cache8_empty(4, Hk, d, page) for _ in range(2))
    ea.entmax_attn_cache8_write(heads_first, repeated, slots, a, page)
    ea.entmax_attn_cache8_write(x, repeated.contiguous(), slots, b, page)
    assert torch.equal(a, b)
    out = [torch.zeros(Hk, 6, d, device="cuda").transpose(0, 1) for _ in range(2)]
    ea.entmax_attn_cache8_read(a, slots, page, d, out=out)
    for s, t in zip(out, ea.entmax_attn_cache8_read(b, slots, page, d, torch.float32)):
        assert torch.equal(s, t)


# ---- decode -------------------------------------------------------------------------------------------------------

def make_cache(ea, lens, Hk, d, page, sigma, seed, spare=3):  # noqa: F811
    """Requests' keys and values written through the library; garbage in every slot that holds none."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    cache, _ = pair(sum(need) + spare, Hk, d, page, seed)
    order, at = rng.permutation(sum(need) + spare), 0
    table = torch.full((len(lens), max(max(need), 1) + 1), -1, dtype=torch.int32)
    ks, vs = [], []
    for r, n in enumerate(lens):
        table[r, :need[r]] = torch.from_numpy(order[at:at + need[r]].astype(np.int32))
        at += need[r]
        pos = torch.arange(n)
        slots = (table[r, pos // page] * page + pos % page).to(torch.int32).cuda()
        k, v = (torch.from_numpy(s * rng.standard_normal((n, Hk, d)).astype(np.float32)) for s in (np.float32(sigma), np.float32(1)))
        ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), slots, cache, page)
        held = ref.Cache8(np.zeros((-(-n // 256) or 1, Hk, part_bytes(d, 256)), np.uint8), d, 256)
        held.write(k.numpy(), v.numpy(), range(n))
        k, v = held.read(range(n))
        ks.append(k)
        vs.append(v)
    return cache, table.cuda(), i32(lens), ks, vs


DECODE = [
    # lens, Hq, Hk, d, dtype, page, alpha, sigma
    ([1], 1, 1, 64, "bf16", 16, 1.5, 1.0),
    ([0, 1, 2, 15, 16, 17, 63, 64, 65], 4, 2, 64, "f32", 16, 1.5, 1.0),
    ([0, 1, 31, 33, 255, 256, 257, 300], 8, 8, 128, "bf16", 256, 1.5, 1.5),
    ([1000, 37, 4099], 32, 8, 128, "bf16", 64, 1.5, 1.5),
    ([700, 1300], 16, 1, 128, "f32", 32, 2.0, 1.5),
    ([700, 90], 40, 2, 64, "bf16", 128, 1.25, 1.5),            # 20 query heads a key head: two column groups
    ([333], 33, 1, 128, "bf16", 16, 1.75, 2.0),                # three, the last with one head
    ([2000, 5], 3, 3, 64, "f32", 64, 2.5, 1.0),
    ([800], 2, 1, 128, "f32", 16, 3.0, 1.0),
    ([6000, 100], 4, 2, 64, "bf16", 64, 1.5, 0.2),             # flat: more candidates than the second kernel's buffer
    ([5000], 2, 2, 128, "f32", 32, 1.1, 1.0),                  # r = 10: hundreds of keys in the support
    ([3000], 2, 1, 64, "bf16", 16, 1.02, 1.5),                 # r = 50
    ([7 * i for i in range(40)], 16, 2, 64, "bf16", 64, 1.5, 1.5),             # 640 heads: four waves each in the second kernel
    ([33 * i for i in range(1, 34)], 16, 1, 128, "bf16", 32, 1.25, 1.0),
    ([50000], 8, 2, 64, "bf16", 128, 1.5, 1.5),
    ([70000], 8, 2, 128, "f32", 64, 1.5, 1.5),                 # sixteen waves in the second kernel
    ([70000], 2, 1, 64, "bf16", 256, 1.5, 0.2),                # and flat
    ([3 * i for i in range(70)], 32, 4, 64, "bf16", 16, 1.5, 1.5),             # 2240 heads: two waves each
    ([9 * i for i in range(70)], 16, 1, 128, "f32", 32, 2.0, 0.3),             # 1120, flat
]


@pytest.mark.parametrize("lens,Hq,Hk,d,dtype,page,alpha,sigma", DECODE)
def test_decode_from_the_cache(ea, lens, Hq, Hk, d, dtype, page, alpha, sigma):  # noqa: F811
    cache, table, ln, ks, vs = make_cache(ea, lens, Hk, d, page, sigma, seed=sum(lens) + d)
    g = torch.Generator().manual_seed(9)
    q = (torch.randn(len(lens), Hq, d, generator=g) * sigma).to(DT[dtype])
    got = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, alpha, page)
    again = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, alpha, page)
    for a, b in zip(got, again):
        assert torch.equal(a, b)                                   # bit for bit
    check_decode(q, ks, vs, alpha, *(t.cpu() for t in got), dtype)
    got = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, alpha, page, max_len=max(lens))     # (another split over the waves)
    check_decode(q, ks, vs, alpha, *(t.cpu() for t in got), dtype)


WINDOWS = [
    # lens, Hq, Hk, d, dtype, page, alpha, window, sinks
    ([0, 1, 2, 63, 64, 65, 66, 127, 128, 129, 200], 4, 2, 64, "bf16", 16, 1.5, 1, 0),          # the last key alone: p = 1
    ([0, 1, 2, 63, 64, 65, 66, 127, 128, 129, 200], 4, 2, 64, "f32", 16, 1.5, 1, 1),
    ([5, 64, 66, 100, 128, 130, 191, 192, 193, 400, 1000], 8, 2, 128, "bf16", 32, 1.5, 64, 4),
    ([5, 64, 66, 100, 128, 130, 191, 192, 193, 400, 1000], 8, 2, 128, "f32", 64, 2.0, 65, 64),
    ([64 + i for i in range(0, 130, 7)], 2, 1, 64, "bf16", 16, 1.5, 66, 65),                   # sinks and window meet, or nearly so
    ([300, 301, 700], 4, 4, 64, "f32", 256, 1.25, 200, 150),
    ([3000, 10, 2047], 16, 2, 128, "bf16", 64, 1.5, 1000, 4),
    ([500, 20], 4, 1, 64, "bf16", 16, 1.5, 2 ** 40, 7),                                        # longer than any request
    ([500, 20], 4, 1, 64, "bf16", 16, 1.5, 30, 2 ** 31 - 1),                                   # all of them sinks
    ([20000, 5], 32, 8, 128, "bf16", 64, 1.5, 4096, 16),
]


@pytest.mark.parametrize("lens,Hq,Hk,d,dtype,page,alpha,window,sinks", WINDOWS)
def test_decode_of_a_sliding_window(ea, lens, Hq, Hk, d, dtype, page, alpha, window, sinks):  # noqa: F811
    cache, table, ln, ks, vs = make_cache(ea, lens, Hk, d, page, 1.5, seed=sum(lens) + d)
    q = (1.5 * torch.randn(len(lens), Hq, d, generator=torch.Generator().manual_seed(2))).to(DT[dtype])
    # the entries of pages without a key that is seen may be anything, and what is not seen in the others, too
    for r, n in enumerate(lens):
        see = ref.visible(n, window, sinks)
        for b in range(table.shape[1]):
            part = see[b * page:(b + 1) * page]
            if not part.any():
                table[r, b] = [-1, 2 ** 31 - 1, -2 ** 31, cache.shape[0]][b % 4]
            elif not part.all():
                hidden = [int(table[r, b]) * page + int(i) for i in np.flatnonzero(~part)]
                other = [s for s in hidden if not see[(b * page + s % page) // 16 * 16:][:16].any()]       # of blocks of 16 that are hidden whole
                bad = torch.full((len(other), Hk, d), float("nan"), device="cuda")
                ea.entmax_attn_cache8_write(bad, bad, i32(other), cache, page)
    got = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, alpha, page, max_len=max(lens), window=window, sinks=sinks)
    check_decode(q, ks, vs, alpha, *(t.cpu() for t in got), dtype, window, sinks)
    again = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, alpha, page, max_len=max(lens), window=window, sinks=sinks)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_decode_hides_what_a_window_hides_inside_a_block(ea):  # noqa: F811
    # NaN in every single key next to the visible ones, in blocks of 16 that they share
    n, d, page, window, sinks = 300, 64, 64, 90, 5
    cache, table, ln, ks, vs = make_cache(ea, [n], 1, d, page, 1.0, seed=6)
    q = torch.randn(1, 2, d, generator=torch.Generator().manual_seed(1))
    parts = ref.Cache8(cache.cpu().numpy(), d, page)
    for j in np.flatnonzero(~ref.visible(n, window, sinks)):
        pg, row = int(table[0, j // page]), j % page
        for i in (0, 1):
            parts.codes[i][pg, 0, row, j % d] = -128
            parts.scales[i][pg, 0, row // 16] = -abs(parts.scales[i][pg, 0, row // 16])
    cache.copy_(torch.from_numpy(parts.bytes()))
    got = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, 1.5, page, window=window, sinks=sinks)
    check_decode(q, ks, vs, 1.5, *(t.cpu() for t in got), "f32", window, sinks)
    for w, s in ((window + 1, sinks), (window, sinks + 1), (0, 0)):
        got = ea.entmax_attn_decode_cache8(q.cuda(), cache, table, ln, 1.5, page, window=w, sinks=s)
        assert torch.isnan(got[0]).all() and torch.isnan(got[1]).all() and (got[2] == -1).all()


def test_decode_marks_what_it_cannot_answer(ea):  # noqa: F811
    lens, d, page = [40] * 7, 64, 16
    cache, table, ln, ks, vs = make_cache(ea, lens, 1, d, page, 1.0, seed=32)
    q = torch.randn(7, 2, d, generator=torch.Generator().manual_seed(1)).cuda()
    clean = ea.entmax_attn_decode_cache8(q, cache, table, ln, 1.5, page, max_len=48)
    ln = i32([40, -1, 49, 40, 40, 40, 40])
    bad = table.clone()
    bad[3, 1] = cache.shape[0]
    bad[4, 2] = -5
    q2 = q.clone()
    q2[5, 1, 3] = float("inf")
    q2[6, 0, 3] = float("nan")
    got = ea.entmax_attn_decode_cache8(q2, cache, bad, ln, 1.5, page, max_len=48)
    for r in range(1, 5):
        assert torch.isnan(got[0][r]).all() and torch.isnan(got[1][r]).all() and (got[2][r] == -1).all(), r
    for r, h in ((5, 1), (6, 0)):
        assert torch.isnan(got[0][r, h]).all() and got[2][r, h] == -1
    for r, h in ((0, 0), (0, 1), (5, 0), (6, 1)):
        assert torch.equal(got[0][r, h], clean[0][r, h])
    # a key that is not finite, seen and behind the end
    k = torch.randn(1, 1, d).cuda()
    k[0, 0, 5] = float("nan")
    ea.entmax_attn_cache8_write(k, k, i32([int(table[0, 2]) * page + 7]), cache, page)
    ln = i32([40] * 7)
    got = ea.entmax_attn_decode_cache8(q, cache, table, ln, 1.5, page)
    assert torch.isnan(got[0][0]).all() and torch.isfinite(got[0][1:]).all()
    got = ea.entmax_attn_decode_cache8(q, cache, table, i32([39] + [40] * 6), 1.5, page)
    assert torch.isfinite(got[0]).all()
    # its slot written again: the block's mark stays, the key is as good as any
    k = torch.nan_to_num(k)
    ea.entmax_attn_cache8_write(k, k, i32([int(table[0, 2]) * page + 7]), cache, page)
    assert torch.isfinite(ea.entmax_attn_decode_cache8(q, cache, table, ln, 1.5, page)[0]).all()
    # a value that is not finite counts where it is in the support: alpha = 2, a query along one key far above the others
    v = torch.zeros(1, 1, d, device="cuda")
    v[0, 0, 9] = float("inf")
    k = 100 * q[1, :1, None].transpose(0, 1)
    ea.entmax_attn_cache8_write(k, v, i32([int(table[1, 2]) * page + 7]), cache, page)
    got = ea.entmax_attn_decode_cache8(q, cache, table, ln, 2.0, page)
    assert got[2][1, 0] == 1 and torch.isnan(got[0][1, 0, 9]) and torch.isnan(got[0][1, 0]).sum() == 1


@pytest.mark.parametrize("e,finite", [(103, True), (104, False), (127, False)])
def test_decode_of_the_largest_products(ea, e, finite):  # noqa: F811
    # 2^e is the power of two of the query's largest element, scales are 1
    d, page = 64, 16
    cache = ea.entmax_attn_cache8_empty(1, 1, d, page)
    k = torch.zeros(2, 1, d)
    k[0, 0, 0], k[1, 0, 1] = 127, 127
    ea.entmax_attn_cache8_write(k.cuda(), torch.ones(2, 1, d).cuda(), i32([0, 1]), cache, page)
    for dtype in ("bf16", "f32"):
        q = torch.zeros(1, 2, d)
        q[0, 0, 0], q[0, 1, 0] = 1.5 * 2.0 ** e, 1.0
        got = ea.entmax_attn_decode_cache8(q.to(DT[dtype]).cuda(), cache, i32([[0]]), i32([2]), 1.5, page)
        assert torch.isfinite(got[0][0, 1]).all() and (torch.isfinite(got[0][0, 0]).all().item() is finite) and (got[2][0, 0].item() == (1 if finite else -1))


@pytest.mark.parametrize("d,G", [(64, 3), (64, 17), (128, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decode_scores_of_single_elements(ea, dtype, d, G):  # noqa: F811
    """Request i's only key is 127 times the unit vector i, so that its score is 127 q_i: with alpha = 2 and p = 1, tau = 127 q_i /
    sqrt(d) - 1.  127 q_i of an element known to 24 bits has up to 31: one rounding of the score, one of tau.  Rows of 2^20: the 1
    takes nothing off."""
    exact, known = ref.TERMS[dtype]
    g = torch.Generator().manual_seed(d + G)
    q = torch.randn(G, d, generator=g).sign() * torch.exp2(torch.rand(G, d, generator=g) * 40 - 39.999) * 2.0 ** 20
    q[:, ::2] = (torch.rand(G, d // 2, generator=g) * 2 - 1) * 2.0 ** 20             # half of them within a few binades of the largest
    q[:, 0] = 1.99 * 2.0 ** 19
    q[0, 2] = float(np.nextafter(np.float32(2.0 ** 20), np.float32(0)))               # all bits set
    q = q.to(DT[dtype])
    cache = ea.entmax_attn_cache8_empty(d, 1, d, 16)
    table = torch.arange(d, dtype=torch.int32, device="cuda")[:, None].contiguous()
    ea.entmax_attn_cache8_write(127 * torch.eye(d)[:, None].cuda(), torch.ones(d, 1, d).cuda(), table[:, 0] * 16, cache, 16)
    O, tau, support = ea.entmax_attn_decode_cache8(q.cuda().expand(d, G, d).contiguous(), cache, table, i32([1] * d), 2.0, 16)
    x = 127 * q.double().numpy().T                                                    # [request, head]
    top = np.abs(x).max(0)
    scale = 1 / np.sqrt(np.float64(d))
    want = x * scale - 1
    err = np.abs(tau.double().cpu().numpy() - want)
    # the score is rounded where its two parts become floats and where they are added: 3 u; 1 / 127 is no scale of 1: none here
    tol = np.abs(want) * U + 3 * U * np.abs(x) * scale + np.where(np.abs(x) < exact * top, known * top * scale, 0.0) + 2.0 ** -52 * top
    assert (err <= tol).all(), ((err > tol).mean(), (err / tol).max())
    assert (O == 1).all() and (support == 1).all()


def test_decode_queries_of_wide_range(ea):  # noqa: F811
    lens, Hq, d, page = [500], 12, 128, 16
    cache, table, ln, ks, vs = make_cache(ea, lens, 2, d, page, 1.0, seed=31)
    g = torch.Generator().manual_seed(10)
    q = torch.randn(1, Hq, d, generator=g) * torch.exp2(-torch.rand(1, Hq, d, generator=g) * 30)
    q[0, 1] *= 1e-30
    q[0, 2] = 0
    q[0, 3, 1:] = 0
    q[0, 4] *= 2.0 ** 10
    q[0, 5, ::2] *= 2.0 ** -40
    for dtype in ("bf16", "f32"):
        x = q.to(DT[dtype])
        got = ea.entmax_attn_decode_cache8(x.cuda(), cache, table, ln, 1.5, page)
        check_decode(x, ks, vs, 1.5, *(t.cpu() for t in got), dtype)


@pytest.mark.parametrize("alpha", [1.5, 2.0, 3.0])
def test_decode_of_the_longest_request_with_equal_scores(ea, alpha):  # noqa: F811
    """2^22 keys of zero, one page serving for all: tau = -N^(-1/r), as close to the maximum as it can be, and every p = 1/N.  Bounds
    as for the 4-bit cache, whose second kernel this is."""
    N, r = 1 << 22, 1 / (alpha - 1)
    cache = ea.entmax_attn_cache8_empty(1, 1, 64, 256)
    ea.entmax_attn_cache8_write(torch.zeros(256, 1, 64, device="cuda"), 127 * torch.ones(256, 1, 64, device="cuda"), i32(list(range(256))), cache, 256)
    table = torch.zeros(1, N // 256, dtype=torch.int32, device="cuda")
    O, tau, support = ea.entmax_attn_decode_cache8(torch.ones(1, 1, 64, device="cuda"), cache, table, i32([N]), alpha, 256)
    assert (support == N).all()
    assert ((O / 127 - 1).abs() <= (N // 256 + N // 512 + 64) * U).all(), O
    want = -float(N) ** (-1 / r)
    assert (tau.double().cpu() - want).abs().item() <= abs(want) * (N // 512 + 64) * U / r + 6e-8, (tau, want)


def test_two_decodes_at_once_and_on_another_stream(ea):  # noqa: F811
    cache, table, ln, ks, vs = make_cache(ea, [3000, 500], 2, 128, 32, 1.5, seed=40)
    g = torch.Generator().manual_seed(12)
    qa, qb = ((1.5 * torch.randn(2, 8, 128, generator=g)).to(torch.bfloat16).cuda() for _ in range(2))
    args = [dict(), dict(window=700, sinks=3)]
    wa, wb = (ea.entmax_attn_decode_cache8(x, cache, table, ln, 1.5, 32, **a) for x, a in zip((qa, qb), args))
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    ws = [torch.empty(ea.entmax_attn_decode_cache8_workspace_bytes(2, 8, 2, 128, table.shape[1] * 32, **a), dtype=torch.uint8, device="cuda") for a in args]
    for _ in range(5):
        with torch.cuda.stream(sa):
            a = ea.entmax_attn_decode_cache8(qa, cache, table, ln, 1.5, 32, workspace=ws[0], **args[0])
        with torch.cuda.stream(sb):
            b = ea.entmax_attn_decode_cache8(qb, cache, table, ln, 1.5, 32, workspace=ws[1], **args[1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a + b, wa + wb))


# ---- pages --------------------------------------------------------------------------------------------------------

class Shared:
    """The library's and the reference's state side by side."""

    def __init__(self, lens, n_pages, blocks, page, rng, free=None):
        need = [-(-n // page) for n in lens]
        order, at = rng.permutation(n_pages), 0
        table = rng.integers(-3, n_pages + 3, (len(lens), blocks))           # (entries behind a request's pages are anything)
        for r in range(len(lens)):
            table[r, :need[r]] = order[at:at + need[r]]
            at += need[r]
        spare = order[at:] if free is None else order[at:at + free]
        self.want = ref.Pages(table, spare, n_pages, page)
        self.page, self.lens = page, list(lens)
        self.table, self.free, self.count, self.shares = i32(self.want.table), i32(self.want.stack), i32([len(spare)]), i32(self.want.shares)

    def check(self):
        w = self.want
        assert self.count.item() == w.count
        assert self.free[:w.count].tolist() == w.stack[:w.count]
        assert self.shares.tolist() == w.shares
        np.testing.assert_array_equal(self.table.cpu().numpy(), np.array(w.table))

    def fork(self, ea, parents, new, **how):  # noqa: F811
        out = ea.entmax_attn_cache_fork(i32(self.lens), i32(parents), i32(new), self.table, self.free, self.count, self.shares, self.page, **how)
        lens, moves, status = self.want.fork(self.lens, parents, new)
        assert out[0].tolist() == lens and out[2].tolist() == status
        assert out[1].tolist() == [list(m) for m in moves] + [[-1, -1]] * (len(lens) - len(moves))
        self.check()
        self.lens = lens
        return out


@pytest.mark.parametrize("R,blocks,page,pages", [(1, 4, 16, 10), (5, 8, 16, 60), (70, 12, 32, 900), (1100, 5, 16, 4000), (4096, 2, 64, 9000),
                                                 # (in four launches)
                                                 (1100, 30, 16, 20000), (40, 800, 16, 17000), (4096, 9, 32, 20000), (3, 6000, 16, 10000)])
def test_forks_against_the_reference(ea, R, blocks, page, pages):  # noqa: F811
    rng = np.random.default_rng(R)
    s = Shared([int(n) for n in rng.integers(0, blocks * page // 2, R)], pages, blocks, page, rng)
    for step in range(6 if R < 1000 else 3):
        s.fork(ea, *ref.random_fork(rng, s.lens))
    s.fork(ea, list(range(R)), [0] * R)                                      # all end: every page is free again
    assert s.count.item() == pages and s.shares.sum().item() == 0 and sorted(s.free.tolist()) == list(range(pages))


def test_forks_that_leave_many_pages(ea):  # noqa: F811
    # tens of thousands of entries left, with and without other holders: the stack is built in several pieces
    rng = np.random.default_rng(16)
    R, blocks, page = 300, 200, 16
    s = Shared([int(n) for n in rng.integers(80 * page, blocks * page + 1, R)], 45000, blocks, page, rng)
    s.fork(ea, [r if r < 150 else r - 150 for r in range(R)], [s.lens[r % 150] for r in range(R)])           # half of them leave theirs
    s.fork(ea, *ref.random_fork(rng, s.lens))
    s.fork(ea, list(range(R)), [n // 9 for n in s.lens])
    s.fork(ea, list(range(R)), [0] * R)
    assert s.count.item() == 45000 and s.shares.sum().item() == 0 and sorted(s.free.tolist()) == list(range(45000))


@pytest.mark.parametrize("blocks", [4, 3000])                                # (one launch, four launches)
def test_forks_where_no_page_is_left(ea, blocks):  # noqa: F811
    rng = np.random.default_rng(7)
    s = Shared([40, 0, 0, 0, 33, 0], 8, blocks, 16, rng, free=2)
    out = s.fork(ea, [0, 0, 0, 4, 4, 4], [40, 40, 33, 33, 33, 32])           # copies for 1, 2 and 3, two pages left
    assert out[2].tolist() == [2, 1, 0, 0]
    s.fork(ea, list(range(6)), [0, 40 if s.lens[1] == 40 else s.lens[1], 0, 0, 0, 16])


@pytest.mark.parametrize("blocks", [4, 9000])
def test_forks_with_arguments_out_of_range(ea, blocks):  # noqa: F811
    rng = np.random.default_rng(8)
    lens = [40, -1, blocks * 16 + 1, 20, 0, 7]
    s = Shared([40, 0, 0, 20, 0, 7], 20, blocks, 16, rng)
    s.lens = lens
    out = s.fork(ea, [6, 1, 2, -1, 0, 1], [3, 0, 10, 5, 41, 0])              # a parent that is none (twice), lengths of their own, above the parent's
    assert out[2].tolist() == [0, 0, 6, 0] and out[0].tolist() == lens
    # ids out of range are met, counted and left alone
    t = s.table.clone()
    t[0, 1] = 20
    out = ea.entmax_attn_cache_fork(i32([40, 0]), i32([0, 0]), i32([0, 40]), t[:2].contiguous(), s.free, s.count, s.shares, 16)
    assert out[2].tolist()[3] == 2


@pytest.mark.parametrize("blocks", [10, 3000])
def test_forks_as_lens_itself_and_captured(ea, blocks):  # noqa: F811
    # lens_out = lens and a workspace kept; captured once, replayed with other parents and lengths, eager work between
    rng = np.random.default_rng(9)
    R, page, pages = 6, 16, 80
    a, b = (Shared([100, 0, 33, 0, 16, 0], pages, blocks, page, np.random.default_rng(1)) for _ in range(2))
    lens, parents, new = i32(a.lens), i32(list(range(R))), i32(a.lens)
    out = (lens, torch.empty(R, 2, dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda"))
    ws = torch.empty(ea.entmax_attn_cache_fork_workspace_bytes(R, blocks), dtype=torch.uint8, device="cuda")
    cache = torch.from_numpy(garbage(pages, 1, 64, page, 3)).cuda()
    mirror = cache.clone()

    def step():
        ea.entmax_attn_cache_fork(lens, parents, new, a.table, a.free, a.count, a.shares, page, out=out, workspace=ws)
        ea.entmax_attn_cache_copy(cache, out[1], out[2][:1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                               # (changes nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(25):
        p, n = ref.random_fork(rng, b.lens)
        if k % 6 == 5:
            p, n = [0] * R, [100 if b.lens[0] >= 100 else b.lens[0]] * R
        parents.copy_(i32(p))
        new.copy_(i32(n))
        graph.replay()
        res = b.fork(ea, p, n)
        ea.entmax_attn_cache_copy(mirror, res[1], res[2][:1])
        torch.cuda.synchronize()
        for x, y in ((lens, res[0]), (out[1], res[1]), (out[2], res[2]), (a.table, b.table), (a.shares, b.shares), (a.count, b.count), (cache, mirror)):
            assert torch.equal(x, y), k
        torch.randn(1000, device="cuda").sum().item()


@pytest.mark.parametrize("R,blocks,page,pages,shares", [(1, 1, 16, 1, True), (1, 2, 16, 2, False), (3, 5, 64, 31, True), (20, 9, 32, 64, True),
                                                        (100, 7, 16, 1025, False), (300, 40, 16, 70000, True), (2, 3, 16, 600000, True)])
def test_compaction_against_the_reference(ea, R, blocks, page, pages, shares):  # noqa: F811
    rng = np.random.default_rng(R + pages)
    most = min(blocks, pages // R)
    s = Shared([int(n) for n in rng.integers(0, most * page + 1, R)], pages, blocks, page, rng)
    if shares:
        s.fork(ea, *ref.random_fork(rng, s.lens))
    raw = np.random.default_rng(pages).integers(0, 256, (pages, 1, 64), dtype=np.uint8)      # (pages of 64 bytes: what stands in them is all the same)
    cache = torch.from_numpy(raw).cuda()
    held = [[raw[p] for p in s.want.table[r][:s.want.size(n)]] for r, n in enumerate(s.lens)]
    before = [t.clone() for t in (s.table, s.free, s.shares)]
    args = (i32(s.lens), s.table, s.free, s.count, s.shares if shares else None, page)
    out = ea.entmax_attn_cache_compact(*args)
    for t, b in zip((s.table, s.free, s.shares), before):
        assert torch.equal(t, b)
    # in place
    moves, status = torch.empty(pages // 2, 2, dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    ea.entmax_attn_cache_compact(*args, out=(s.table, s.free, s.shares if shares else None, moves, status))
    want, used = s.want.compact(s.lens)
    for x, y in zip(out, (s.table, s.free, s.shares if shares else None, moves, status)):
        assert (x is None and y is None) or torch.equal(x, y)
    s.check()
    assert status.tolist() == [len(want), used, 0, 0]
    assert moves.tolist() == [list(m) for m in want] + [[-1, -1]] * (pages // 2 - len(want))
    smaller = torch.zeros((max(used, 1), 1, cache.shape[2]), dtype=torch.uint8, device="cuda")
    smaller.copy_(cache[:max(used, 1)])
    ea.entmax_attn_cache_copy(cache, moves, status[:1], dst=smaller)          # into another, smaller cache
    ea.entmax_attn_cache_copy(cache, moves, status[:1])
    assert torch.equal(smaller[:used], cache[:used])
    got = cache.cpu().numpy()
    for r, n in enumerate(s.lens):
        for b in range(s.want.size(n)):
            assert (got[s.want.table[r][b]] == held[r][b]).all()


def test_compaction_of_what_is_inconsistent(ea):  # noqa: F811
    # ids out of range or twice on the stack, a free page in a table, lengths out of range: counted, left, and nothing else is touched
    table, free = i32([[0, 5, 9], [3, 8, 1], [7, 7, 7]]), i32([4, 4, 11, -1, 5, 6, 2, 0, 0, 0])
    out = ea.entmax_attn_cache_compact(i32([48, -1, 100]), table, free, i32([7]), None, 16)
    # free: 2, 4, 5, 6; used = 6: holes 2, 4, 5; moved 7, 8, 9
    assert out[0].tolist() == [[0, 5, 5], [3, 8, 1], [7, 7, 7]]
    assert out[3].tolist()[:3] == [[7, 2], [8, 4], [9, 5]] and out[4].tolist() == [3, 6, 2, 4]


def test_copies_of_pages(ea):  # noqa: F811
    for pages, Hk, d, page in ((9, 1, 64, 16), (40, 3, 128, 32), (12, 8, 128, 256)):
        for four in (False, True):
            cache = ea.entmax_attn_cache4_empty(pages, Hk, d, page) if four else ea.entmax_attn_cache8_empty(pages, Hk, d, page)
            cache.copy_(torch.randint(0, 256, cache.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(pages)))
            want = cache.clone()
            moves = i32([[1, 5], [1, 6], [-1, 3], [2, pages], [2, -1], [pages, 4], [0, 8], [3, 7]])
            ea.entmax_attn_cache_copy(cache, moves, i32([7]))                # (the eighth is not asked for)
            want[5], want[6], want[8] = want[1], want[1], want[0]
            assert torch.equal(cache, want)
            ea.entmax_attn_cache_copy(cache, moves, i32([0]))
            ea.entmax_attn_cache_copy(cache, moves, i32([-3]))
            ea.entmax_attn_cache_copy(cache, moves[:0], i32([5]))
            assert torch.equal(cache, want)
            ea.entmax_attn_cache_copy(cache, moves, i32([100]))
            want[7] = want[3]
            assert torch.equal(cache, want)
    with pytest.raises(ValueError):
        ea.entmax_attn_cache_copy(cache, moves, i32([1]), dst=cache[:, :4].contiguous())


def test_pages_on_another_stream(ea):  # noqa: F811
    # fork, copies and compaction enqueued on a stream of their own behind a long kernel, with the default stream idle
    rng = np.random.default_rng(11)
    s = Shared([100, 0, 33, 0], 60, 3000, 16, rng)
    cache = torch.from_numpy(garbage(60, 1, 64, 16, 3)).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        a = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            a = (a @ a).clamp(-1, 1)
        parents, new, lens = i32([0, 0, 2, 2]), i32([100, 90, 33, 33]), i32(s.lens)
        out = ea.entmax_attn_cache_fork(lens, parents, new, s.table, s.free, s.count, s.shares, 16)
        ea.entmax_attn_cache_copy(cache, out[1], out[2][:1])
        packed = ea.entmax_attn_cache_compact(out[0], s.table, s.free, s.count, s.shares, 16)
        ea.entmax_attn_cache_copy(cache, packed[3], packed[4][:1])
    side.synchronize()
    want, moves, status = s.want.fork(s.lens, [0, 0, 2, 2], [100, 90, 33, 33])
    assert out[0].tolist() == want and out[2].tolist() == status and out[1].tolist()[:len(moves)] == [list(m) for m in moves]
    s.check()
    moved, used = s.want.compact(want)
    assert packed[4].tolist() == [len(moved), used, 0, 0] and packed[3].tolist()[:len(moved)] == [list(m) for m in moved]
    np.testing.assert_array_equal(packed[0].cpu().numpy(), np.array(s.want.table))


# ---- in turn ------------------------------------------------------------------------------------------------------

def test_serving_with_samples_of_one_prompt(ea):  # noqa: F811
    """Two prompts, four samples of one and a copy of the other; tokens for all, samples that end or fork again, a compaction in
    the middle: each step against the tokens each request stands for."""
    R, Hq, Hk, d, page, blocks, pages = 6, 8, 2, 64, 16, 12, 60
    g = torch.Generator(device="cuda").manual_seed(3)
    cache, _ = pair(pages, Hk, d, page, seed=1)
    dev = dict(dtype=torch.int32, device="cuda")
    lens, table = torch.zeros(R, **dev), torch.full((R, blocks), -1, **dev)
    free, count, shares = torch.arange(pages, **dev), torch.full((1,), pages, **dev), torch.zeros(pages, **dev)
    freq = torch.pow(10000.0, -torch.arange(d // 2, dtype=torch.float64) / (d // 2)).float().cuda()
    own = [ref.Cache8(np.zeros((1, Hk, part_bytes(d, 256)), np.uint8), d, 256) for _ in range(R)]      # each request's tokens in a cache of its own

    def grow(new):
        nonlocal lens
        old = lens.tolist()
        lens, start, slots, positions, status = ea.entmax_attn_cache_tables(lens, i32(new), table, free, count, page, 100)
        assert status.tolist()[1:] == [0, 0, 0]
        x = torch.randn(100, 1, Hq + 2 * Hk, d, generator=g, device="cuda").to(torch.bfloat16)
        q, k = ea.entmax_attn_qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq:Hq + Hk], positions[:, None], freq)
        v = x[:, 0, Hq + Hk:]
        ea.entmax_attn_cache8_write(k[:, :, 0], v, slots, cache, page)
        for r, (a, b) in enumerate(zip(old, new)):
            rows = slice(start[r].item(), start[r].item() + b - a)
            own[r].write(k[rows, :, 0].float().cpu().numpy(), v[rows].float().cpu().numpy(), range(a, b))

    def attend(**how):
        q = torch.randn(R, Hq, d, generator=g, device="cuda").to(torch.bfloat16)
        got = ea.entmax_attn_decode_cache8(q, cache, table, lens, 1.5, page, **how)
        kv = [o.read(range(n)) for o, n in zip(own, lens.tolist())]
        check_decode(q.cpu(), [a for a, _ in kv], [b for _, b in kv], 1.5, *(t.cpu() for t in got), "bf16", **how)

    def fork(parents, new):
        nonlocal lens, own
        lens, moves, status = ea.entmax_attn_cache_fork(lens, i32(parents), i32(new), table, free, count, shares, page)
        ea.entmax_attn_cache_copy(cache, moves, status[:1])
        assert status.tolist()[1:] == [0, 0, 0]
        own = [ref.Cache8(own[p].bytes(), d, 256) for p in parents]

    grow([43, 32, 0, 0, 0, 0])
    fork([0, 1, 0, 0, 1, 0], [43, 32, 43, 43, 32, 40])
    attend()
    for t in range(1, 4):
        grow([43 + t, 32 + t, 43 + t, 43 + t, 32 + t, 40 + t])
        attend()
    fork([2, 1, 2, 2, 4, 5], [46, 35, 46, 30, 0, 43])
    grow([47, 36, 47, 33, 0, 44])
    attend()
    out = ea.entmax_attn_cache_compact(lens, table, free, count, shares, page)
    ea.entmax_attn_cache_copy(cache, out[3], out[4][:1])
    table, free, shares = out[:3]
    attend(window=20, sinks=3)
    used = out[4][1].item()
    # the rest of the cache can be given back
    cache = cache[:used + 12].clone()
    free, shares = torch.full((used + 12,), -1, **dev), shares[:used + 12].clone()
    free[:12] = torch.arange(used + 11, used - 1, -1, **dev)
    count.fill_(12)
    grow([60, 50, 60, 40, 20, 60])
    attend()
    fork(list(range(R)), [0] * R)
    assert count.item() == used + 12 and shares.sum().item() == 0


def test_rows_and_decode_captured_and_replayed(ea):  # noqa: F811
    # a step with a token each as a graph, replayed with other rows and lengths, against eager steps on a second cache
    R, Hq, Hk, d, page, blocks = 4, 8, 2, 128, 16, 10
    dev = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(R * blocks, **dev).view(R, blocks)
    caches = [ea.entmax_attn_cache8_empty(R * blocks, Hk, d, page) for _ in range(2)]
    lens, slots = torch.zeros(R, **dev), torch.full((R,), -1, **dev)
    rows, q = torch.zeros(R, 2 * Hk, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(R, Hq, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(ea.entmax_attn_decode_cache8_workspace_bytes(R, Hq, Hk, d, blocks * page, 50, 4), dtype=torch.uint8, device="cuda")

    def step(cache, ws):
        ea.entmax_attn_cache8_write(rows[:, :Hk], rows[:, Hk:], slots, cache, page)
        return ea.entmax_attn_decode_cache8(q, cache, table, lens, 1.5, page, window=50, sinks=4, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(caches[0], ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(caches[0], ws)
    g = torch.Generator(device="cuda").manual_seed(4)
    for t in range(70):
        lens.fill_(t + 1)
        slots.copy_(table[:, t // page] * page + t % page)
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda") * (1 + t % 5))
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        graph.replay()
        want = step(caches[1], None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), t
        assert torch.equal(*caches)
        torch.randn(1000, device="cuda").sum().item()


def test_chunked_prefill_attends_to_the_cache_as_it_is(ea):  # noqa: F811
    # the keys of a prompt are written, read back and attended to by entmax_attn_fwd: the last row equals the decode
    N, H, d, page = 192, 2, 64, 64
    g = torch.Generator().manual_seed(22)
    q, k, v = ((1.5 * torch.randn(1, H, N, d, generator=g)).cuda() for _ in range(3))
    cache, slots = ea.entmax_attn_cache8_empty(3, H, d, page), i32(list(range(N)))
    ea.entmax_attn_cache8_write(k[0].transpose(0, 1), v[0].transpose(0, 1), slots, cache, page)
    K, V = torch.empty_like(k), torch.empty_like(v)
    ea.entmax_attn_cache8_read(cache, slots, page, d, out=(K[0].transpose(0, 1), V[0].transpose(0, 1)))
    O, tau, _ = ea.entmax_attn_fwd(q, K, V, 1.5, True)
    o, t, _ = ea.entmax_attn_decode_cache8(q[:, :, -1].contiguous(), cache, i32([[0, 1, 2]]), i32([N]), 1.5, page)
    # the fp32 forward's own bar is 1e-5 on O and on tau
    assert (O[:, :, -1] - o).abs().max() <= 2e-5 and (tau[:, :, -1] - t).abs().max() <= 2e-5


def test_cache_beyond_four_gigabytes(ea):  # noqa: F811
    # pages at the end of a cache of 5.3 GB: rows, copies and the decode
    Hk, d, page, n, pages = 8, 128, 256, 600, 10001
    cache = ea.entmax_attn_cache8_empty(pages, Hk, d, page)
    assert cache.numel() > 2 ** 32
    ids = [pages - 1, pages // 2, pages - 7]
    rng = np.random.default_rng(50)
    k, v = rows_of(rng, n, Hk, d, "f32", 0.0), rows_of(rng, n, Hk, d, "f32", 0.0)
    pos = torch.arange(n)
    slots = (torch.tensor(ids)[pos // page] * page + pos % page).to(torch.int32).cuda()
    ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), slots, cache, page)
    held = ref.Cache8(np.zeros((3, Hk, part_bytes(d, page)), np.uint8), d, page)
    held.write(k.numpy(), v.numpy(), range(n))
    ks, vs = held.read(range(n))
    q = torch.randn(1, 16, d, generator=torch.Generator().manual_seed(51)).to(torch.bfloat16)
    for table in (ids, [pages - 3, 5, pages - 2]):
        for a, b in zip(ids, table):
            if a != b:
                ea.entmax_attn_cache_copy(cache, i32([[a, b]]), i32([1]))
        at = (torch.tensor(table)[pos // page] * page + pos % page).to(torch.int32).cuda()
        same_rows(ea.entmax_attn_cache8_read(cache, at, page, d, torch.float32), (ks, vs), torch.float32)
        got = ea.entmax_attn_decode_cache8(q.cuda(), cache, i32([table]), i32([n]), 1.5, page)
        check_decode(q, [ks], [vs], 1.5, *(t.cpu() for t in got), "bf16")
