"""The operators beside the attention on the GPU against their definitions in 64 bits: query/key norm with rotation and its
gradient, the step of a scheduler, rows of the 4-bit cache, the decode from it, and all of them in turn.

u = 2^-24, half a step of fp32 relative to the value; a rounding to `dtype` adds finfo.eps / 2."""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ea():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_15180_amd as ea
    ea.lib()
    return ea


def rounding(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


# ---- query/key norm with rotation ---------------------------------------------------------------------------------

ROPE = [
    # B, N, Hq, Hk, d, dtype, rot, axes, interleaved, norm, weights
    (1, 1, 1, 1, 64, "f32", 64, 1, False, True, True),
    (3, 1, 32, 8, 128, "bf16", 128, 1, False, True, True),
    (2, 37, 5, 3, 64, "bf16", 24, 3, False, True, True),
    (1, 129, 4, 1, 128, "f32", 64, 2, True, True, True),
    (2, 65, 3, 2, 128, "bf16", 40, 4, True, True, False),
    (1, 50, 2, 2, 64, "f32", 0, 1, False, True, True),
    (1, 33, 2, 1, 128, "bf16", 128, 2, False, False, False),
    (4, 300, 6, 6, 64, "f32", 64, 3, True, False, False),
    (1, 5000, 3, 1, 64, "bf16", 64, 1, False, True, True),
]


def rope_inputs(B, N, Hq, Hk, d, dtype, rot, axes, weights, seed=3):
    g = torch.Generator().manual_seed(seed)
    rows = (torch.randn(B, N, Hq + Hk + 1, d, generator=g) * 3).to(DT[dtype])
    pairs = rot // 2
    sections = [pairs // axes + (k < pairs % axes) for k in range(axes)]
    pos = torch.randint(-5, 200000, (axes, B, N), generator=g).to(torch.int32)
    pos.view(-1)[0] = 2 ** 31 - 1
    freq = torch.rand(pairs, generator=g) if pairs else None
    if pairs:
        freq[0] = 1.0
    w = [1 + 0.3 * torch.randn(d, generator=g) if weights else None for _ in range(2)]
    return rows, pos, freq, sections, w


def gpu(*t):
    return [None if x is None else x.cuda() for x in t]


def pair_norms(a, rot, interleaved):
    """|first| + |second| of each element's pair (an element that is not rotated: itself); a [..., d] >= 0."""
    out = a.clone()
    if interleaved:
        s = a[..., 0:rot:2] + a[..., 1:rot:2]
        out[..., 0:rot:2] = s
        out[..., 1:rot:2] = s
    else:
        s = a[..., :rot // 2] + a[..., rot // 2:rot]
        out[..., :rot // 2] = s
        out[..., rot // 2:rot] = s
    return out


@pytest.mark.parametrize("B,N,Hq,Hk,d,dtype,rot,axes,interleaved,norm,weights", ROPE)
def test_norm_rope_forward(ea, B, N, Hq, Hk, d, dtype, rot, axes, interleaved, norm, weights):
    rows, pos, freq, sections, w = rope_inputs(B, N, Hq, Hk, d, dtype, rot, axes, weights)
    dev, p, f, wq, wk = gpu(rows, pos, freq, *w)
    q, k = dev[:, :, :Hq], dev[:, :, Hq:Hq + Hk]                     # views of one projection's rows
    got = ea.entmax_attn_qk_norm_rope_fwd(q, k, p, f, wq, wk, 1e-5, norm, sections, interleaved)
    cos, sin = ref.rotation(pos, freq if rot else torch.zeros(0), sections if rot else [0])
    for y, x, wt in zip(got, (rows[:, :, :Hq], rows[:, :, Hq:Hq + Hk]), w):
        want = ref.prep(x.double(), None if wt is None else wt.double(), cos, sin, interleaved, 1e-5, norm)
        # the sum of squares 12 u, halved by the root with the mean's and eps's 2 u and the root's own 2 u: 9 u; two products
        # 2 u; cosine and sine 4 u absolute (the hardware's 1.3e-7, and the angle's rounding); two products and a sum 2 u each
        flat = ref.prep(x.double(), None if wt is None else wt.double(), cos[..., :0], sin[..., :0], interleaved, 1e-5, norm)
        tol = 20 * U * pair_norms(flat.abs(), rot, interleaved) + rounding(DT[dtype]) * want.abs() * 1.01 + 1e-37
        err = (y.double().cpu() - want).abs()
        assert y.shape == want.shape and y.dtype == DT[dtype] and y.is_contiguous()
        assert (err <= tol).all(), (err / tol).max()
        print("  of allowed", (err / tol).max().item(), flush=True)


@pytest.mark.parametrize("B,N,Hq,Hk,d,dtype,rot,axes,interleaved,norm,weights", ROPE)
def test_norm_rope_gradient(ea, B, N, Hq, Hk, d, dtype, rot, axes, interleaved, norm, weights):
    rows, pos, freq, sections, w = rope_inputs(B, N, Hq, Hk, d, dtype, rot, axes, weights)
    g = torch.Generator().manual_seed(4)
    dys = [torch.randn(B, H, N, d, generator=g) for H in (Hq, Hk)]
    dev, p, f, wq, wk, dq, dk = gpu(rows, pos, freq, *w, *dys)
    q, k = dev[:, :, :Hq], dev[:, :, Hq:Hq + Hk]
    # gradients into views of one buffer laid out like the projection's rows, whose other rows stay as they were
    grad = torch.full_like(dev, 7.0)
    got = ea.entmax_attn_qk_norm_rope_bwd(q, k, dq, dk, p, f, wq, wk, 1e-5, norm, sections, interleaved, out=(grad[:, :, :Hq], grad[:, :, Hq:Hq + Hk]))
    again = ea.entmax_attn_qk_norm_rope_bwd(q, k, dq, dk, p, f, wq, wk, 1e-5, norm, sections, interleaved)
    assert (grad[:, :, Hq + Hk:] == 7).all()
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b)        # in either layout, and from call to call
    cos, sin = ref.rotation(pos, freq if rot else torch.zeros(0), sections if rot else [0])
    tokens = B * N
    per_lane = -(-tokens // (256 // (d // 8)) // 1024) + 1
    for which, (x, wt, dy, H) in enumerate(zip((rows[:, :, :Hq], rows[:, :, Hq:Hq + Hk]), w, dys, (Hq, Hk))):
        x, dy = x.double(), dy.double()
        wd = torch.ones(d, dtype=torch.float64) if wt is None else wt.double()
        gr = ref.rotate(dy.transpose(1, 2), cos, -sin, interleaved)
        big = pair_norms(dy.abs(), rot, interleaved).transpose(1, 2)             # bounds |gr|, and its error by 6 u
        if norm:
            rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
            xh = x * rstd
            want = rstd * (gr * wd - xh * (gr * wd * xh).mean(-1, keepdim=True))
            # g 6 u, times w 1 u; xh 10 u; the mean's products and sum 30 u; the last products and the difference
            tol = 56 * U * rstd * (big * wd.abs() + xh.abs() * (big * wd.abs() * xh.abs()).mean(-1, keepdim=True))
        else:
            want, tol = gr, 8 * U * big
        tol = tol + rounding(DT[dtype]) * want.abs() * 1.01 + 1e-37
        err = (got[which].double().cpu() - want).abs()
        assert (err <= tol).all(), (err / tol).max()
        if wt is None:
            assert got[2 + which] is None
            continue
        dw = (gr * xh).sum((0, 1, 2))
        # a term 17 u; a lane adds up `per_lane` tokens of H heads, then 8 sums of sums, the rest in 64 bits
        tol = (17 + per_lane * H + 8 + 1) * U * (big * xh.abs()).sum((0, 1, 2))
        err = (got[2 + which].double().cpu() - dw).abs()
        assert (err <= tol).all(), (err / tol).max()


def test_norm_rope_gradient_against_differences(ea):
    # <dy, f(x + h v) - f(x - h v)> / 2h of the library's own fp32 forward against <dx, v>
    B, N, H, d = 1, 40, 3, 128
    rows, pos, freq, sections, w = rope_inputs(B, N, H, H, d, "f32", d, 2, True, seed=11)
    dev, p, f, wq, wk = gpu(rows, pos, freq, *w)
    q, k = dev[:, :, :H].contiguous(), dev[:, :, H:2 * H].contiguous()
    g = torch.Generator().manual_seed(5)
    dy, v = torch.randn(B, H, N, d, generator=g).cuda(), torch.randn(B, N, H, d, generator=g).cuda()
    h = 2.0 ** -7
    fw = lambda x: (ea.entmax_attn_qk_norm_rope_fwd(x, k, p, f, wq, wk, 1e-5, True, sections)[0].double() * dy.double())      # noqa: E731
    num = (fw(q + h * v) - fw(q - h * v)).sum() / (2 * h)
    dx = ea.entmax_attn_qk_norm_rope_bwd(q, k, dy, dy, p, f, wq, wk, 1e-5, True, sections)[0]
    got = (dx.double() * v.double()).sum()
    # forward error 20 u sqrt(2) sum|y| / h at most, and h^2 / 6 times the third derivative: |x| is about 3 sqrt(d) and |v| sqrt(d), so
    # that it is below (1/3)^3 * 15 |y| for each element
    size = fw(q).abs().sum()
    assert (num - got).abs() <= size * (20 * U * 2 / h + h * h / 6 * 15 / 27)


def test_norm_rope_rows_that_repeat_and_zero_rows(ea):
    # a batch that is one row repeated (strides of 0), and rows of zeros, which the eps keeps finite
    g = torch.Generator().manual_seed(6)
    one = torch.randn(1, 1, 2, 64, generator=g).cuda()
    one[0, 0, 1] = 0
    q = one.expand(3, 7, 2, 64)
    pos = torch.zeros(3, 7, dtype=torch.int32, device="cuda")
    freq = torch.rand(32, generator=g).cuda()
    y, _ = ea.entmax_attn_qk_norm_rope_fwd(q, q, pos, freq)
    flat, _ = ea.entmax_attn_qk_norm_rope_fwd(q.contiguous(), q.contiguous(), pos, freq)
    assert torch.equal(y, flat) and (y[:, 1] == 0).all()
    dy = torch.randn(3, 2, 7, 64, generator=g).cuda()
    a = ea.entmax_attn_qk_norm_rope_bwd(q, q, dy, dy, pos, freq)
    b = ea.entmax_attn_qk_norm_rope_bwd(q.contiguous(), q.contiguous(), dy, dy, pos, freq)
    assert torch.equal(a[0], b[0]) and torch.isfinite(a[0]).all()
    with pytest.raises(ea.EntmaxAttnError):                         # a gradient cannot be written into repeated rows
        ea.entmax_attn_qk_norm_rope_bwd(q, q, dy, dy, pos, freq, out=(one.expand(3, 7, 2, 64), one.expand(3, 7, 2, 64)))


# ---- the step of a scheduler --------------------------------------------------------------------------------------

def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


class Pair:
    """The library's tables and the reference's, step by step."""

    def __init__(self, ea, R, blocks, page, n_pages, seed):
        self.ea, self.page, self.blocks = ea, page, blocks
        self.rng = np.random.default_rng(seed)
        free = self.rng.permutation(n_pages)
        self.table = torch.full((R, blocks), -1, dtype=torch.int32, device="cuda")
        self.free, self.count = i32(free), i32([n_pages])
        self.want = ref.Scheduler(self.table.tolist(), free, n_pages, page)
        self.lens = [0] * R

    def step(self, new, max_tokens, in_place=False):
        lens = i32(self.lens)
        out = None
        if in_place:
            R = len(self.lens)
            out = (lens,) + tuple(torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (R + 1, max_tokens, max_tokens, 4))
        got = self.ea.entmax_attn_cache_tables(lens, i32(new), self.table, self.free, self.count, self.page, max_tokens, out=out)
        want = self.want.step(self.lens, new, max_tokens)
        for name, a, b in zip(("lens", "start", "slots", "positions", "status"), got, want):
            assert a.tolist() == list(b), name
        assert self.count.item() == self.want.count and self.table.tolist() == self.want.table
        assert self.free.tolist()[:self.want.count] == self.want.stack[:self.want.count]
        self.lens = want[0]
        return want


@pytest.mark.parametrize("R,blocks,page,n_pages,max_tokens", [
    (1, 1, 16, 1, 16), (1, 700, 16, 650, 20000), (3, 5, 64, 9, 200), (64, 16, 32, 300, 4096), (65, 16, 256, 200, 4097), (1000, 40, 16, 9000, 70000),
    (1025, 8, 128, 2000, 100), (4096, 4, 16, 9000, 30000)])
def test_tables_follow_the_scheduler(ea, R, blocks, page, n_pages, max_tokens):
    s = Pair(ea, R, blocks, page, n_pages, seed=R)
    rng, most = s.rng, blocks * page
    refused = 0
    for turn in range(8):
        new = np.array(s.lens)
        what = rng.random(R)
        new = np.where(what < 0.4, np.minimum(new + 1, most), new)
        new = np.where((what > 0.4) & (what < 0.55), 0, new)
        new = np.where((what > 0.55) & (what < 0.8), rng.integers(0, most + 1, R), new)
        if turn == 3:
            new = np.full(R, most)                       # more than there are pages, or rows
        if turn == 5 and R > 2:
            new[R // 2], new[0] = -1, most + 1           # lengths that cannot be
        refused += s.step(new.tolist(), max_tokens, in_place=turn % 2 == 1)[4][1]
    assert refused or R * blocks <= n_pages


def test_tables_step_and_the_step_back(ea):
    s = Pair(ea, 50, 20, 16, 700, seed=8)
    s.step(s.rng.integers(0, 200, 50).tolist(), 20000)
    before = (list(s.lens), s.free.tolist()[:s.want.count], s.count.item())
    new = s.rng.integers(0, 320, 50).tolist()
    s.step(new, 20000)
    s.step(before[0], 20000)
    assert (list(s.lens), s.free.tolist()[:s.want.count], s.count.item()) == before


def test_tables_meet_page_ids_that_cannot_be(ea):
    # a free page and a page of a shrinking request outside the cache: counted, and no slot in them
    table, free, count = i32([[99, -1], [1, -1]]), i32([-7, 0, 2, 3]), i32([1])
    out = ea.entmax_attn_cache_tables(i32([16, 3]), i32([0, 3]), table, free, count, 16, 8)
    assert out[4].tolist() == [0, 0, 0, 1] and count.item() == 2 and free.tolist()[:2] == [-7, 99]
    out = ea.entmax_attn_cache_tables(i32([0, 3]), i32([4, 20]), table, free, count, 16, 40)
    assert out[4].tolist() == [21, 0, 0, 2] and out[2].tolist()[:21] == [-1] * 4 + [16 + k for k in range(3, 16)] + [-1] * 4
    # a count that cannot be is taken as the nearest that can
    out = ea.entmax_attn_cache_tables(i32([0]), i32([40]), i32([[-1] * 4]), i32([5, 4, 3, 2, 1, 0]), i32([77]), 16, 64)
    assert out[0].tolist() == [40] and out[2].tolist()[:3] == [0, 1, 2]


# ---- rows of the 4-bit cache --------------------------------------------------------------------------------------

def special_rows(T, Hk, d, dtype, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, Hk, d)) * np.exp(rng.standard_normal((T, Hk, d // 32, 1)) * 4).repeat(32, -1).reshape(T, Hk, d)
    f = x.reshape(-1, 32)
    put = [np.zeros(32), np.full(32, -0.0), np.r_[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, np.full(24, -1.0)], np.r_[7.0, np.full(31, 0.75)],
           np.r_[-7.03125, np.full(31, 0.5)], np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), -np.inf], np.r_[np.ones(7), np.nan, np.ones(24)],
           np.full(32, 2.0 ** -126), np.full(32, 2.0 ** -127 * 1.5), np.full(32, 3.3e38), np.r_[1e30, np.full(31, 1e-30)], np.full(32, 2.0 ** -133)]
    for i, row in enumerate(put):
        if i < len(f):
            f[(i * 5) % len(f)] = row
    return torch.from_numpy(x.reshape(T, Hk, d)).to(DT[dtype])


@pytest.mark.parametrize("T,Hk,d,dtype,page", [(1, 1, 64, "bf16", 16), (7, 3, 128, "f32", 32), (131, 2, 64, "f32", 64), (1000, 8, 128, "bf16", 128),
                                               (513, 5, 64, "bf16", 256), (300, 1, 128, "f32", 16)])
def test_cache_rows(ea, T, Hk, d, dtype, page):
    rng = np.random.default_rng(T)
    k, v = special_rows(T, Hk, d, dtype, 1), special_rows(T, Hk, d, dtype, 2)
    pages = -(-T // page) + 2
    slots = torch.from_numpy(rng.permutation(pages * page)[:T].astype(np.int32))
    skip = torch.from_numpy(rng.random(T) < 0.1)
    slots[skip] = torch.where(torch.arange(T) % 2 == 0, -1 - torch.arange(T), pages * page + torch.arange(T))[skip].to(torch.int32)
    # rows of a projection's output: keys and values side by side, tokens apart
    both = torch.stack([k, v], 1).cuda()
    cache = ea.entmax_attn_cache4_empty(pages, Hk, d, page)
    cache.fill_(0xA5)
    ea.entmax_attn_cache4_write(both[:, 0], both[:, 1], slots.cuda(), cache, page)
    want = np.full((2, pages * page, Hk, d), np.nan)
    raw = ref.decode_cache(np.full(cache.shape, 0xA5, np.uint8), d, page)
    for w, x in enumerate((k, v)):
        want[w] = raw[w].transpose(0, 2, 1, 3).reshape(pages * page, Hk, d)      # slots that no row went to
        want[w][slots[~skip].numpy()] = ref.quantise(x[~skip].double().numpy())[2]
    got = ref.decode_cache(cache.cpu().numpy(), d, page)
    for w in range(2):
        np.testing.assert_array_equal(got[w].transpose(0, 2, 1, 3).reshape(pages * page, Hk, d), want[w])
    # read back in both types, into rows of other strides, rows of other slots left as they were
    for dt in (torch.bfloat16, torch.float32):
        out = torch.full((2, Hk, T, d), 3.0, dtype=dt, device="cuda")
        ea.entmax_attn_cache4_read(cache, slots.cuda(), page, d, out=(out[0].transpose(0, 1), out[1].transpose(0, 1)))
        exp = np.full((2, T, Hk, d), 3.0)
        exp[:, ~skip.numpy()] = want[:, slots[~skip].numpy()]
        np.testing.assert_array_equal(out.double().cpu().numpy().transpose(0, 2, 1, 3), exp)


def test_cache_rows_none_and_zero_page(ea):
    cache = ea.entmax_attn_cache4_empty(2, 1, 64, 16)
    none = torch.zeros(0, 1, 64, device="cuda")
    slots = torch.zeros(0, dtype=torch.int32, device="cuda")
    ea.entmax_attn_cache4_write(none, none, slots, cache, 16)
    k, v = ea.entmax_attn_cache4_read(cache, slots, 16, 64)
    assert k.shape == (0, 1, 64) and (cache == 0).all()
    k, v = ea.entmax_attn_cache4_read(cache, i32([0, 31]), 16, 64)
    assert (k == 0).all() and (v == 0).all()


def test_strides_of_dimensions_of_one(ea):
    """A channels-first layer's output of one token: torch leaves the dimension of one a stride that no row could have."""
    g = torch.Generator().manual_seed(8)
    x = torch.randn(6, 64, 1, generator=g).cuda().transpose(1, 2)                # [6,1,64], strides 64, 1, 1
    assert x.stride() == (64, 1, 1)
    slots, cache, same = i32([3, 9, 0, 17, 31, 8]), ea.entmax_attn_cache4_empty(2, 1, 64, 16), ea.entmax_attn_cache4_empty(2, 1, 64, 16)
    ea.entmax_attn_cache4_write(x, x, slots, cache, 16)
    y = torch.empty(6, 1, 64, device="cuda").copy_(x)
    ea.entmax_attn_cache4_write(y, y, slots, same, 16)
    assert torch.equal(cache, same)
    out = [torch.full((6, 64, 1), 3.0, device="cuda").transpose(1, 2) for _ in range(2)]
    ea.entmax_attn_cache4_read(cache, slots, 16, 64, out=out)
    for a, b in zip(out, ea.entmax_attn_cache4_read(cache, slots, 16, 64, torch.float32)):
        assert torch.equal(a, b)
    q, r = x.as_strided((6, 1, 1, 64), (64, 1, 3, 1)), y.view(6, 1, 1, 64)
    pos, freq, dy = i32([[5]] * 6), torch.rand(32, generator=g).cuda(), torch.randn(6, 1, 1, 64, generator=g).cuda()
    for a, b in zip(ea.entmax_attn_qk_norm_rope_fwd(q, q, pos, freq), ea.entmax_attn_qk_norm_rope_fwd(r, r, pos, freq)):
        assert torch.equal(a, b)
    grads = [torch.empty(6 * 64, device="cuda").as_strided((6, 1, 1, 64), (64, 1, 3, 1)) for _ in range(2)]
    ea.entmax_attn_qk_norm_rope_bwd(q, q, dy, dy, pos, freq, out=grads)
    for a, b in zip(grads, ea.entmax_attn_qk_norm_rope_bwd(r, r, dy, dy, pos, freq)):
        assert torch.equal(a, b)


# ---- decode from the cache ----------------------------------------------------------------------------------------

def make_cache(ea, lens, Hk, d, page, sigma, seed, keys=None, spare=3):
    """Requests' keys and values written through the library; garbage (NaN scales among it) in every slot that holds none."""
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    blocks = max(max(need), 1) + 1
    order = rng.permutation(sum(need) + spare)
    table = torch.full((len(lens), blocks), -1, dtype=torch.int32)
    cache = ea.entmax_attn_cache4_empty(sum(need) + spare, Hk, d, page)
    cache.copy_(torch.randint(0, 256, cache.shape, generator=g, dtype=torch.uint8))
    cache[:, :, ::7] = 255
    at, ks, vs = 0, [], []
    for r, n in enumerate(lens):
        table[r, :need[r]] = torch.from_numpy(order[at:at + need[r]].astype(np.int32))
        at += need[r]
        k = (torch.randn(n, Hk, d, generator=g) * sigma) if keys is None else keys(r, n, g)
        v = torch.randn(n, Hk, d, generator=g)
        pos = torch.arange(n)
        slots = (table[r, pos // page] * page + pos % page).to(torch.int32)
        ea.entmax_attn_cache4_write(k.cuda(), v.cuda(), slots.cuda(), cache, page)
        ks.append(ref.quantise(k.double().numpy())[2])
        vs.append(ref.quantise(v.double().numpy())[2])
    return cache, table.cuda(), i32(lens), ks, vs


def check_decode(q, ks, vs, alpha, O, tau, support, dtype):
    """q [R, Hq, d]; against the float64 oracle.  What the kernel may differ by: a score is a sum of d products in fp32, off by at
    most d u sum |q k| in any order, plus what the 8-bit terms leave of elements far below their row's largest; scores enter the solve as
    c (s - max), 4 u more; the threshold moves by at most as much as the scores, and by what F = 1 is known to: a
    power is off by (2 + 2 r) u relative (r times the logarithm's half step over the range that counts), a sum of n
    terms by its 12 levels: 2e-6 covers both for r <= 4, r / 4 of it above."""
    from oracle import entmax_oracle as eo
    R, Hq, d = q.shape
    r = 1 / (alpha - 1)
    worst = 0.0
    for i in range(R):
        n, Hk = ks[i].shape[:2]
        if n == 0:
            assert (O[i] == 0).all() and (tau[i] == 0).all() and (support[i] == 0).all()
            continue
        G = Hq // Hk
        K, V = (np.repeat(x.transpose(1, 0, 2), G, 0)[None] for x in (ks[i], vs[i]))
        qi = q[i].double().numpy()[None]
        want = eo.attn_decode(qi, K, V, alpha)
        c = (alpha - 1) / np.sqrt(d)
        small = np.abs(qi) < np.abs(qi).max(-1, keepdims=True) * 2.0 ** (-12 if dtype == "bf16" else -6)
        lost = np.abs(qi).max(-1, keepdims=True) * (2.0 ** -20 if dtype == "bf16" else 2.0 ** -30) * small
        ds = d * U * (np.abs(K) @ np.abs(qi)[..., None])[..., 0] + (np.abs(K) @ lost[..., None])[..., 0]
        eta = 2 * c * ds.max(-1, keepdims=True) + 4 * U + 2e-6 * max(1.0, r / 4)
        x = (alpha - 1) * want["z"] - want["tau"][..., None]
        p = lambda y: np.maximum(y, 0) ** r               # noqa: E731
        dp = np.maximum(p(x + eta) - p(x), p(x) - p(x - eta))
        tol = ((dp + (24 + 4 * r) * U * p(x))[..., None] * np.abs(V)).sum(2)
        err = np.abs(O[i].double().numpy() - want["O"][0])
        assert (err <= tol[0]).all(), (i, n, (err / tol[0]).max())
        terr = np.abs(tau[i].double().numpy() - want["tau"][0])
        assert (terr <= eta[0, :, 0] + 2 * U * np.abs(want["tau"][0])).all(), (i, n, terr.max())
        got = support[i].numpy()
        assert ((got >= (x > eta).sum(-1)[0]) & (got <= (x > -eta).sum(-1)[0])).all() or r > 8
        worst = max(worst, (err / (tol[0] + 1e-300)).max())
        print(f"  request {i} n={n} |dO| {err.max():.2e} |dtau| {terr.max():.2e} support {got.mean():.1f}", flush=True)
    return worst


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
    ([2000], 2, 1, 128, "f32", 16, 1.004, 1.5),                # r = 250
    ([100, 0, 1000, 17], 8, 1, 64, "f32", 16, 1.5, 1.5),       # eight heads side by side twice, and one more than that
    ([100, 1000], 9, 1, 64, "bf16", 32, 1.75, 1.5),
    ([7 * i for i in range(40)], 16, 2, 64, "bf16", 64, 1.5, 1.5),             # 640 heads: four waves each in the second kernel
    ([33 * i for i in range(1, 34)], 16, 1, 128, "bf16", 32, 1.25, 1.0),
    ([70000], 8, 2, 64, "bf16", 128, 1.5, 1.5),
]


@pytest.mark.parametrize("lens,Hq,Hk,d,dtype,page,alpha,sigma", DECODE)
def test_decode_from_the_cache(ea, lens, Hq, Hk, d, dtype, page, alpha, sigma):
    cache, table, ln, ks, vs = make_cache(ea, lens, Hk, d, page, sigma, seed=sum(lens) + d)
    g = torch.Generator().manual_seed(9)
    q = (torch.randn(len(lens), Hq, d, generator=g) * sigma).to(DT[dtype])
    got = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, ln, alpha, page)
    again = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, ln, alpha, page)
    short = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, ln, alpha, page, max_len=max(lens))
    for a, b in zip(got, again):
        assert torch.equal(a, b)                                   # bit for bit
    assert (got[0] - short[0]).abs().max() <= 1e-4                 # (another split over the waves)
    check_decode(q, ks, vs, alpha, *(t.cpu() for t in got), dtype)


def test_decode_queries_of_wide_range(ea):
    # elements far below the largest of their row, the largest and smallest rows, zeros
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
        got = ea.entmax_attn_decode_cache4(x.cuda(), cache, table, ln, 1.5, page)
        check_decode(x, ks, vs, 1.5, *(t.cpu() for t in got), dtype)


def test_decode_marks_what_it_cannot_answer(ea):
    lens, d, page = [40, 40, 40, 40, 40, 40], 64, 16
    cache, table, ln, ks, vs = make_cache(ea, lens, 1, d, page, 1.0, seed=32)
    q = torch.randn(6, 2, d, generator=torch.Generator().manual_seed(1)).cuda()
    clean = ea.entmax_attn_decode_cache4(q, cache, table, ln, 1.5, page, max_len=48)
    ln = i32([40, -1, 49, 40, 40, 40])
    bad = table.clone()
    bad[3, 1] = cache.shape[0]
    bad[4, 2] = -5
    q2 = q.clone()
    q2[5, 1, 3] = float("inf")
    got = ea.entmax_attn_decode_cache4(q2, cache, bad, ln, 1.5, page, max_len=48)
    for r in range(1, 5):
        assert torch.isnan(got[0][r]).all() and torch.isnan(got[1][r]).all() and (got[2][r] == -1).all(), r
    assert torch.isnan(got[0][5, 1]).all() and got[2][5, 1] == -1
    assert torch.equal(got[0][0], clean[0][0]) and torch.equal(got[0][5, 0], clean[0][5, 0])
    # a key that is not finite, seen and behind the end
    k = torch.randn(1, 1, d).cuda()
    k[0, 0, 5] = float("nan")
    ea.entmax_attn_cache4_write(k, k, i32([int(table[0, 2]) * page + 7]), cache, page)
    got = ea.entmax_attn_decode_cache4(q, cache, table, i32([40, 40, 40, 40, 40, 40]), 1.5, page)
    assert torch.isnan(got[0][0]).all() and torch.isfinite(got[0][1:]).all()
    got = ea.entmax_attn_decode_cache4(q, cache, table, i32([39, 40, 40, 40, 40, 40]), 1.5, page)
    assert torch.isfinite(got[0]).all()


@pytest.mark.parametrize("alpha", [1.001, 1.0001, 1.00001])
def test_decode_with_alpha_next_to_one(ea, alpha):
    """r = 1 / (alpha - 1) is the power of the probabilities, up to 1e5 here: y is rounded by 2 u, its logarithm (log2, 2^-22 at the
    most) by 4 u, the exponent of up to 64 by 64 u; a score's error d u sum |q k| counts 1 / sqrt(d) each in p and in
    the largest score.  The sum of the p that O is divided by doubles it all."""
    from oracle import entmax_oracle as eo
    alpha = float(np.float32(alpha))
    r, d = 1 / (alpha - 1), 64
    cache, table, lens, ks, vs = make_cache(ea, [1500], 1, d, 32, 1.0, 17)
    q = torch.randn(1, 2, d, generator=torch.Generator().manual_seed(5))
    O, tau, support = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, lens, alpha, 32)
    K, V = (np.repeat(x[0].transpose(1, 0, 2), 2, 0)[None] for x in (ks, vs))
    want = eo.attn_decode(q.double().numpy(), K, V, alpha)
    ds = d * U * (np.abs(K[0]) @ np.abs(q[0].double().numpy())[..., None]).max() + 2.0 ** -30 * np.abs(K).sum(-1).max() * q.abs().max().item()
    tol = 2 * (6 * r * U + (64 + 24) * U + 2 * ds / np.sqrt(d))
    err = np.abs(O[0].double().cpu().numpy() - want["O"][0]) / np.einsum("hn,hnd->hd", want["P"][0], np.abs(V[0]))
    assert (err <= tol).all(), (err.max(), tol)
    print("  of allowed", err.max() / tol, flush=True)


@pytest.mark.parametrize("alpha", [1.5, 1.9999, 2.0, 3.0])
def test_decode_of_the_longest_request_with_equal_scores(ea, alpha):
    """2^22 keys of zero, one page serving for all: tau = -N^(-1/r), as close to the maximum as it can be, and every p = 1/N."""
    N, r = 1 << 22, 1 / (alpha - 1)
    cache = ea.entmax_attn_cache4_empty(1, 1, 64, 256)
    ea.entmax_attn_cache4_write(torch.zeros(256, 1, 64, device="cuda"), torch.ones(256, 1, 64, device="cuda"), i32(list(range(256))), cache, 256)
    table = torch.zeros(1, N // 256, dtype=torch.int32, device="cuda")
    O, tau, support = ea.entmax_attn_decode_cache4(torch.ones(1, 1, 64, device="cuda"), cache, table, i32([N]), alpha, 256)
    # a lane adds up to N / 8 / 32 of the output's terms and N / 8 / 64 of the p and of the solve's, then 64 over lanes and waves;
    # F = N (-tau)^r: an error of F is r times tau's relative one.  The solve ends where a step is below 3e-8 (or 26 halvings)
    assert (support == N).all()
    assert ((O - 1).abs() <= (N // 256 + N // 512 + 64) * U).all(), O
    want = -float(N) ** (-1 / r)
    assert (tau.double().cpu() - want).abs().item() <= abs(want) * (N // 512 + 64) * U / r + 6e-8, (tau, want)


def test_decode_agrees_with_the_decode_of_a_contiguous_cache(ea):
    R, H, n, d, page = 2, 4, 777, 128, 64
    cache, table, ln, ks, vs = make_cache(ea, [n] * R, H, d, page, 1.5, seed=33)
    q = (1.5 * torch.randn(R, H, d, generator=torch.Generator().manual_seed(2))).to(torch.bfloat16)
    pos = torch.arange(n, device="cuda")
    K, V = torch.empty(2, R, H, n, d, dtype=torch.bfloat16, device="cuda")
    for r in range(R):
        slots = (table[r, pos // page] * page + pos % page).to(torch.int32)
        ea.entmax_attn_cache4_read(cache, slots, page, d, out=(K[r].transpose(0, 1), V[r].transpose(0, 1)))
    a = ea.entmax_attn_decode(q.cuda(), K, V, 1.5)
    b = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, ln, 1.5, page)
    # both are held to the oracle; the other one stops its solve at 1e-4 of tau
    assert (a[0] - b[0]).abs().max() <= 2e-3 and (a[1] - b[1]).abs().max() <= 2e-4


# ---- in turn ------------------------------------------------------------------------------------------------------

class Serving:
    """A layer of a served model, step by step: projections -> norm and rotation -> cache -> decode."""

    def __init__(self, ea, R, Hq, Hk, d, page, n_pages, blocks, max_tokens):
        self.ea, self.shape, self.page, self.max_tokens = ea, (R, Hq, Hk, d), page, max_tokens
        dev = dict(dtype=torch.int32, device="cuda")
        self.lens, self.table = torch.zeros(R, **dev), torch.full((R, blocks), -1, **dev)
        self.free, self.count = torch.arange(n_pages, **dev), torch.full((1,), n_pages, **dev)
        self.cache = ea.entmax_attn_cache4_empty(n_pages, Hk, d, page)
        self.out = tuple(torch.empty(n, **dev) for n in (R, R + 1, max_tokens, max_tokens, 4))
        self.freq = torch.pow(10000.0, -torch.arange(d // 2, dtype=torch.float64) / (d // 2)).float().cuda()
        self.w = (1 + 0.1 * torch.randn(2, d, generator=torch.Generator().manual_seed(0))).cuda()
        self.ws = torch.empty(ea.entmax_attn_decode_cache4_workspace_bytes(R, Hq, Hk, d, blocks * page), dtype=torch.uint8, device="cuda")

    def step(self, new, rows):
        """new [R]: lengths after the step; rows [max_tokens, Hq + 2 Hk, d]: projections of the new tokens.  Attends with the last new
        token of each request."""
        ea, (R, Hq, Hk, d) = self.ea, self.shape
        lens, start, slots, positions, status = ea.entmax_attn_cache_tables(self.lens, new, self.table, self.free, self.count, self.page,
                                                                            self.max_tokens, out=(self.lens,) + self.out[1:])
        x = rows[:, None]
        q, k = ea.entmax_attn_qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq:Hq + Hk], positions[:, None], self.freq, self.w[0], self.w[1])
        ea.entmax_attn_cache4_write(k[:, :, 0], rows[:, Hq + Hk:], slots, self.cache, self.page)
        last = (start[1:] - 1).clamp(min=0)
        q = q[:, :, 0].index_select(0, last)
        return ea.entmax_attn_decode_cache4(q, self.cache, self.table, lens, 1.5, self.page, workspace=self.ws)


def serving_reference(s, history, rows_of_last):
    """O of the last step in 64 bits from the projections of all tokens: [R, Hq, d].  K as the library's own bf16 holds it goes into
    the rounding to 4 bits, whose borders a difference of one bf16 step can cross."""
    ea, (R, Hq, Hk, d) = s.ea, s.shape
    qs, ks, vs = [], [], []
    for r in range(R):
        x = history[r][:, None]                                      # [n, 1, heads, d]
        pos = torch.arange(x.shape[0], dtype=torch.int32, device="cuda")[:, None]
        q, k = ea.entmax_attn_qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq:Hq + Hk], pos, s.freq, s.w[0], s.w[1])
        cos, sin = ref.rotation(pos.cpu()[None], s.freq.cpu(), [d // 2])
        want = ref.prep(x[:, :, Hq:Hq + Hk].cpu().double(), s.w[1].cpu().double(), cos, sin, False, 1e-6, True)
        assert (k.cpu().double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() * 1.01
        qs.append(q[-1, :, 0].cpu())
        ks.append(ref.quantise(k[:, :, 0].cpu().double().numpy())[2])
        vs.append(ref.quantise(x[:, 0, Hq + Hk:].cpu().double().numpy())[2])
    return torch.stack(qs), ks, vs


def test_serving_steps(ea):
    # prompts, then a token each, a request that ends and one that starts, a draft taken back: every step against a
    # recomputation from the projections of all its tokens
    R, Hq, Hk, d, page = 3, 8, 2, 64, 16
    s = Serving(ea, R, Hq, Hk, d, page, n_pages=40, blocks=12, max_tokens=200)
    g = torch.Generator(device="cuda").manual_seed(3)
    history = [torch.zeros(0, Hq + 2 * Hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(R)]
    for new in ([50, 16, 1], [51, 17, 2], [52, 18, 3], [53, 100, 4], [54, 90, 5], [55, 0, 6], [56, 33, 100], [57, 34, 101]):
        rows = torch.randn(s.max_tokens, Hq + 2 * Hk, d, generator=g, device="cuda").to(torch.bfloat16)
        rows[199] = float("nan")                                     # rows behind the last one are padding
        at = 0
        for r, n in enumerate(new):
            grow = max(0, n - len(history[r]))
            history[r] = torch.cat([history[r], rows[at:at + grow]])[:n]
            at += grow
        O, tau, support = s.step(i32(new), rows)
        if any(n == 0 for n in new) or new[1] == 90:                 # (nothing new to attend with in one of them)
            continue
        q, ks, vs = serving_reference(s, history, rows)
        check_decode(q, ks, vs, 1.5, O.cpu(), tau.cpu(), support.cpu(), "bf16")


def test_serving_step_captured_and_replayed(ea):
    # one step as a graph, replayed with other lengths and rows, with eager work and synchronisation between the replays
    R, Hq, Hk, d, page = 4, 8, 2, 128, 16
    eager, graphed = (Serving(ea, R, Hq, Hk, d, page, n_pages=60, blocks=10, max_tokens=R) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(4)
    new, rows = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, Hq + 2 * Hk, d, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graphed.step(new, rows)                                      # (all lengths 0: changes nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, tau, support = graphed.step(new, rows)
    for step in range(1, 40):
        new.fill_(step)
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        graph.replay()
        want = eager.step(new, rows)
        torch.cuda.synchronize()
        for a, b in zip((O, tau, support), want):
            assert torch.equal(a, b), step
        assert torch.equal(eager.cache, graphed.cache)
        torch.randn(1000, device="cuda").sum().item()


def test_two_decodes_at_once_and_on_another_stream(ea):
    cache, table, ln, ks, vs = make_cache(ea, [3000, 500], 2, 128, 32, 1.5, seed=40)
    g = torch.Generator().manual_seed(12)
    qa, qb = ((1.5 * torch.randn(2, 8, 128, generator=g)).to(torch.bfloat16).cuda() for _ in range(2))
    wa, wb = (ea.entmax_attn_decode_cache4(x, cache, table, ln, 1.5, 32) for x in (qa, qb))
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    n = ea.entmax_attn_decode_cache4_workspace_bytes(2, 8, 2, 128, table.shape[1] * 32)
    ws = torch.empty(2, n, dtype=torch.uint8, device="cuda")
    for _ in range(5):
        with torch.cuda.stream(sa):
            a = ea.entmax_attn_decode_cache4(qa, cache, table, ln, 1.5, 32, workspace=ws[0])
        with torch.cuda.stream(sb):
            b = ea.entmax_attn_decode_cache4(qb, cache, table, ln, 1.5, 32, workspace=ws[1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a + b, wa + wb))


def test_training_step_through_norm_rotation_and_attention(ea):
    # projections -> norm and rotation -> entmax attention -> its gradient -> the gradient of norm and rotation, against
    # automatic differentiation of the whole in 64 bits
    B, N, H, d, alpha = 1, 128, 2, 64, 1.5
    g = torch.Generator().manual_seed(21)
    rows = torch.randn(B, N, 3 * H, d, generator=g)
    w = 1 + 0.2 * torch.randn(2, d, generator=g)
    do = torch.randn(B, H, N, d, generator=g)
    pos = torch.arange(N, dtype=torch.int32)[None]
    freq = torch.pow(10000.0, -torch.arange(d // 2, dtype=torch.float64) / (d // 2)).float()
    x, wd, p, f, dod = gpu(rows, w, pos, freq, do)
    q, k = ea.entmax_attn_qk_norm_rope_fwd(x[:, :, :H], x[:, :, H:2 * H], p, f, wd[0], wd[1])
    v = x[:, :, 2 * H:].transpose(1, 2).contiguous()
    O, tau, mask = ea.entmax_attn_fwd(q, k, v, alpha, True)
    dQ, dK, dV = ea.entmax_attn_bwd(q, k, v, O, dod, tau, alpha, True, block_mask=mask)
    dq, dk, dwq, dwk = ea.entmax_attn_qk_norm_rope_bwd(x[:, :, :H], x[:, :, H:2 * H], dQ, dK, p, f, wd[0], wd[1])
    X, W = rows.double().requires_grad_(True), w.double().requires_grad_(True)
    cos, sin = ref.rotation(pos[None], freq, [d // 2])
    Q = ref.prep(X[:, :, :H], W[0], cos, sin, False, 1e-6, True)
    K = ref.prep(X[:, :, H:2 * H], W[1], cos, sin, False, 1e-6, True)
    s = (Q @ K.mT) * (alpha - 1) / d ** 0.5
    s = s.masked_fill(torch.ones(N, N).triu(1).bool(), -float("inf"))
    top = torch.sort(s, -1, descending=True).values
    n = torch.arange(1, N + 1).double()
    safe = torch.where(torch.isinf(top), torch.full_like(top, -1e3), top)
    mean, square = safe.cumsum(-1) / n, (safe * safe).cumsum(-1) / n
    t = mean - torch.sqrt(((1 / n) - (square - mean * mean)).clamp(min=1e-30))
    size = ((t <= safe) & ~torch.isinf(top)).sum(-1, keepdim=True)
    want_o = (s - t.gather(-1, size - 1)).clamp(min=0) ** 2 @ X[:, :, 2 * H:].transpose(1, 2)
    grads = torch.autograd.grad((want_o * do.double()).sum(), (X, W))
    # the attention's own bars in fp32: 1e-5 on O, 1e-5 (1 + |gradient|) on its gradients, which the norm's gradient scales by
    # rstd |w| and adds up over a head (64 elements) and, for the weights, over all rows
    assert (O.double().cpu() - want_o).abs().max() <= 2e-5
    scale = 1e-5 * (1 + grads[0].abs().max())
    got = torch.cat([dq, dk], 2).double().cpu()
    assert (got - grads[0][:, :, :2 * H]).abs().max() <= 8 * scale
    assert (dV.transpose(1, 2).double().cpu() - grads[0][:, :, 2 * H:]).abs().max() <= scale
    assert (torch.stack([dwq, dwk]).double().cpu() - grads[1]).abs().max() <= 1e-5 * N * H * 3


def test_chunked_prefill_attends_to_the_cache_as_it_is(ea):
    # the keys of a prompt are written to the cache, read back and attended to by entmax_attn_fwd: the last row equals the decode
    N, H, d, page = 192, 2, 64, 64
    g = torch.Generator().manual_seed(22)
    q, k, v = ((1.5 * torch.randn(1, H, N, d, generator=g)).to(torch.bfloat16).cuda() for _ in range(3))
    cache = ea.entmax_attn_cache4_empty(3, H, d, page)
    slots = i32(list(range(N)))
    ea.entmax_attn_cache4_write(k[0].transpose(0, 1), v[0].transpose(0, 1), slots, cache, page)
    K, V = torch.empty_like(k), torch.empty_like(v)
    ea.entmax_attn_cache4_read(cache, slots, page, d, out=(K[0].transpose(0, 1), V[0].transpose(0, 1)))
    O, tau, _ = ea.entmax_attn_fwd(q, K, V, 1.5, True)
    o, t, _ = ea.entmax_attn_decode_cache4(q[:, :, -1].contiguous(), cache, i32([[0, 1, 2]]), i32([N]), 1.5, page)
    assert (O[:, :, -1] - o).abs().max() <= 1e-2 and (tau[:, :, -1] - t).abs().max() <= 1e-3      # the forward's bars for bf16


# ---- past 2^32 bytes ----------------------------------------------------------------------------------------------

def test_cache_beyond_four_gigabytes(ea):
    # pages at the end of a cache of 5.6 GB
    Hk, d, page, n, pages = 8, 128, 256, 600, 20000
    cache = ea.entmax_attn_cache4_empty(pages, Hk, d, page)
    assert cache.numel() > 2 ** 32
    ids = [pages - 1, pages // 2, pages - 7]
    g = torch.Generator().manual_seed(50)
    k, v = torch.randn(n, Hk, d, generator=g), torch.randn(n, Hk, d, generator=g)
    pos = torch.arange(n)
    slots = (torch.tensor(ids)[pos // page] * page + pos % page).to(torch.int32).cuda()
    ea.entmax_attn_cache4_write(k.cuda(), v.cuda(), slots, cache, page)
    K, V = ea.entmax_attn_cache4_read(cache, slots, page, d, torch.float32)
    ks, vs = ref.quantise(k.double().numpy())[2], ref.quantise(v.double().numpy())[2]
    np.testing.assert_array_equal(K.double().cpu().numpy(), ks)
    np.testing.assert_array_equal(V.double().cpu().numpy(), vs)
    q = torch.randn(1, 16, d, generator=g).to(torch.bfloat16)
    got = ea.entmax_attn_decode_cache4(q.cuda(), cache, i32([ids]), i32([n]), 1.5, page)
    check_decode(q, [ks], [vs], 1.5, *(t.cpu() for t in got), "bf16")


def test_norm_rope_beyond_two_gigabytes(ea):
    # the last tokens of 262144 with 66 rows each: 4.4 GB in and out
    N, Hq, Hk, d = 262144, 64, 2, 128
    rows = torch.randn(1, N, Hq + Hk, d, device="cuda", dtype=torch.bfloat16, generator=torch.Generator(device="cuda").manual_seed(51))
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[None]
    freq = torch.rand(d // 2, generator=torch.Generator().manual_seed(52))
    q, k = ea.entmax_attn_qk_norm_rope_fwd(rows[:, :, :Hq], rows[:, :, Hq:], pos, freq.cuda())
    assert rows.numel() > 2 ** 31                                   # (elements; q_out has 2 ** 32 bytes)
    cos, sin = ref.rotation(pos[None, :, -3:].cpu(), freq, [d // 2])
    for y, x in ((q, rows[:, -3:, :Hq]), (k, rows[:, -3:, Hq:])):
        want = ref.prep(x.cpu().double(), None, cos, sin, False, 1e-6, True)
        err = (y[:, :, -3:].cpu().double() - want).abs()
        assert (err <= 2.0 ** -8 * want.abs() * 1.01 + 20 * U * pair_norms(want.abs(), d, False) * 2 + 1e-37).all()
    dy = torch.randn(1, Hq, N, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(53))
    dk = torch.zeros(1, Hk, N, d, device="cuda")
    dq = ea.entmax_attn_qk_norm_rope_bwd(rows[:, :, :Hq], rows[:, :, Hq:], dy, dk, pos, freq.cuda())[0]
    part = ea.entmax_attn_qk_norm_rope_bwd(rows[:, -3:, :Hq], rows[:, -3:, Hq:], dy[:, :, -3:].contiguous(), dk[:, :, -3:].contiguous(),
                                           pos[:, -3:].contiguous(), freq.cuda())[0]
    assert torch.equal(dq[:, -3:], part)
