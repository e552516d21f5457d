"""Host-only checks of the operators beside the attention: what their entry points refuse, and the definitions the GPU tests
compare with against each other (differences for the gradient, brute force for the 4-bit rounding)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2604_15180_amd as ea
from tests import operators_ref as ref

NULL, ALPHA, SHAPE, DTYPE, WORKSPACE, LAYOUT = -1, -2, -3, -4, -5, -8
A = 0x1000                                                   # never dereferenced: every call below is refused


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(ea.lib_path()):
        from paper_2604_15180_amd import build
        build.build()
    return ea.lib()


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def fwd(L, q=A, k=A, qo=A, ko=A, qs=(64, 64, 64), ks=(64, 64, 64), wq=None, wk=None, pos=A, freq=A, B=1, Hq=1, Hk=1, N=1, d=64, t=1,
        rot=64, axes=1, sections=None, norm=1, eps=1e-6):
    sec = (ctypes.c_int * len(sections))(*sections) if sections else None
    return L.entmax_attn_qk_norm_rope_fwd(q, k, qo, ko, qs and i64(*qs), ks and i64(*ks), wq, wk, pos, freq, B, Hq, Hk, N, d, t, rot, axes, sec,
                                          0, norm, eps, None)


def test_norm_rope_refusals(L):
    for missing in ("q", "k", "qo", "ko", "qs", "ks", "pos", "freq"):
        assert fwd(L, **{missing: None}) == NULL, missing
    assert fwd(L, t=2) == DTYPE
    for bad in (dict(B=0), dict(N=0), dict(Hq=0), dict(Hk=-1), dict(d=96), dict(d=32), dict(rot=66), dict(rot=68), dict(rot=-8), dict(axes=0),
                dict(axes=5, sections=(8, 8, 8, 4, 4)), dict(axes=2, sections=(16, 15)), dict(axes=2, sections=(40, -8)), dict(sections=(31,)),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(norm=0, wq=A), dict(B=1 << 14, N=1 << 14)):
        assert fwd(L, **bad) == SHAPE, bad
    assert fwd(L, axes=2) == NULL                            # several axes without sections
    for bad in (dict(q=A + 8), dict(ko=A + 4), dict(qs=(64, 64, 4)), dict(ks=(64, -64, 64)), dict(qs=(64, 2, 64), t=0), dict(wq=A + 4)):
        assert fwd(L, **bad) == LAYOUT, bad
    assert ea.entmax_attn_qk_norm_rope_workspace_bytes(96) == 0 and ea.entmax_attn_qk_norm_rope_workspace_bytes(64) % 256 == 0


def bwd(L, dqo=A, dko=A, dq=A, dk=A, ds=(1024, 128, 64), dks=(1024, 128, 64), dwq=None, dwk=None, B=2, Hq=2, Hk=2, N=8, ws=A, nbytes=1 << 30, norm=1):
    st = i64(1024, 128, 64)
    return L.entmax_attn_qk_norm_rope_bwd(A, A, dqo, dko, dq, dk, st, st, ds and i64(*ds), dks and i64(*dks), None, None, A, A, dwq, dwk,
                                          B, Hq, Hk, N, 64, 1, 64, 1, None, 0, norm, 1e-6, ws, nbytes, None)


def test_norm_rope_gradient_refusals(L):
    for missing in ("dqo", "dko", "dq", "dk", "ds", "dks"):
        assert bwd(L, **{missing: None}) == NULL, missing
    assert bwd(L, dwq=A, ws=None) == WORKSPACE
    assert bwd(L, dwq=A, ws=A + 64) == WORKSPACE
    assert bwd(L, dwk=A, nbytes=256) == WORKSPACE
    assert bwd(L, dwk=A, norm=0) == SHAPE
    # rows of a gradient that overlap: repeated, or with steps smaller than what lies inside them
    for bad in ((0, 128, 64), (1024, 128, 0), (1024, 64, 64), (512, 128, 64), (1024, 128, 32), (64, 64, 1024)):
        assert bwd(L, ds=bad) == LAYOUT, bad
        assert bwd(L, dks=bad) == LAYOUT, bad


def tables(L, lens=A, new=A + 64, table=A, free=A, count=A, out=A, start=A, slots=A, positions=A, status=A, R=1, blocks=4, page=16, pages=8, rows=4):
    return L.entmax_attn_cache_tables(lens, new, table, free, count, out, start, slots, positions, status, R, blocks, page, pages, rows, None)


def test_tables_refusals(L):
    for missing in ("lens", "new", "table", "free", "count", "out", "start", "slots", "positions", "status"):
        assert tables(L, **{missing: None}) == NULL, missing
    for bad in (dict(R=0), dict(R=4097), dict(blocks=0), dict(page=8), dict(page=48), dict(page=512), dict(pages=0), dict(rows=-1),
                dict(rows=(1 << 30) + 1), dict(blocks=1 << 20, page=16), dict(pages=1 << 27, page=16)):
        assert tables(L, **bad) == SHAPE, bad
    assert tables(L, out=A + 64) == LAYOUT                   # lens_out over new_lens


def rows(f, k=A, v=A, ks=(64, 64), vs=(64, 64), slots=A, cache=A, T=1, Hk=1, d=64, t=1, pages=4, page=16):
    a = (k, v, ks and i64(*ks), vs and i64(*vs), slots, cache)
    if f.__name__.endswith("read"):
        a = (cache, slots, k, v, ks and i64(*ks), vs and i64(*vs))
    return f(*a, T, Hk, d, t, pages, page, None)


def test_cache_row_refusals(L):
    for f in (L.entmax_attn_cache4_write, L.entmax_attn_cache4_read):
        for missing in ("k", "v", "ks", "vs", "slots", "cache"):
            assert rows(f, **{missing: None}) == NULL, missing
        assert rows(f, t=9) == DTYPE
        for bad in (dict(T=-1), dict(Hk=0), dict(d=32), dict(page=24), dict(pages=0), dict(pages=1 << 27), dict(T=1 << 30, Hk=64)):
            assert rows(f, **bad) == SHAPE, bad
        for bad in (dict(k=A + 8), dict(cache=A + 4), dict(ks=(4, 64)), dict(vs=(64, -64))):
            assert rows(f, **bad) == LAYOUT, bad
        assert rows(f, T=0, k=None, v=None, slots=None) == 0
    # rows that are written must not overlap; rows that are read may
    for bad in ((0, 64), (64, 64), (64, 0), (96, 64), (64, 100 * 8)):
        assert rows(L.entmax_attn_cache4_read, T=20, Hk=2, ks=bad) == LAYOUT, bad
    assert ea.entmax_attn_cache4_page_bytes(8, 128, 64) == 64 * 8 * 136
    assert ea.entmax_attn_cache4_page_bytes(8, 128, 60) == 0 and ea.entmax_attn_cache4_page_bytes(0, 128, 64) == 0


def decode(L, q=A, cache=A, table=A, lens=A, O=A, tau=A, R=1, Hq=2, Hk=1, d=64, t=1, max_len=64, blocks=4, pages=8, page=16, alpha=1.5, ws=A, nbytes=1 << 40):
    return L.entmax_attn_decode_cache4(q, cache, table, lens, O, tau, None, R, Hq, Hk, d, t, max_len, blocks, pages, page, alpha, ws, nbytes, None)


def test_decode_refusals(L):
    for missing in ("q", "cache", "table", "lens", "O", "tau"):
        assert decode(L, **{missing: None}) == NULL, missing
    assert decode(L, t=5) == DTYPE
    for bad in (dict(R=0), dict(R=65536), dict(Hq=3, Hk=2), dict(Hk=0), dict(d=80), dict(max_len=0), dict(max_len=65), dict(blocks=0),
                dict(pages=0), dict(page=17), dict(pages=1 << 28), dict(max_len=(1 << 22) + 1, blocks=1 << 20)):
        assert decode(L, **bad) == SHAPE, bad
    for alpha in (1.0, 3.5, float("nan"), float("inf")):
        assert decode(L, alpha=alpha) == ALPHA
    assert decode(L, q=A + 8) == LAYOUT and decode(L, cache=A + 8) == LAYOUT
    assert decode(L, ws=None) == WORKSPACE and decode(L, ws=A + 128) == WORKSPACE and decode(L, nbytes=100) == WORKSPACE
    f = ea.entmax_attn_decode_cache4_workspace_bytes
    assert f(1, 32, 8, 128, 1000) >= 32 * 1000 * 4 and f(1, 32, 7, 128, 1000) == 0 and f(1, 32, 8, 128, 0) == 0


def test_bindings_refuse_cpu_tensors_and_wrong_types():
    x = torch.zeros(1, 1, 1, 64)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        ea.entmax_attn_qk_norm_rope_fwd(x, x, i, torch.zeros(32))
    with pytest.raises(ValueError):
        ea.entmax_attn_cache_tables(i[0], i[0], i, i[0], i[0], 16, 4)
    with pytest.raises(ValueError):
        ea.entmax_attn_cache4_write(x[0], x[0], i[0], torch.zeros(1, 1, 16 * 68, dtype=torch.uint8), 16)
    with pytest.raises(ValueError):
        ea.entmax_attn_decode_cache4(x[0], torch.zeros(1, 1, 16 * 68, dtype=torch.uint8), i, i[0], 1.5, 16)
    with pytest.raises(ValueError):
        ea.entmax_attn_cache4_empty(0, 1, 64, 16, device="cpu")
    assert ea.entmax_attn_cache4_empty(3, 2, 64, 16, device="cpu").shape == (3, 2, 16 * 68)


@pytest.mark.parametrize("n", [0, 4, 6, 10])
def test_tables_binding_refuses_outputs_of_another_number(n):
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="token_start"):
        ea.entmax_attn_cache_tables(i, i, i[None], i, i, 16, 1, out=(i,) * n)


def test_bindings_refuse_a_workspace_that_is_a_view_of_less():
    x, i = torch.zeros(1, 1, 1, 64), torch.zeros(1, 1, dtype=torch.int32)
    w, f, ws = torch.ones(64), torch.zeros(32), torch.zeros(1, dtype=torch.uint8).expand(1 << 24)
    with pytest.raises(ValueError, match="workspace"):
        ea.entmax_attn_qk_norm_rope_bwd(x, x, x, x, i, f, w, w, workspace=ws)
    with pytest.raises(ValueError, match="workspace"):
        ea.entmax_attn_decode_cache4(x[0], torch.zeros(1, 1, 16 * 68, dtype=torch.uint8), i, i[0], 1.5, 16, workspace=ws)


def test_strerror_of_layout(L):
    assert "overlap" in ea.entmax_attn_strerror(LAYOUT)


@pytest.mark.parametrize("interleaved,rot", [(False, 64), (True, 64), (False, 24), (True, 40), (False, 0)])
def test_reference_gradient_against_differences(interleaved, rot):
    # the formulas of the header (dx, dw) and the reference's own automatic gradient against central differences
    g = torch.Generator().manual_seed(7)
    B, N, H, d, eps = 2, 3, 2, 64, 1e-6
    x, w, dy = torch.randn(B, N, H, d, generator=g).double(), torch.randn(d, generator=g).double(), torch.randn(B, H, N, d, generator=g).double()
    pairs = rot // 2
    cos, sin = ref.rotation(torch.randint(0, 1000, (2, B, N), generator=g), torch.rand(pairs, generator=g), [pairs // 2, pairs - pairs // 2])
    f = lambda x, w: (ref.prep(x, w, cos, sin, interleaved, eps, True) * dy).sum()      # noqa: E731
    gr = ref.rotate(dy.transpose(1, 2), cos, -sin, interleaved)
    rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh = x * rstd
    dx, dw = rstd * (gr * w - xh * (gr * w * xh).mean(-1, keepdim=True)), (gr * xh).sum((0, 1, 2))
    xr, wr = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    auto = torch.autograd.grad(f(xr, wr), (xr, wr))
    assert (auto[0] - dx).abs().max() < 1e-12 and (auto[1] - dw).abs().max() < 1e-12
    for _ in range(4):
        v, u, h = torch.randn(x.shape, generator=g).double(), torch.randn(d, generator=g).double(), 1e-5
        num = (f(x + h * v, w + h * u) - f(x - h * v, w - h * u)) / (2 * h)
        assert abs(num - (dx * v).sum() - (dw * u).sum()) < 1e-6 * (1 + abs(num))      # (the third derivative times h^2, and 1e-16 |f| / h)


def test_reference_rounding_to_levels():
    x = np.zeros((9, 32))
    x[0, :9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.25000001]      # ties go to even codes
    x[1, 0] = 7.0                                                           # still the small scale: rounded to 6
    x[2, 0] = 7.0000005                                                     # the next scale: 3.50000025 -> 4
    x[3, 0], x[4, 0], x[5, 0] = -1e-45, np.inf, np.nan
    x[6, 0] = 3.4028234663852886e38
    x[7, :2] = [2.0 ** -126, -2.0 ** -127]
    x[8] = -0.0
    codes, byte, val = ref.quantise(x)
    assert codes[0, :9].tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 1]
    assert byte[1, 0] == 127 and val[1, 0] == 6 and byte[2, 0] == 128 and val[2, 0] == 8
    assert byte[3, 0] == 1 and val[3, 0] == 0 and byte[4, 0] == byte[5, 0] == 255 and np.isnan(val[4]).all()
    assert byte[6, 0] == 252 and val[6, 0] == 6 * 2.0 ** 125
    assert val[7, :2].tolist() == [2.0 ** -126, -2.0 ** -127] and (codes[8] == 8).all()
    rng = np.random.default_rng(1)
    y = rng.standard_normal((100, 64)) * np.exp(rng.standard_normal((100, 1)) * 5)
    c, b, v = ref.quantise(y)
    scale = np.repeat(np.ldexp(1.0, b - 127), 32, -1)
    assert (np.abs(v - y) <= scale * np.where(np.abs(y) > 4 * scale, 1.0, np.where(np.abs(y) > 2 * scale, 0.5, 0.25)) + 1e-300).all()
