"""Every variant that the launch rules of the operators beside the attention can choose, on data that would show an error: parts
of all lengths in the decode's score kernel, long supports with few, many and very many heads, several rows a thread in the
cache's kernels, several sets of tokens a work-group in the gradient of norm and rotation."""
import numpy as np
import pytest
import torch

from oracle import entmax_oracle as eo
from tests import test_gpu_operators as base
from tests.test_gpu_operators import DT, U, ea  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def check(q, ks, vs, alpha, got, dtype, sampled=None):
    """Against the 64-bit oracle, for any r = 1 / (alpha - 1).  A score is a sum of d products in fp32, off by at most d u sum |q k|, and by what
    the 8-bit terms leave of small elements; it enters the solve as x = c (s - max), 4 u of at most 1 more.  F = sum [x - tau]^r is
    known to 3 u for each y and 4 u for its logarithm, r times over, to 64 u for exponents up to 64, and to its sums' length
    (n / 256 a lane, 64 over lanes and waves); dF = -r G dtau with G >= F, so that tau is off by a part in r of that, and by the
    last step, 3e-8.  p is a power of y, and O is divided by the sum of the p."""
    r, d = 1 / (alpha - 1), q.shape[-1]
    c = (alpha - 1) / np.sqrt(d)
    exact, known = (2.0 ** -17, 2.0 ** -25) if dtype == "bf16" else (2.0 ** -6, 2.0 ** -30)
    O, tau, support = (t.cpu() for t in got)
    for i in range(q.shape[0]) if sampled is None else sampled:
        n, Hk = ks[i].shape[:2]
        if n == 0:
            assert (O[i] == 0).all() and (tau[i] == 0).all() and (support[i] == 0).all()
            continue
        K, V = (np.repeat(x.transpose(1, 0, 2), q.shape[1] // Hk, 0)[None] for x in (ks[i], vs[i]))
        qi = q[i].double().numpy()[None]
        want = eo.attn_decode(qi, K, V, alpha)
        a = np.abs(qi)
        lost = a.max(-1, keepdims=True) * known * (a < a.max(-1, keepdims=True) * exact)
        ds = d * U * (np.abs(K) @ a[..., None])[..., 0] + (np.abs(K) @ lost[..., None])[..., 0]
        eta = (2 * c * ds.max(-1, keepdims=True) + (4 + 7) * U + (64 + 64 + n / 256) * U / r + 3e-8)
        x = (alpha - 1) * want["z"] - want["tau"][..., None]
        p = lambda y: np.maximum(y, 0) ** r                                     # noqa: E731
        dp = np.maximum(p(x + eta) - p(x), p(x) - p(x - eta)) + (4 * r + 64) * U * p(x)
        # O / sum p: the errors of the p count twice, as they are and in the sum
        tol = 2 * (dp[..., None] * np.abs(V)).sum(2) + (2 * dp.sum(-1) + (n / 256 + 128) * U)[..., None] * (p(x)[..., None] * np.abs(V)).sum(2)
        err = np.abs(O[i].double().numpy() - want["O"][0])
        assert (err <= tol[0]).all(), (i, n, (err / tol[0]).max())
        terr = np.abs(tau[i].double().numpy() - want["tau"][0])
        assert (terr <= eta[0, :, 0] + 2 * U * np.abs(want["tau"][0])).all(), (i, n, terr.max())
        # keys whose p is no fp32 number (below 2^-150) are not counted, nor need be those whose p is none of full length
        surely, perhaps = (p(x - eta) > 2.0 ** -125).sum(-1)[0], (p(x + eta) > 2.0 ** -150).sum(-1)[0]
        got_n = support[i].numpy()
        assert ((got_n >= surely) & (got_n <= perhaps)).all(), (i, n, got_n, surely, perhaps)
        print(f"  request {i} n={n} |dO| {err.max():.2e} of allowed {(err / (tol[0] + 1e-300)).max():.3f} |dtau| {terr.max():.2e}", flush=True)


# ---- the score kernel: two tiles on their way per wave ------------------------------------------------------------

def part_of(R, Hq, Hk, max_len):
    """Keys per wave of the score kernel, as its launch rule has it."""
    groups = R * Hk * -(-(Hq // Hk) // 16)
    return min(max((max_len * groups // (8192 if R > 1 else 4096) + 63) // 64 * 64, 64), 512)


# A wave works on the blocks wave, wave + 4, ... of its work-group: requests whose first wave has 1 .. 8 of them, the others as many or
# one less, and one that takes a second work-group.
LENS = [64 * (4 * (m - 1) + m % 4 + 1) - 13 * m for m in range(1, 9)] + [2900]


@pytest.mark.parametrize("part", [128, 192, 256, 384, 512])
@pytest.mark.parametrize("d,dtype,G,page", [
    (128, "bf16", 4, 64), (128, "f32", 3, 16), (128, "bf16", 20, 256), (64, "bf16", 4, 16), (64, "f32", 8, 128), (64, "bf16", 16, 32),
    (64, "f32", 9, 16), (64, "f32", 16, 64)])
def test_decode_parts_of_all_lengths(ea, d, dtype, G, page, part):  # noqa: F811
    R, Hk = len(LENS), 2
    Hq = Hk * G
    groups = R * Hk * -(-G // 16)
    max_len = (part - 20) * 8192 // groups                          # what the tables could hold, far above the lengths
    assert part_of(R, Hq, Hk, max_len) == part
    cache, table, lens, ks, vs = base.make_cache(ea, LENS, Hk, d, page, 1.5, seed=part + d + G)
    wide = torch.full((R, -(-max_len // page)), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    q = (1.5 * torch.randn(R, Hq, d, generator=torch.Generator().manual_seed(part))).to(DT[dtype])
    got = ea.entmax_attn_decode_cache4(q.cuda(), cache, wide, lens, 1.5, page, max_len=max_len)
    for a, b in zip(got, ea.entmax_attn_decode_cache4(q.cuda(), cache, wide, lens, 1.5, page, max_len=max_len)):
        assert torch.equal(a, b)
    check(q, ks, vs, 1.5, got, dtype)


@pytest.mark.parametrize("d,dtype,page", [(128, "bf16", 64), (64, "f32", 16)])
def test_decode_parts_of_one_long_request(ea, d, dtype, page):  # noqa: F811
    n, Hk, Hq, max_len = 9000, 2, 8, 1 << 20
    assert part_of(1, Hq, Hk, max_len) == 512
    cache, table, lens, ks, vs = base.make_cache(ea, [n], Hk, d, page, 1.5, seed=3)
    wide = torch.full((1, max_len // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    q = (1.5 * torch.randn(1, Hq, d, generator=torch.Generator().manual_seed(4))).to(DT[dtype])
    check(q, ks, vs, 1.5, ea.entmax_attn_decode_cache4(q.cuda(), cache, wide, lens, 1.5, page, max_len=max_len), dtype)


# ---- the solve: candidates beyond a wave's buffer -----------------------------------------------------------------

@pytest.mark.parametrize("d,dtype,R,Hq,alpha,sigma", [
    (64, "bf16", 1, 8, 1.5, 0.2), (128, "f32", 1, 8, 1.1, 1.0),                     # four work-groups a head
    (64, "f32", 13, 8, 1.5, 0.2), (128, "bf16", 13, 8, 1.05, 1.0), (128, "f32", 13, 8, 2.5, 0.05), (64, "bf16", 13, 8, 2.0, 0.02),
    (64, "bf16", 75, 8, 1.5, 0.2), (128, "f32", 75, 8, 1.25, 0.5), (128, "bf16", 75, 8, 1.05, 1.0)])
def test_decode_long_supports_of_many_heads(ea, d, dtype, R, Hq, alpha, sigma):  # noqa: F811
    """Eight waves with 750 candidates and more each for up to 511 heads, four with 1500 from 512 on; one request is long."""
    alpha = float(np.float32(alpha))
    lens = [6000] + [(37 * i) % 300 for i in range(1, R)]
    cache, table, ln, ks, vs = base.make_cache(ea, lens, 1, d, 64, sigma, seed=R + d)
    q = (sigma * torch.randn(R, Hq, d, generator=torch.Generator().manual_seed(R))).to(DT[dtype])
    got = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, ln, alpha, 64)
    check(q, ks, vs, alpha, got, dtype, sampled=range(0, R, 1 + R // 12))


@pytest.mark.parametrize("alpha,dtype,d,n", [(1.1, "f32", 128, 5000), (1.05, "bf16", 64, 900), (1.02, "bf16", 64, 3000), (1.004, "f32", 128, 2000),
                                             (1.004, "bf16", 128, 700)])
def test_decode_support_and_output_of_large_powers(ea, alpha, dtype, d, n):  # noqa: F811
    alpha = float(np.float32(alpha))
    cache, table, ln, ks, vs = base.make_cache(ea, [n, 40], 2, d, 32, 1.5, seed=n)
    q = (1.5 * torch.randn(2, 4, d, generator=torch.Generator().manual_seed(n))).to(DT[dtype])
    check(q, ks, vs, alpha, ea.entmax_attn_decode_cache4(q.cuda(), cache, table, ln, alpha, 32), dtype)


# ---- the cache's rows, four items a thread ------------------------------------------------------------------------

@pytest.mark.parametrize("T,Hk,d,dtype,page", [(2077, 8, 64, "bf16", 64), (1031, 8, 128, "bf16", 16), (4111, 4, 64, "f32", 256), (2061, 4, 128, "f32", 32)])
def test_cache_rows_of_long_prompts(ea, T, Hk, d, dtype, page):  # noqa: F811
    assert T * 2 * Hk * d // 8 >= 1 << 18 and T * 2 * Hk * d // 8 % 1024
    base.test_cache_rows(ea, T, Hk, d, dtype, page)


# ---- the gradient of norm and rotation, several sets of tokens a work-group ---------------------------------------

@pytest.mark.parametrize("B,N,Hq,Hk,d,dtype,rot,axes,interleaved", [
    (1, 33001, 2, 1, 64, "bf16", 64, 1, False), (2, 20011, 1, 1, 64, "f32", 24, 3, True), (1, 17003, 2, 1, 128, "f32", 128, 2, False),
    (3, 11003, 1, 2, 128, "bf16", 40, 1, True)])
def test_norm_rope_gradient_of_many_tokens(ea, B, N, Hq, Hk, d, dtype, rot, axes, interleaved):  # noqa: F811
    assert B * N > 1024 * (256 // (d // 8))
    base.test_norm_rope_gradient(ea, B, N, Hq, Hk, d, dtype, rot, axes, interleaved, True, True)


# ---- one channel far above the others -----------------------------------------------------------------------------

def test_decode_of_queries_with_one_large_channel(ea):  # noqa: F811
    """One channel 128 times the others, in queries and in keys, at full length."""
    lens, d, page = [3000, 500], 128, 64

    def keys(r, n, g):
        k = torch.randn(n, 2, d, generator=g)
        k[:, :, 7] *= 0.05
        return k
    cache, table, ln, ks, vs = base.make_cache(ea, lens, 2, d, page, 1.0, seed=12, keys=keys)
    q = torch.randn(2, 8, d, generator=torch.Generator().manual_seed(3))
    q[:, :, 7] *= 128
    for dtype in ("bf16", "f32"):
        x = q.to(DT[dtype])
        check(x, ks, vs, 1.5, ea.entmax_attn_decode_cache4(x.cuda(), cache, table, ln, 1.5, page), dtype)
