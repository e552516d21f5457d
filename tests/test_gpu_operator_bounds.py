"""The bounds that the operators beside the attention state, held one by one, and the variants that their launch rules choose."""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref
from tests.test_gpu_operators import DT, U, ea, i32  # noqa: F401  (ea: the fixture)

pytestmark = pytest.mark.gpu


def one_key_requests(ea, k, v, d, page=16):  # noqa: F811
    """A request of one key each: k, v [R, Hk, d] -> cache, table, lens."""
    R, Hk = k.shape[:2]
    cache = ea.entmax_attn_cache4_empty(R, Hk, d, page)
    table = torch.arange(R, dtype=torch.int32, device="cuda")[:, None].contiguous()
    ea.entmax_attn_cache4_write(k.cuda(), v.cuda(), table[:, 0] * page, cache, page)
    return cache, table, i32([1] * R)


# ---- what a score knows of the query ------------------------------------------------------------------------------

# dtype, exact down to this part of the row's largest element, known to this part below
TERMS = [("f32", 2.0 ** -6, 2.0 ** -30), ("bf16", 2.0 ** -17, 2.0 ** -25)]


@pytest.mark.parametrize("d,G", [(64, 3), (64, 11), (128, 5)])
@pytest.mark.parametrize("dtype,exact,known", TERMS)
def test_decode_scores_of_single_elements(ea, dtype, exact, known, d, G):  # noqa: F811
    """Request i's only key is the unit vector i, so that its score is element i of the query: with alpha = 2 and p = 1,
    tau = q_i / sqrt(d) - 1, formed in 64 bits and rounded once.  Rows of 2^20: the 1 takes nothing off."""
    g = torch.Generator().manual_seed(d + G)
    q = torch.randn(G, d, generator=g).sign() * torch.exp2(torch.rand(G, d, generator=g) * 40 - 39.999) * 2.0 ** 20
    q[:, ::2] = (torch.rand(G, d // 2, generator=g) * 2 - 1) * 2.0 ** 20             # half of them within a few binades of the largest
    q[:, 0] = 1.99 * 2.0 ** 19
    q = q.to(DT[dtype])
    cache, table, lens = one_key_requests(ea, torch.eye(d)[:, None], torch.ones(d, 1, d), d)
    O, tau, support = ea.entmax_attn_decode_cache4(q.cuda().expand(d, G, d).contiguous(), cache, table, lens, 2.0, 16)
    x = q.double().numpy().T                                                          # [request, head]
    top = np.abs(x).max(0)
    scale = 1 / np.sqrt(np.float64(d))
    want = x * scale - 1
    err = np.abs(tau.double().cpu().numpy() - want)
    tol = np.abs(want) * U + np.where(np.abs(x) < exact * top, known * top * scale, 0.0) + 2.0 ** -52 * top
    assert (err <= tol).all(), ((err > tol).mean(), (err / tol).max())
    assert (O == 1).all() and (support == 1).all()


# ---- alpha above 2 ------------------------------------------------------------------------------------------------


def near_ties(ea, alpha, counts, delta):  # noqa: F811
    """256 * counts[j] keys with the score -LEVELS[j] * delta, with values of 2^j: what the decode gives, and the
    definition's tau, weights of a key of each level and x in 64 bits."""
    page, d, r = 256, 64, 1 / (alpha - 1)
    n, level = 256 * np.array(counts, dtype=np.float64), ref.LEVELS[:len(counts)]
    k, v = torch.zeros(len(counts), page, 1, d), torch.zeros(len(counts), page, 1, d)
    k[..., 0] = -torch.from_numpy(level).float()[:, None, None]
    k[..., 1] = 6                                                               # (so that all blocks have the scale 1; its query element is 0)
    v[:] = 2.0 ** torch.arange(len(counts))[:, None, None, None]
    cache = ea.entmax_attn_cache4_empty(len(counts), 1, d, page)
    ea.entmax_attn_cache4_write(k.flatten(0, 1).cuda(), v.flatten(0, 1).cuda(), i32(list(range(256 * len(counts)))), cache, page)
    table = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).to(torch.int32)[None].cuda()
    q = torch.zeros(1, 1, d)
    q[0, 0, 0] = delta = float(np.float32(delta))
    got = ea.entmax_attn_decode_cache4(q.cuda(), cache, table, i32([int(n.sum())]), alpha, page)
    x = -(alpha - 1) / 8 * delta * level
    lo, hi = 0.0, 1.0                                                           # of -tau
    for _ in range(200):
        mid = (lo + hi) / 2
        lo, hi = (mid, hi) if (n * np.maximum(x + mid, 0) ** r).sum() < 1 else (lo, mid)
    return got, n, x, hi, r


def check_near_ties(got, n, x, t, r):
    """What a solve in fp32 may be off by: a power is 2^(r log2 y), the logarithm to 2^-23 of itself, the product to 2^-24, the power to
    2^-22; x to 4 u of itself; sums of N / 512 terms a lane and 64 over lanes and waves.  F grows with t at least as t^r does."""
    O, tau, support = got
    total = n.sum()
    y = x + t
    L = max(abs(np.log2(y[y > 0]))) * r
    power = 0.7 * L * (2.0 ** -23 + 2.0 ** -24) + 2.0 ** -22
    dt = (power + (total / 512 + 64) * U) / r * t + 5 * U * t
    assert abs(tau.item() + t) <= dt, (tau.item(), -t, dt)
    dy = dt + 4 * U * abs(x)
    p = lambda y: np.maximum(y, 0) ** r                                         # noqa: E731
    v = 2.0 ** np.arange(len(n))
    dp = np.maximum(p(y + dy) - p(y), p(y) - p(y - dy)) + power * p(y)
    want = (n * p(y) * v).sum() / (n * p(y)).sum()
    tol = (n * dp * abs(v - want)).sum() / (n * p(y)).sum() * 1.1 + 2 * want * (total / 256 + 96) * U
    assert (O[0, 0] - want).abs().max() <= tol, (O[0, 0, 0].item(), want, tol)
    assert n[y > dy].sum() <= support.item() <= n[y > -dy].sum()


@pytest.mark.parametrize("alpha", [2.25, 2.5, 3.0])
@pytest.mark.parametrize("n,m,at", [(8, 1, 1.5), (8, 1, 0.5), (40, 2, 1.02), (40, 2, 0.97), (1200, 5, 1.5), (1200, 500, 0.8), (15700, 300, 0.5)])
def test_decode_threshold_of_near_ties_with_alpha_above_two(ea, n, m, at, alpha):  # noqa: F811
    """256 n keys with the largest score, and others `at` and twice `at` times as far below it as the threshold of the former
    alone, N^-(alpha - 1) down to 6e-14."""
    alpha = float(np.float32(alpha))
    delta = 2 * at * (256.0 * n) ** -(alpha - 1) * 8 / (alpha - 1)                 # (the first level is 0.5)
    check_near_ties(*near_ties(ea, alpha, [n, m, m], delta))


# ---- long supports ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("alpha,counts,delta", [
    (1.95, [1006, 88, 9, 2, 11, 2, 5171, 4557], 1.5118186e-06), (1.95, [1010, 1, 333, 1020, 91, 295, 6609, 3829], 3.0919838e-07),
    (1.97, [1006, 190, 1, 98, 27, 2947, 1, 5965], 1.5801573e-06), (1.97, [3159, 3583, 12, 258, 6700, 62, 132, 36], 5.305047e-07),
    (1.99, [3160, 624, 85, 62, 23, 3, 7517, 90], 2.9965974e-07), (2.0, [3160, 624, 85, 62, 23, 3, 7517, 90], 2.9965974e-07),
    (2.0, [31, 7, 2, 40], 3e-4), (1.9, [100, 20, 30, 1, 1, 40], 2e-4), (1.75, [9000, 500, 3000], 2e-4)])
def test_decode_threshold_of_many_near_ties(ea, alpha, counts, delta):  # noqa: F811
    """Thousands to millions of keys within 1e-4 to 1e-6 of the largest score: -tau is itself of that size, and the first step of the
    solve, from -1, is known to 2^-24 of 1."""
    check_near_ties(*near_ties(ea, float(np.float32(alpha)), counts, delta))


# ---- scales at the ends of their range ----------------------------------------------------------------------------

@pytest.mark.parametrize("d,dtype,G", [(128, "bf16", 20), (64, "f32", 20), (64, "bf16", 5)])
def test_decode_limit_of_keys_and_queries(ea, d, dtype, G):  # noqa: F811
    """A head is infinite where the power of two in its query's largest element times a key's scale reaches 2^109; whatever the
    heads beside it hold.  Head h of the queries has its largest element in [2^h, 2^(h+1)); the request's keys have the scale 2^(109 - h0)."""
    heads = torch.arange(G, dtype=torch.float64)
    q = torch.zeros(1, G, d, dtype=torch.float64)
    q[0, :, 5] = 1.75 * torch.exp2(heads)
    q[0, :, 9] = -torch.exp2(heads)
    for h0 in (0, 3, G - 1, G):
        scale = 2.0 ** (109 - h0)
        k, v = torch.zeros(1, 1, d), torch.ones(1, 1, d)
        k[0, 0, 5], k[0, 0, 9] = 4 * scale, 2 * scale                                # (4: the largest of a block gets the scale 1)
        cache, table, lens = one_key_requests(ea, k, v, d)
        O, tau, support = (x[0].cpu() for x in ea.entmax_attn_decode_cache4(q.to(DT[dtype]).cuda(), cache, table, lens, 2.0, 16))
        over = heads >= h0
        assert torch.isnan(O[over]).all() and torch.isnan(tau[over]).all() and (support[over] == -1).all(), h0
        assert (O[~over] == 1).all() and (support[~over] == 1).all(), h0
        want = (1.75 * 4 - 2) * torch.exp2(heads) * scale / d ** 0.5                 # (less 1, which is nothing beside it)
        assert ((tau.double() - want)[~over].abs() <= want[~over] * 2 * U).all(), h0


def test_decode_and_read_agree_on_the_smallest_scale(ea):  # noqa: F811
    """Scale byte 0, 2^-127, which no write leaves but a page may hold."""
    d, page = 64, 16
    g = torch.Generator().manual_seed(1)
    cache = ea.entmax_attn_cache4_empty(1, 1, d, page)                          # (all scale bytes 0 or as written)
    cache.copy_(torch.randint(0, 256, cache.shape, generator=g, dtype=torch.uint8))
    scales = slice(page * d // 2, page * d // 2 + page * d // 32)
    cache[0, 0, scales] = 0
    cache[0, 0, page * d // 2 + page * d // 32:][scales] = 0
    k, v = ea.entmax_attn_cache4_read(cache, i32([0]), page, d, torch.float32)
    want = ref.decode_cache(cache.cpu().numpy(), d, page)
    np.testing.assert_array_equal(k[0, 0].double().cpu().numpy(), want[0][0, 0, 0])
    np.testing.assert_array_equal(v[0, 0].double().cpu().numpy(), want[1][0, 0, 0])
    q = torch.zeros(1, 1, d)
    q[0, 0, 3] = 2.0 ** 108
    O, tau, _ = ea.entmax_attn_decode_cache4(q.cuda(), cache, i32([[0]]), i32([1]), 2.0, page)
    assert torch.equal(O[0, 0], v[0, 0])                                        # p = 1
    assert tau.item() == np.float32(want[0][0, 0, 0, 3] * 2.0 ** 108 / 8 - 1)


# ---- sine and cosine ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_in_fp32_is_known_to_fp32(ea, interleaved):  # noqa: F811
    """Pairs of (1, 0): the outputs are the cosine and the sine themselves, rounded from 64 bits: half a step, and as much again
    for a sum of products."""
    B, N, d = 1, 3000, 128
    g = torch.Generator().manual_seed(6)
    x = torch.zeros(B, N, 1, d)
    x[..., slice(0, d, 2) if interleaved else slice(0, d // 2)] = 1
    pos = torch.randint(-200000, 200000, (1, B, N), generator=g).to(torch.int32)
    freq = torch.pow(10000.0, -torch.arange(d // 2, dtype=torch.float64) / (d // 2)).float()
    y, _ = ea.entmax_attn_qk_norm_rope_fwd(x.cuda(), x.cuda(), pos.cuda(), freq.cuda(), norm=False, interleaved=interleaved)
    cos, sin = ref.rotation(pos, freq, [d // 2])
    want = ref.rotate(x.double(), cos, sin, interleaved).transpose(1, 2)
    err = (y.double().cpu() - want).abs()
    print("  largest error, in half steps of 1:", err.max().item() / U, flush=True)
    # relative: the angle's rounding to fp32 u (times the angle, at most pi / 4 for a half that matters), a polynomial's last two
    # roundings; absolute: the 64-bit angle, 200000 2^-52
    assert (err <= 3 * U * want.abs() + 2e-10).all(), (err / U).max()


# ---- rows whose squares pass the largest float --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_rows_whose_squares_overflow(ea, dtype):  # noqa: F811
    """Sums of squares from 2^128 on: zeros.  64 elements of 2^61 are the first, of 2^60 still normed."""
    x = torch.ones(1, 1, 2, 64)
    x[0, 0, 0], x[0, 0, 1] = 2.0 ** 61, 2.0 ** 60
    x = x.to(DT[dtype]).cuda()
    y, _ = ea.entmax_attn_qk_norm_rope_fwd(x, x, None, None)
    assert (y[0, 0] == 0).all() and (y[0, 1] == 1).all()
