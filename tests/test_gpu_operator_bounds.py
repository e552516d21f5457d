"""The bounds that the operators beside the attention state, held one by one, and the variants that their launch rules choose."""
import numpy as np
import pytest
import torch

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
TERMS = [("f32", 2.0 ** -6, 2.0 ** -30)]


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
