"""Rows of the 8-bit cache on the GPU: what a block that grows in several calls has lost of the rows that were written, and every byte around
slots that are skipped."""
import numpy as np
import pytest
import torch

from tests import paged_ref as ref
from tests.test_cache8_bounds import GROWTHS, grown_rows, within_half_the_scales
from tests.test_gpu_operators import DT, ea, i32  # noqa: F401  (ea: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("growth", GROWTHS)
def test_rows_of_a_block_that_grows(ea, dtype, growth):  # noqa: F811
    # against the rows themselves, not against what the cache held before: half of every scale that the block had since
    Hk, d, page, blocks = 3, 128, 32, 40
    rng = np.random.default_rng(GROWTHS.index(growth))
    x = torch.from_numpy(grown_rows(rng, growth, 16 * blocks, 2 * Hk, d)).to(DT[dtype])
    cache = ea.entmax_attn_cache8_empty(blocks * 16 // page, Hk, d, page)
    calls = 0
    scales, at = [], 0
    while at < 16:                                                # all blocks side by side, a token (or a few) of each per call
        n = min(int(rng.integers(1, 4)) if growth == "chunks" else 1, 16 - at)
        slots = (16 * np.arange(blocks)[:, None] + np.arange(at, at + n)).reshape(-1)
        rows = x[slots].cuda()
        ea.entmax_attn_cache8_write(rows[:, :Hk], rows[:, Hk:], i32(slots.tolist()), cache, page)
        now = ref.Cache8(cache.cpu().numpy(), d, page)
        scales.append((at, at + n, [np.abs(s) for s in now.scales]))
        at += n
        calls += 1
    got = ea.entmax_attn_cache8_read(cache, i32(list(range(16 * blocks))), page, d, torch.float32)
    worst = within_half_the_scales(scales, [t.cpu().numpy() for t in got], [x[:, :Hk].float().numpy(), x[:, Hk:].float().numpy()])
    print(f"  {growth} {dtype}: {calls} calls, largest error {worst:.1f} of 1/254 of a block's largest", flush=True)


def test_all_bytes_around_skipped_slots(ea):  # noqa: F811
    # slots that are negative or past the cache directly in front of and behind others, in blocks that hold finite rows already
    Hk, d, page, pages = 2, 64, 32, 4
    rng = np.random.default_rng(19)
    want = ref.Cache8(np.zeros((pages, Hk, ref.part_bytes(d, page)), np.uint8), d, page)
    cache = ea.entmax_attn_cache8_empty(pages, Hk, d, page)
    for slots in (list(range(10)) + list(range(32, 43)) + list(range(64, 73)) + list(range(96, 100)) + list(range(112, 128)),
                  [-1, 4 * page, 40, 41, -7, 70, 71, 2 ** 31 - 1, 127, 126, 125, 112, 0, -2 ** 31, 99, 98],
                  [-1, 10, 11, 4 * page, -3, 43, -2 ** 31], [44, 2 ** 31 - 1, 72, 73, 74, -1, -1, 16]):
        k, v = (torch.from_numpy((rng.standard_normal((len(slots), Hk, d)) * np.exp(rng.standard_normal((len(slots), 1, 1)))).astype(np.float32))
                for _ in range(2))
        ea.entmax_attn_cache8_write(k.cuda(), v.cuda(), i32(slots), cache, page)
        want.write(k.numpy(), v.numpy(), slots)
        np.testing.assert_array_equal(cache.cpu().numpy(), want.bytes())
