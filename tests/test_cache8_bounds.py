"""What the header states of the 8-bit cache and the decode from it in figures, on the CPU."""
import random

import numpy as np
import pytest

import paper_2604_15180_amd as ea
from tests import paged_ref as ref

GROWTHS = ["normal", "rising 5 %", "largest rising 1 %", "doubling", "falling", "chunks"]


def grown_rows(rng, growth, n, Hk, d):
    """n rows, sixteen to a block, as a request meets them that grows a token at a time."""
    x = rng.standard_normal((n, Hk, d))
    k = (np.arange(n) % 16)[:, None, None]
    if growth == "rising 5 %":
        x *= 1.05 ** k
    elif growth == "largest rising 1 %":                          # every token's largest is a little above the last one's
        x = np.clip(x / 5, -0.99, 0.99)
        x[:, :, :1] = 1
        x *= 1.01 ** k
    elif growth == "doubling":
        x *= 2.0 ** k
    elif growth == "falling":
        x *= 0.9 ** k
    return x.astype(np.float32)


def within_half_the_scales(scales, got, rows):
    """scales: of each call the rows it wrote of every block, first and behind the last, and the scales of keys and values after it.  A row is off by
    half the scale that it was written with, and half of each larger one that came to its block later: the sum of its roundings.  Beside it stands
    what float32 leaves of a scale (127 half steps of 2^-24: where 127 s is below the largest element, or a value is formed): 2^-15 of a
    half.  Returns the largest error in 1/254 of the block's last scale times 127."""
    worst = 0.0
    for g, x, i in zip(got, rows, (0, 1)):
        n, Hk, d = x.shape
        allowed = np.zeros((n // 16, 16, Hk))
        last = None
        for a, b, s in scales:
            s = s[i].transpose(0, 2, 1).reshape(-1, Hk)[:n // 16].astype(np.float64)       # [blocks, Hk]
            allowed[:, a:b] += s[:, None] / 2
            if last is not None:
                assert (s >= last).all()
                allowed[:, :a] += np.where(s > last, s / 2, 0.0)[:, None]
            last = s
        err = np.abs(g.astype(np.float64) - x).reshape(n // 16, 16, Hk, d).max(-1)
        assert (err <= allowed * (1 + 2.0 ** -15)).all(), (err / allowed).max()
        assert (allowed <= 8 * last[:, None] * (1 + 2.0 ** -20)).all()                     # (sixteen roundings at most: 16/254 of the largest)
        worst = max(worst, (2 * err / last[:, None]).max())
    return worst


@pytest.mark.parametrize("growth", GROWTHS)
def test_a_block_that_grows_is_off_by_half_of_each_scale_it_had(growth):
    Hk, d, page, blocks = 2, 64, 64, 24
    rng = np.random.default_rng(GROWTHS.index(growth))
    x = grown_rows(rng, growth, 16 * blocks, 2 * Hk, d)
    c = ref.Cache8(np.zeros((16 * blocks // page, Hk, ref.part_bytes(d, page)), np.uint8), d, page)
    scales, at = [], 0
    while at < 16:
        n = min(int(rng.integers(1, 4)) if growth == "chunks" else 1, 16 - at)
        slots = (16 * np.arange(blocks)[:, None] + np.arange(at, at + n)).reshape(-1)
        c.write(x[slots][:, :Hk], x[slots][:, Hk:], slots)
        scales.append((at, at + n, [np.abs(s).copy() for s in c.scales]))
        at += n
    worst = within_half_the_scales(scales, c.read(np.arange(16 * blocks)), [x[:, :Hk], x[:, Hk:]])
    assert worst <= 16 * (1 + 2.0 ** -15)
    if growth == "largest rising 1 %":                            # (a 254th of the largest is what one call's rounding is off by, not a bound here)
        assert worst > 1 + 2.0 ** -15
    print(f"  {growth}: largest error {worst:.2f} of 1/254 of a block's largest")


def test_a_block_depends_on_the_calls_that_wrote_it():
    d, page = 64, 16
    x = grown_rows(np.random.default_rng(1), "rising 5 %", 16, 1, d)
    caches = [ref.Cache8(np.zeros((1, 1, ref.part_bytes(d, page)), np.uint8), d, page) for _ in range(2)]
    caches[0].write(x, x, range(16))
    for t in range(16):
        caches[1].write(x[t:t + 1], x[t:t + 1], [t])
    assert caches[0].scales[0] == caches[1].scales[0] and (caches[0].codes[0] != caches[1].codes[0]).any()
    top = np.abs(x).max()
    assert np.abs(caches[0].read(range(16))[0] - x).max() <= top / 254 * (1 + 2.0 ** -15) < np.abs(caches[1].read(range(16))[0] - x).max()


def test_the_decode_s_workspace_is_what_the_header_says():
    rng = random.Random(4)
    some = [(1, 1, 1, 0, 0), (1, 8, 64, 0, 0), (64, 32, 32768, 100, 4), (64, 32, 32768, 4000, 4), (3, 33, 65, 1, 0), (1, 1, 1 << 22, 2 ** 31 - 1, 2 ** 31 - 1),
            (65535, 1, 63, 64, 1), (2, 2, 4000, 66, 65)]
    some += [(rng.choice([1, 3, 64]), rng.choice([1, 8, 33]), int(2 ** rng.uniform(0, 22)), rng.choice([0, int(2 ** rng.uniform(0, 22.5))]),
              int(2 ** rng.uniform(0, 10)) - 1) for _ in range(2000)]
    for R, Hq, max_len, window, sinks in some:
        n = min(max_len, window + sinks) if window else max_len
        for d in (64, 128):
            size = ea.entmax_attn_decode_cache8_workspace_bytes(R, Hq, Hq, d, max_len, window, sinks)
            assert 4.125 * R * Hq * n <= size <= 4.125 * R * Hq * (n + 445) + 510, (R, Hq, max_len, window, sinks, size)
