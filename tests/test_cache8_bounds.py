"""What the header states of the 8-bit cache and the decode from it in figures, on the CPU."""
import random

import paper_2604_15180_amd as ea


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
