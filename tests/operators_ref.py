"""The operators beside the attention in 64 bits on the CPU, written from their definitions: query/key norm with rotation,
the step of a scheduler, rows in 4 bits.  (The attention over the cache is compared with oracle.entmax_oracle.)"""
import numpy as np
import torch

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rotation(positions, inv_freq, sections):
    """cos, sin [B, N, pairs] in 64 bits; positions [axes, B, N]."""
    axis = np.repeat(np.arange(len(sections)), sections)
    t = positions.double()[torch.as_tensor(axis)].permute(1, 2, 0) * inv_freq.double()
    return torch.cos(t), torch.sin(t)


def rotate(x, cos, sin, interleaved):
    """x [B, N, H, d]; cos, sin [B, N, pairs]."""
    rot = 2 * cos.shape[-1]
    c, s = cos[:, :, None], sin[:, :, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([y, x[..., rot:]], -1)


def prep(x, w, cos, sin, interleaved, eps, norm):
    """x [B, N, H, d] in 64 bits -> [B, H, N, d]."""
    y = x
    if norm:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if w is not None:
            y = y * w
    return rotate(y, cos, sin, interleaved).transpose(1, 2)


def quantise(x):
    """float64 array [..., d] (d a multiple of 32) -> (codes 0..15 [..., d], scale bytes [..., d/32], values [..., d])."""
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    amax = np.abs(blocks).max(-1)
    finite = np.isfinite(blocks).all(-1)
    safe = np.where(finite, amax, 1.0)
    s = np.frexp(safe)[1].astype(np.int64) - 3
    s = np.where(safe == 0, -126, s)
    s = np.clip(s + (safe > np.ldexp(7.0, s)), -126, 125)
    y = np.abs(np.where(finite[..., None], blocks, 0.0)) / np.ldexp(1.0, s)[..., None]
    # nearest level; of two as near, the one with the even code
    dist = np.abs(y[..., None] - LEVELS) + 1e-13 * (np.arange(8) % 2)
    code = dist.argmin(-1)
    neg = np.signbit(np.where(finite[..., None], blocks, 0.0))
    values = np.where(neg, -1.0, 1.0) * LEVELS[code] * np.ldexp(1.0, s)[..., None]
    values = np.where(finite[..., None], values, np.nan)
    byte = np.where(finite, s + 127, 255)
    return (code + 8 * neg).reshape(x.shape), byte, values.reshape(x.shape)


def decode_cache(cache, d, page):
    """cache uint8 [pages, Hk, bytes] -> keys, values [pages, Hk, page, d] in 64 bits."""
    a, b = page * d // 2, page * d // 32
    out = []
    for o in (0, a + b):
        codes = cache[..., o:o + a].reshape(cache.shape[:2] + (page, d // 2))
        byte = cache[..., o + a:o + a + b].reshape(cache.shape[:2] + (page, d // 32)).astype(np.int64)
        c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (d,))
        scale = np.where(byte == 255, np.nan, np.ldexp(1.0, byte - 127))
        out.append(np.where(c & 8, -1.0, 1.0) * LEVELS[c & 7] * np.repeat(scale, 32, -1))
    return out


class Scheduler:
    """The step of entmax_attn_cache_tables, one request after the other."""

    def __init__(self, table, free, n_pages, page):
        self.table, self.n_pages, self.page = [list(map(int, r)) for r in table], n_pages, page
        self.stack = list(map(int, free)) + [None] * (n_pages - len(free))       # None: whatever stands there
        self.count = len(free)

    def step(self, lens, new, max_tokens):
        page, blocks = self.page, len(self.table[0])
        lens, new = list(map(int, lens)), list(map(int, new))
        ok = [0 <= a <= blocks * page and 0 <= b <= blocks * page for a, b in zip(lens, new)]
        pages = [(-(-a // page), -(-b // page)) if k else (0, 0) for a, b, k in zip(lens, new, ok)]
        for r in reversed(range(len(lens))):
            for b in reversed(range(pages[r][1], pages[r][0])):
                self.stack[self.count] = self.table[r][b]
                self.count += 1
        out, start, slots, positions, refused = [], [0], [], [], 0
        stop_pages = stop_rows = False
        for r in range(len(lens)):
            grow = max(0, new[r] - lens[r]) if ok[r] else 0
            want = max(0, pages[r][1] - pages[r][0])
            end = start[-1] + grow
            wanted_so_far = sum(max(0, q - p) for p, q in pages[:r + 1])
            if r == 0:
                have = self.count
            stop_pages = bool(want) and wanted_so_far > have
            stop_rows = bool(grow) and end > max_tokens
            granted = not (stop_pages or stop_rows)
            refused += ok[r] and not granted
            if granted:
                for b in range(pages[r][0], pages[r][1]):
                    self.count -= 1
                    self.table[r][b] = self.stack[self.count]
            out.append(new[r] if ok[r] and granted else lens[r])
            start.append(end)
            for p in range(lens[r], lens[r] + grow):
                if len(slots) < max_tokens:
                    slots.append(self.table[r][p // page] * page + p % page if granted else -1)
                    positions.append(p)
        status = [min(start[-1], max_tokens), refused, len(ok) - sum(ok), 0]
        slots += [-1] * (max_tokens - len(slots))
        positions += [0] * (max_tokens - len(positions))
        return out, start, slots, positions, status
