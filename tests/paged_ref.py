"""The 8-bit cache, the visible keys of a sliding window and the bookkeeping of shared pages from their definitions, on the CPU in 64
bits and in whole numbers.  (The attention over the cache is compared with oracle.entmax_oracle.)"""
import numpy as np
import torch

U = 2.0 ** -24                 # half a step of fp32, relative to the value
BLOCK = 16


def part_bytes(d, page):
    return 2 * page * d + max(16, page // 2)


class Cache8:
    """Keys ([0]) and values ([1]): codes [pages, Hk, page, d], scales [pages, Hk, page / 16] whose sign bit marks blocks with codes -128."""

    def __init__(self, raw, d, page):
        """raw: uint8 array [pages, Hk, bytes], whatever stands in it."""
        n, b = page * d, page // BLOCK
        self.raw, self.d, self.page = raw.copy(), d, page
        tail = np.ascontiguousarray(raw[..., 2 * n:2 * n + 8 * b]).view(np.float32)
        self.codes = [raw[..., i * n:(i + 1) * n].view(np.int8).reshape(raw.shape[:2] + (page, d)).copy() for i in (0, 1)]
        self.scales = [tail[..., i * b:(i + 1) * b].copy() for i in (0, 1)]

    def bytes(self):
        out, n, b = self.raw.copy(), self.page * self.d, self.page // BLOCK
        for i in (0, 1):
            out[..., i * n:(i + 1) * n] = self.codes[i].reshape(self.raw.shape[:2] + (n,)).view(np.uint8)
            at = 2 * n + 4 * i * b
            out[..., at:at + 4 * b] = np.ascontiguousarray(self.scales[i]).view(np.uint8)
        return out

    def write(self, K, V, slots):
        """K, V [T, Hk, d] float32 arrays, slots [T]; the rows of a block stand next to each other."""
        slots = [int(s) if 0 <= s < self.raw.shape[0] * self.page else None for s in slots]
        t = 0
        while t < len(slots):
            if slots[t] is None:
                t += 1
                continue
            u = t
            while u < len(slots) and slots[u] is not None and slots[u] // BLOCK == slots[t] // BLOCK:
                u += 1
            pg, blk = slots[t] // self.page, slots[t] % self.page // BLOCK
            rows = [s % BLOCK for s in slots[t:u]]
            for x, codes, scales in ((K, self.codes[0], self.scales[0]), (V, self.codes[1], self.scales[1])):
                for h in range(x.shape[1]):
                    v = x[t:u, h].astype(np.float64)
                    fine = np.isfinite(v)
                    top = np.abs(np.where(fine, v, 0.0)).max()
                    need = max(float(np.float32(top / 127)), 2.0 ** -126) if top > 0 else 0.0
                    first = min(rows)
                    was = scales[pg, h, blk] if first else np.float32(0)
                    old = abs(float(was))
                    s = max(old, need)
                    part = codes[pg, h, blk * BLOCK:(blk + 1) * BLOCK]
                    if s > old:
                        kept = part[:first].astype(np.float64)
                        part[:first] = np.where(kept == -128, -128, np.rint(kept * old / s))
                    c = np.clip(np.rint(np.where(fine, v, 0.0) / (s if s > 0 else 1.0)), -127, 127)
                    part[rows] = np.where(fine, c, -128)
                    strange = not fine.all() or bool(np.signbit(was))
                    scales[pg, h, blk] = np.float32(-s if strange else s)
            t = u

    def values(self):
        """[pages, Hk, page, d] each, in 64 bits."""
        out = []
        for codes, scales in zip(self.codes, self.scales):
            with np.errstate(invalid="ignore"):              # (garbage scales)
                s = np.repeat(np.abs(scales.astype(np.float64)), BLOCK, -1)[..., None]
            out.append(np.where(codes == -128, np.nan, codes * s))
        return out

    def read(self, slots):
        at = np.asarray(slots, dtype=np.int64)
        return [v[at // self.page, :, at % self.page] for v in self.values()]


def visible(n, window, sinks):
    j = np.arange(n)
    return np.ones(n, bool) if window == 0 else (j < sinks) | (j >= n - window)


# exact down to this part of the row's largest element, known to this part of it below
TERMS = {"bf16": (2.0 ** -13, 2.0 ** -21), "f32": (2.0 ** -4, 2.0 ** -28)}


def check_decode(q, ks, vs, alpha, O, tau, support, dtype, window=0, sinks=0):
    """q [R, Hq, d]; ks, vs: of each request its keys and values [n, Hk, d] as the cache holds them; against the float64 oracle over the
    visible ones.  What a kernel may differ by: a score's integer sum is exact and rounded five times, less than d u sum |q k|,
    plus what the 8-bit terms leave of elements far below their row's largest; scores enter the solve as
    c (s - max), 4 u more; the threshold moves by at most as much as the scores, and by what F = 1 is known to: a
    power is off by (2 + 2 r) u relative (r times the logarithm's half step over the range that counts), a sum of n
    terms by its 12 levels: 2e-6 covers both for r <= 4, r / 4 of it above."""
    from oracle import entmax_oracle as eo
    R, Hq, d = q.shape
    r = 1 / (alpha - 1)
    exact, known = TERMS[dtype]
    for i in range(R):
        n, Hk = ks[i].shape[:2]
        if n == 0:
            assert (O[i] == 0).all() and (tau[i] == 0).all() and (support[i] == 0).all()
            continue
        see = visible(n, window, sinks)
        K, V = (np.repeat(x[see].transpose(1, 0, 2), Hq // Hk, 0)[None] for x in (ks[i], vs[i]))
        qi = q[i].double().numpy()[None]
        want = eo.attn_decode(qi, K, V, alpha)
        c, most = (alpha - 1) / np.sqrt(d), np.abs(qi).max(-1, keepdims=True)
        lost = most * known * (np.abs(qi) < most * exact)
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
        print(f"  request {i} n={n} |dO| {err.max():.2e} |dtau| {terr.max():.2e} support {got.mean():.1f}", flush=True)


class Pages:
    """Tables, the stack of free pages and the holders of each page, one request after the other."""

    def __init__(self, table, free, n_pages, page, shares=None):
        self.table, self.n_pages, self.page = [list(map(int, r)) for r in table], n_pages, page
        self.stack = list(map(int, free)) + [-1] * (n_pages - len(free))
        self.count = len(free)
        self.shares = [0] * n_pages if shares is None else list(map(int, shares))

    def size(self, n):
        return -(-n // self.page)

    def fork(self, lens, parents, new):
        R, blocks = len(lens), len(self.table[0])
        fine = [0 <= n <= blocks * self.page for n in lens]
        invalid = 0
        parents, new = list(parents), list(new)
        for r in range(R):
            p = parents[r]
            if not (fine[r] and 0 <= p < R and fine[p] and 0 <= new[r] <= lens[p]):
                parents[r], new[r] = r, lens[r] if fine[r] else 0
                invalid += 1
        had = [self.table[r][:self.size(lens[r]) if fine[r] else 0] for r in range(R)]
        now = [list(had[parents[r]][:self.size(new[r])]) for r in range(R)]
        holders = {}
        for p in set(sum(had, []) + sum(now, [])):
            # everyone who holds it now: the shares say how many in all, of which some are left here
            holders[p] = self.shares[p] + 1 - sum(h.count(p) for h in had) + sum(h.count(p) for h in now)
        gone = [p for p in holders if holders[p] == 0]
        order = []
        for r in reversed(range(R)):
            for p in reversed(had[r]):
                if p in gone and p not in order:
                    order.append(p)
        for p in order:
            self.stack[self.count] = p
            self.count += 1
            self.shares[p] = 0
        ends = {}
        for r in range(R):
            if new[r] % self.page:
                ends.setdefault(now[r][-1], []).append(r)
        keep = {}
        for p, rs in ends.items():
            if holders[p] == len(rs):                      # nobody holds it whole
                own = [r for r in rs if parents[r] == r]
                keep[p] = (own or rs)[0]
        moves, refused, out = [], 0, list(new)
        for r in range(R):
            if not fine[r]:
                out[r] = lens[r]
            if new[r] % self.page == 0 or holders[now[r][-1]] == 1 or keep.get(now[r][-1]) == r:
                continue
            if self.count == 0:
                refused += 1
                out[r] = new[r] - new[r] % self.page
                now[r][-1] = (now[r][-1],)                 # (an entry behind the request's last page: not compared)
                continue
            self.count -= 1
            to = self.stack[self.count]
            moves.append((now[r][-1], to))
            now[r][-1] = to
        for p in holders:
            if p not in gone:
                self.shares[p] = holders[p] - 1
        for a, to in moves:
            self.shares[a] -= 1
            self.shares[to] = 0
        for r in range(R):
            for b, p in enumerate(now[r]):
                if isinstance(p, tuple):
                    self.shares[p[0]] -= 1
                    p = p[0]
                self.table[r][b] = p
        return out, moves, [len(moves), refused, invalid, 0]

    def compact(self, lens):
        free = set(self.stack[:self.count])
        used = self.n_pages - len(free)
        to = dict(zip((p for p in range(used, self.n_pages) if p not in free), (p for p in range(used) if p in free)))
        for r, n in enumerate(lens):
            for b in range(self.size(n)):
                self.table[r][b] = to.get(self.table[r][b], self.table[r][b])
        shares = [0] * self.n_pages
        for p in range(self.n_pages):
            if p not in free:
                shares[to.get(p, p)] = self.shares[p]
        self.shares = shares
        self.stack[:self.count] = [self.n_pages - 1 - i for i in range(self.count)]
        return sorted(to.items()), used


def random_fork(rng, lens):
    """A step of beams, samples, truncations and ends: (parents, new lengths)."""
    R = len(lens)
    parents, new = [], []
    for r in range(R):
        p = int(rng.integers(0, R)) if rng.random() < 0.5 else r
        parents.append(p)
        new.append(int(rng.choice([lens[p], lens[p], int(rng.integers(0, lens[p] + 1)), 0], p=[0.4, 0.2, 0.3, 0.1])))
    return parents, new


def ints(v):
    return torch.tensor(v, dtype=torch.int32)
