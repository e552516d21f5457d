"""The 8-bit paged cache and the bookkeeping of pages that requests share, as they are measured.

* "rows":    keys and values of new tokens appended to the pages of an 8-bit cache, and read back as the cache holds them;
* "decode":  one query per head and request against that cache, over all its tokens or a sliding window and the first few;
* "fork":    requests forked from others (pages shared, a page that is partly filled copied), and ended again;
* "compact": pages moved to the front of a cache, in the tables and in memory.

`run` computes a case either with elementary torch operations (`own` false) or with the library (`own` true).

The 8-bit cache.  A page holds `page` tokens of every key/value head; a head's part of it is the codes of its keys
[page][d] and of its values [page][d], signed bytes, then the float32 scales of its keys [page/16] and of its values
[page/16], and zeros up to a multiple of 16 bytes.  The d values of 16 neighbouring tokens share a scale; a value is its code times
the scale's magnitude, and code -128 is not a number (the scale of a block that holds one has its sign bit set).  Rows that are
appended to a block keep its scale unless their largest magnitude over 127 is more: then that is the scale, and the codes in
front of them are rounded once more.  A row 0 starts its block anew.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
BLOCK = 16


# ---- the cases ----------------------------------------------------------------------------------------------------

def _rows(name, R, new, Hk, d, dtype="bf16", page=64):
    return dict(name=name, kind="rows", R=R, new=new, Hk=Hk, d=d, dtype=dtype, page=page)


def _decode(name, R, Hq, Hk, longest, d, alpha, sigma, dtype="bf16", page=64, window=0, sinks=0):
    return dict(name=name, kind="decode", R=R, Hq=Hq, Hk=Hk, longest=longest, d=d, alpha=alpha, sigma=sigma, dtype=dtype,
                page=page, window=window, sinks=sinks)


def listed():
    return [
        # a step of 64 requests, one token each: latency; most go behind others in their block
        _rows("rows: 64 requests, a token each", 64, 1, 8, 128),
        # a long prompt
        _rows("rows: prompt of 16001", 1, 16001, 8, 128),
        # chunks of prompts of a small float32 model, in small pages
        _rows("rows: 24 chunks of 127, f32", 24, 127, 5, 64, dtype="f32", page=16),
        # interactive: one request, shared key heads
        _decode("decode: one of 4001", 1, 32, 8, 4001, 128, 1.5, 2.0),
        # a serving batch with lengths all over the range
        _decode("decode: 48 to 32768", 48, 32, 8, 32768, 128, 1.5, 1.5),
        # the longest, no shared heads
        _decode("decode: one of 131072, 32 key heads", 1, 32, 32, 131072, 128, 1.5, 1.5),
        # float32 queries, head dimension 64, another alpha, small pages, odd numbers of heads
        _decode("decode: 24 to 8191, f32, d 64", 24, 15, 5, 8191, 64, 1.25, 1.5, dtype="f32", page=16),
        # a layer with a sliding window among long requests
        _decode("decode: 64 to 32768, window 4000 + 4", 64, 32, 8, 32768, 128, 1.5, 1.5, window=4000, sinks=4),
        # several answers to each of a few prompts: latency
        dict(name="fork: 8 prompts, 64 requests", kind="fork", prompts=8, samples=8, longest=8191, Hk=8, d=128, page=64),
        # many of them, in small pages
        dict(name="fork: 60 prompts, 1020 requests", kind="fork", prompts=60, samples=17, longest=4097, Hk=2, d=64, page=16),
        # a small cache, a few requests left in it
        dict(name="compact: 16 requests", kind="compact", R=16, longest=4000, Hk=8, d=128, page=64, used=0.5),
        # a large one, a quarter of it free
        dict(name="compact: 200 requests", kind="compact", R=200, longest=16000, Hk=8, d=128, page=64, used=0.75),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(("rows", "decode", "decode", "fork", "compact"))
    d, dtype = rng.choice((64, 128, 128)), rng.choice(("bf16", "bf16", "f32"))
    page = rng.choice((16, 32, 64, 128, 256))
    Hk = rng.choice((1, 2, 3, 4, 8))
    if kind == "rows":
        R = int(_log_uniform(rng, 1, 200))
        return dict(kind=kind, R=R, new=int(_log_uniform(rng, 1, max(2, 16000 * 8 * 128 * 2 / (R * Hk * d * SIZES[dtype])))), Hk=Hk, d=d,
                    dtype=dtype, page=page)
    if kind == "fork":
        prompts = int(_log_uniform(rng, 1, 60))
        return dict(kind=kind, prompts=prompts, samples=rng.randint(2, 17), longest=int(_log_uniform(rng, 50, 4097)), Hk=min(Hk, 2), d=64,
                    page=page)
    if kind == "compact":
        return dict(kind=kind, R=int(_log_uniform(rng, 1, 200)), longest=int(_log_uniform(rng, 300, 16000)), Hk=Hk, d=d, page=page,
                    used=round(rng.uniform(0.2, 0.9), 2))
    Hq = Hk * rng.choice((1, 2, 3, 4, 8, 16)) if Hk < 4 else Hk * rng.choice((1, 2, 4))
    R = int(_log_uniform(rng, 1, 65))
    longest = int(_log_uniform(rng, 100, min(131072, 48 * 32768 * 8 * 128 / (R * Hk * d), 48 * 32768 * 32 / (R * Hq))))
    window = rng.choice((0, 0, 1)) and int(_log_uniform(rng, 1, longest))
    return dict(kind=kind, R=R, Hq=Hq, Hk=Hk, longest=longest, d=d, alpha=rng.choice((1.25, 1.5, 1.5, 1.75, 2.0)),
                sigma=round(rng.uniform(1.2, 2.2), 2), dtype=dtype, page=page, window=window,
                sinks=rng.choice((0, 1, 4, 100)) if window else 0)


def _host_rng(seed):
    return torch.Generator().manual_seed(seed)


def _lengths(R, longest, empty=False):
    """Lengths of R requests: the longest, and others spread over the logarithm of the range, with `empty` one of zero.  They belong
    to the case, not to the seed, so that every seed is the same work."""
    lens = [longest] + [max(1, int(longest ** (0.4 + 0.6 * ((k * 0.618034) % 1.0)))) for k in range(1, R)]
    if empty and R > 4:
        lens[2] = 0
    return lens


def _spans(case):
    """Of a "rows" case: (tokens cached, tokens after) of each request."""
    R, new = case["R"], case["new"]
    have = [(37 * k + 11) % 150 if R > 1 else 0 for k in range(R)]
    more = [new if new < 8 or k == 0 else max(1, int(new * (0.5 + 0.5 * ((k * 0.618034) % 1.0)))) for k in range(R)]
    return [(a, a + b) for a, b in zip(have, more)]


# ---- inputs -------------------------------------------------------------------------------------------------------

def _part_bytes(page, d):
    return 2 * page * d + max(16, page // BLOCK * 8)


def _parts(cache, page, d):
    """Views of a cache [pages, Hk, bytes]: codes of keys and values [pages, Hk, page, d], their scales [pages, Hk, page/16]."""
    n, b = page * d, page // BLOCK
    codes = cache.view(torch.int8)
    kc, vc = (codes[..., o:o + n].unflatten(-1, (page, d)) for o in (0, n))
    ks, vs = (cache.view(torch.float32)[..., o:o + b] for o in (n // 2, n // 2 + b))
    return kc, vc, ks, vs


def _pages(lens, page, blocks, spare, seed):
    """A table of distinct pages in random order, [R, blocks], -1 behind a request's last; those that are left; their number in all."""
    have = torch.tensor([-(-n // page) for n in lens])
    total = int(have.sum())
    order = torch.randperm(total + spare, generator=_host_rng(seed)).to(torch.int32)
    table = torch.full((len(lens), blocks), -1, dtype=torch.int32)
    table[torch.arange(blocks)[None] < have[:, None]] = order[:total]
    return table, order[total:], total + spare


def _fill(cache, page, d, g, sigma=1.0):
    """Random codes, as normal values of that deviation leave them."""
    parts = _parts(cache, page, d)
    for first in range(0, cache.shape[0], 2048):
        for codes, scales in ((parts[0][first:first + 2048], parts[2][first:first + 2048]), (parts[1][first:first + 2048], parts[3][first:first + 2048])):
            codes.copy_((torch.randn(codes.shape, generator=g, device="cuda") * 33.0).round().clamp(-127, 127))
            scales.copy_((0.9 + 0.2 * torch.rand(scales.shape, generator=g, device="cuda")) * (sigma / 33.0))


def _prepare_rows(case, g, seed):
    Hk, d, page = case["Hk"], case["d"], case["page"]
    spans = _spans(case)
    ends = [b for _, b in spans]
    table, _, pages = _pages(ends, page, -(-max(ends) // page), 3, seed)
    slot = lambda r, p: int(table[r, p // page]) * page + p % page  # noqa: E731
    slots = [slot(r, p) for r, (a, b) in enumerate(spans) for p in range(a, b)]
    # read back: the new rows and those that stand in front of them in their block
    back = [slot(r, p) for r, (a, b) in enumerate(spans) for p in range(a // BLOCK * BLOCK, b)]
    rows = torch.randn(len(slots), 2 * Hk, d, generator=g, device="cuda")
    # some channels of the keys are larger than the others, as in trained models
    rows[:, :Hk] *= torch.exp(0.7 * torch.randn(Hk, d, generator=g, device="cuda"))
    rows = rows.to(DTYPES[case["dtype"]])
    cache = torch.zeros(pages, Hk, _part_bytes(page, d), dtype=torch.uint8, device="cuda")
    _fill(cache, page, d, g)
    return dict(case=case, k=rows[:, :Hk], v=rows[:, Hk:], cache=cache, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"),
                back=torch.tensor(back, dtype=torch.int32, device="cuda"))


def _prepare_decode(case, g, seed):
    R, Hq, Hk, d, page = (case[k] for k in ("R", "Hq", "Hk", "d", "page"))
    lens = _lengths(R, case["longest"], empty=True)
    table, _, pages = _pages(lens, page, -(-case["longest"] // page), 4, seed)
    cache = torch.zeros(pages, Hk, _part_bytes(page, d), dtype=torch.uint8, device="cuda")
    _fill(cache, page, d, g)
    _parts(cache, page, d)[2].mul_(case["sigma"])
    q = (case["sigma"] * torch.randn(R, Hq, d, generator=g, device="cuda")).to(DTYPES[case["dtype"]])
    return dict(case=case, q=q, cache=cache, table=table.cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), workspace=None)


def _fork_lengths(case):
    """Lengths of the requests before and of the forks after: request k * samples is a prompt, the others have no token yet.  Most
    continue the whole prompt, some an earlier place of it."""
    n = case["samples"]
    prompts = _lengths(case["prompts"], case["longest"])
    old = [prompts[r // n] if r % n == 0 else 0 for r in range(len(prompts) * n)]
    new = [prompts[r // n] if r % n == 0 or r % 5 else max(1, prompts[r // n] * (r % 7 + 1) // 8) for r in range(len(old))]
    return old, new


def _prepare_fork(case, g, seed):
    Hk, d, page, n = case["Hk"], case["d"], case["page"], case["samples"]
    old, new = _fork_lengths(case)
    R = len(old)
    table, free, pages = _pages(old, page, -(-case["longest"] // page) + 1, R + 9, seed)
    cache = torch.zeros(pages, Hk, _part_bytes(page, d), dtype=torch.uint8, device="cuda")
    _fill(cache, page, d, g)
    stack = torch.full((pages,), -1, dtype=torch.int32)
    stack[:len(free)] = free
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(case=case, cache=cache, old=ints(old), new=ints(new), parents=ints([r // n * n for r in range(R)]), itself=ints(list(range(R))),
                kept=ints([a if r % n == 0 else 0 for r, a in enumerate(old)]), table=table.cuda(), free=stack.cuda(),
                count=ints([len(free)]), shares=torch.zeros(pages, dtype=torch.int32, device="cuda"), workspace=None)


def _prepare_compact(case, g, seed):
    Hk, d, page, R = case["Hk"], case["d"], case["page"], case["R"]
    lens = _lengths(R, case["longest"], empty=True)
    need = sum(-(-n // page) for n in lens)
    table, free, pages = _pages(lens, page, -(-case["longest"] // page) + 1, max(1, int(need * (1 / case["used"] - 1))), seed)
    shares = torch.zeros(pages, dtype=torch.int32)
    if R > 1:                                          # the last request shares the first pages of the first one
        same = min(lens[-1], lens[0]) // page
        free = torch.cat([free, table[-1, :same]])
        table[-1, :same] = table[0, :same]
        shares[table[0, :same].long()] = 1
    cache = torch.zeros(pages, Hk, _part_bytes(page, d), dtype=torch.uint8, device="cuda")
    _fill(cache, page, d, g)
    stack = torch.full((pages,), -1, dtype=torch.int32)
    stack[:len(free)] = free
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(case=case, cache=cache, lens=ints(lens), table=table.cuda(), free=stack.cuda(), count=ints([len(free)]), shares=shares.cuda())


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"rows": _prepare_rows, "decode": _prepare_decode, "fork": _prepare_fork, "compact": _prepare_compact}[case["kind"]](case, g, seed)


# ---- plain forms --------------------------------------------------------------------------------------------------

def _append(x, codes, scales, slots, page):
    """Rows x [T, Hk, d] to their slots.  Quotients in 64 bits: the nearest code is exact."""
    x = x.float()
    finite = torch.isfinite(x)
    block, row = slots.long() // BLOCK, slots.long() % BLOCK
    touched, at = torch.unique_consecutive(block, return_inverse=True)
    first = torch.full_like(touched, BLOCK).scatter_reduce(0, at, row, "amin")
    size = torch.where(finite, x, 0.0).abs().amax(-1)                                            # [T, Hk]
    top = torch.zeros(len(touched), x.shape[1], device=x.device).scatter_reduce(0, at[:, None].expand_as(size), size, "amax")
    need = torch.where(top > 0, (top.double() / 127).float().clamp(min=2.0 ** -126), 0.0)
    pg, part = touched // (page // BLOCK), touched % (page // BLOCK)
    before = torch.where(first[:, None] > 0, scales[pg, :, part], 0.0)
    scale = torch.maximum(before.abs(), need)
    inside = torch.arange(BLOCK, device=x.device)
    kept = codes[pg[:, None], :, part[:, None] * BLOCK + inside].permute(0, 2, 1, 3)             # [blocks, Hk, 16, d]
    again = kept.double() * before.abs().double()[..., None, None] / scale.clamp(min=2.0 ** -126).double()[..., None, None]
    again = again.round().clamp(-127, 127).to(torch.int8)
    again = torch.where(kept == -128, kept, again)
    grown = (scale > before.abs())[..., None, None] & (inside < first[:, None])[:, None, :, None]
    codes[pg[:, None], :, part[:, None] * BLOCK + inside] = torch.where(grown, again, kept).permute(0, 2, 1, 3)
    mine = scale[at][..., None].double()
    fresh = (torch.where(finite, x, 0.0).double() / mine.clamp(min=2.0 ** -126)).round().clamp(-127, 127).to(torch.int8)
    codes[slots.long() // page, :, slots.long() % page] = torch.where(finite, fresh, -128)
    strange = torch.signbit(before) | torch.zeros(len(touched), x.shape[1], device=x.device).scatter_reduce(
        0, at[:, None].expand_as(size), (~finite).any(-1).float(), "amax").bool()
    scales[pg, :, part] = torch.where(strange, -scale, scale)


def _held(codes, scales, page_of, row):
    """Rows as the cache holds them, in 32 bits; page_of, row of any shape -> [..., Hk, d]."""
    c = codes[page_of, :, row]
    v = c.float() * scales[page_of, :, row // BLOCK].abs()[..., None]
    return v.masked_fill(c == -128, math.nan)


def _run_rows(s):
    case = s["case"]
    page, d, cache, dtype = case["page"], case["d"], s["cache"], DTYPES[case["dtype"]]
    if own:
        import paper_2604_15180_amd as ea
        ea.entmax_attn_cache8_write(s["k"], s["v"], s["slots"], cache, page)
        return ea.entmax_attn_cache8_read(cache, s["back"], page, d, dtype)
    kc, vc, ks, vs = _parts(cache, page, d)
    _append(s["k"], kc, ks, s["slots"], page)
    _append(s["v"], vc, vs, s["slots"], page)
    at, row = s["back"].long() // page, s["back"].long() % page
    return _held(kc, ks, at, row).to(dtype), _held(vc, vs, at, row).to(dtype)


def _threshold(x, alpha):
    """tau of rows x = (alpha - 1) z whose maximum is 0 (hidden entries -inf), so that sum [x - tau]_+^(1/(alpha-1)) = 1."""
    if alpha in (1.5, 2.0):
        # the largest prefix of the sorted row whose own root lies below its last entry
        top = torch.sort(x, dim=-1, descending=True).values.clamp(min=-2.0).double()
        n = torch.arange(1, x.shape[-1] + 1, device=x.device, dtype=torch.float64)
        mean = top.cumsum(-1) / n
        if alpha == 2.0:
            tau = mean - 1 / n
        else:
            spread = (top * top).cumsum(-1) - n * mean * mean
            tau = mean - torch.sqrt(((1 - spread) / n).clamp(min=0))
        size = (tau < top).sum(-1, keepdim=True).clamp(min=1)
        return tau.gather(-1, size - 1)
    lo, hi = torch.full_like(x[..., :1], -1.0), torch.zeros_like(x[..., :1])
    for _ in range(26):
        mid = 0.5 * (lo + hi)
        over = (x - mid).clamp(min=0).pow(1 / (alpha - 1)).sum(-1, keepdim=True) >= 1
        lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
    return (0.5 * (lo + hi)).double()


def _run_decode(s):
    case = s["case"]
    R, Hk, d, page, alpha, window, sinks = (case[k] for k in ("R", "Hk", "d", "page", "alpha", "window", "sinks"))
    if own:
        import paper_2604_15180_amd as ea
        if s["workspace"] is None:
            nbytes = ea.entmax_attn_decode_cache8_workspace_bytes(R, case["Hq"], Hk, d, case["longest"], window, sinks)
            s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device=s["q"].device)
        return ea.entmax_attn_decode_cache8(s["q"], s["cache"], s["table"], s["lens"], alpha, page, case["longest"], window=window,
                                            sinks=sinks, workspace=s["workspace"])[:2]
    # the visible positions: all, or the first `sinks` and the last `window`
    length = s["lens"].long()[:, None]
    if window:
        start = (length - window).clamp(min=0)
        n = torch.arange(min(case["longest"], window + sinks), device=start.device)[None]
        few = torch.minimum(start, torch.full_like(start, sinks))
        position = torch.where(n < few, n, start + n - few)
    else:
        position = torch.arange(case["longest"], device=length.device)[None].expand(R, -1)
    hidden = (position >= length)[:, None, None, :]
    position = torch.where(position < length, position, 0)
    at = s["table"].long().clamp(min=0).gather(1, position // page)
    kc, vc, ks, vs = _parts(s["cache"], page, d)
    keys = _held(kc, ks, at, position % page)                                          # [R, n, Hk, d]
    z = torch.matmul(s["q"].float().view(R, Hk, -1, d), keys.permute(0, 2, 3, 1).contiguous()) / math.sqrt(d)
    del keys
    x = ((alpha - 1) * z).masked_fill(hidden, -math.inf)
    top = torch.where(length[..., None, None] > 0, x.amax(-1, keepdim=True), 0.0)
    x = x - top
    tau = torch.where(length[..., None, None] > 0, _threshold(x, alpha), 0.0)
    p = (x - tau).clamp(min=0).pow(1 / (alpha - 1)).float()
    o = torch.matmul(p, _held(vc, vs, at, position % page).transpose(1, 2).contiguous())
    return o.flatten(1, 2), (tau + top).float().flatten(1)


def _fork(lens, parents, new, table, free, count, shares, page):
    """Request r becomes the first new[r] tokens of what request parents[r] held.  -> lengths, moves [R, 2] (-1 behind the last), how
    many of them; table, free, count and shares are updated.  (There are pages enough for every copy.)"""
    R, blocks = table.shape
    n_pages = free.numel()
    old = table.clone()
    have, need = (lens + page - 1) // page, (new + page - 1) // page
    b = torch.arange(blocks, device=table.device)[None]
    itself = parents == torch.arange(R, device=table.device)
    mine = torch.where((b < need[:, None]) & ~itself[:, None], old[parents.long()], old)
    dropped = (b < have[:, None]) & ((b >= need[:, None]) | ~itself[:, None])
    added = (b < need[:, None]) & ~itself[:, None]
    taken, left = mine[added].long(), old[dropped].long()
    holders = shares.scatter_add(0, taken, torch.ones_like(taken, dtype=torch.int32)).scatter_add(0, left, -torch.ones_like(left, dtype=torch.int32))
    # pages that nobody holds any more: the last request's last page first
    index = torch.arange(R * blocks, device=table.device).view(R, blocks)
    last = torch.full((n_pages,), -1, device=table.device).scatter_reduce(0, left, index[dropped], "amax")
    pages = old.clamp(min=0).long()
    gone = dropped & (holders[pages] < 0) & (last[pages] == index)
    place = gone.flatten().flip(0).cumsum(0).flip(0).view(R, blocks) - 1 + count
    flat = torch.cat([free, free.new_zeros(1)])
    flat[torch.where(gone, place, n_pages).flatten()] = old.flatten()
    holders = holders.clamp(min=0)
    top = count + gone.sum()
    # pages that end a request in their middle and that others hold: one of the former keeps it, if nobody holds it whole
    tail = torch.where(new % page > 0, mine.gather(1, (need - 1).clamp(min=0).long()[:, None])[:, 0], -1)
    rank = torch.where(itself, 0, R) + torch.arange(R, device=table.device)
    slot = torch.where(tail >= 0, tail, n_pages).long()
    ones = torch.ones(R, dtype=torch.int32, device=table.device)
    ends = torch.zeros(n_pages + 1, dtype=torch.int32, device=table.device).scatter_add(0, slot, ones)
    best = torch.full((n_pages + 1,), 2 * R, device=table.device).scatter_reduce(0, slot, rank, "amin")
    held = torch.cat([holders, holders.new_zeros(1)])[slot] + 1
    copy = (tail >= 0) & (held > 1) & ((held > ends[slot]) | (best[slot] != rank))
    which = copy.cumsum(0) - 1
    page_of = flat[(top - 1 - which).clamp(min=0)]
    moves = torch.full((R + 1, 2), -1, dtype=torch.int32, device=table.device)
    moves[torch.where(copy, which, R)] = torch.stack([tail, page_of], 1)
    shares.copy_(torch.cat([holders, holders.new_zeros(1)]).scatter_add(0, torch.where(copy, slot, n_pages), -ones)[:n_pages])
    here = copy[:, None] & (b == need[:, None] - 1)
    table.copy_(torch.where(here, page_of[:, None], mine))
    free.copy_(flat[:-1])
    count.copy_(top - copy.sum())
    return new, moves[:-1], copy.sum()


def _copy(cache, moves):
    live = moves[:, 0] >= 0
    spare = moves[:, 1].clamp(min=0).long()[live]
    cache[spare] = cache[moves[:, 0].clamp(min=0).long()[live]]


def _run_fork(s):
    page, table, free, count, shares = s["case"]["page"], s["table"], s["free"], s["count"], s["shares"]
    if own:
        import paper_2604_15180_amd as ea
        if s["workspace"] is None:
            s["workspace"] = torch.empty(ea.entmax_attn_cache_fork_workspace_bytes(*table.shape), dtype=torch.uint8, device=table.device)
        after, moves, status = ea.entmax_attn_cache_fork(s["old"], s["parents"], s["new"], table, free, count, shares, page, workspace=s["workspace"])
        ea.entmax_attn_cache_copy(s["cache"], moves, status[:1])
        back = ea.entmax_attn_cache_fork(after, s["itself"], s["kept"], table, free, count, shares, page, workspace=s["workspace"])
        return after, moves, status[:1], back[0], back[1], table, free, count, shares, s["cache"]
    after, moves, made = _fork(s["old"], s["parents"], s["new"], table, free, count, shares, page)
    _copy(s["cache"], moves)
    back = _fork(after, s["itself"], s["kept"], table, free, count, shares, page)
    return after, moves, made.to(torch.int32)[None], back[0], back[1], table, free, count, shares, s["cache"]


def _run_compact(s):
    page, table, free, shares, lens = s["case"]["page"], s["table"], s["free"], s["shares"], s["lens"]
    if own:
        import paper_2604_15180_amd as ea
        tables, stack, held, moves, status = ea.entmax_attn_cache_compact(lens, table, free, s["count"], shares, page)
        ea.entmax_attn_cache_copy(s["cache"], moves, status[:1])
        return tables, stack, held, moves, status[:1], s["cache"]
    n = free.numel()
    index = torch.arange(n, device=table.device)
    is_free = torch.zeros(n + 1, dtype=torch.bool, device=table.device)
    is_free[torch.where(index < s["count"], free, n).long()] = True
    is_free = is_free[:-1]
    used = n - s["count"]
    hole, far = is_free & (index < used), ~is_free & (index >= used)
    # the lowest hole is filled by the lowest page behind the used ones, and so on
    moves = torch.full((n // 2 + 1, 2), -1, dtype=torch.int32, device=table.device)
    moves[torch.where(far, far.cumsum(0) - 1, n // 2), 0] = index.to(torch.int32)
    moves[torch.where(hole, hole.cumsum(0) - 1, n // 2), 1] = index.to(torch.int32)
    moves = moves[:-1]
    to = torch.where(far, torch.cat([moves[:, 1], moves.new_zeros(1)])[torch.where(far, far.cumsum(0) - 1, n // 2)], index.to(torch.int32))
    b = torch.arange(table.shape[1], device=table.device)[None]
    live = b < ((lens + page - 1) // page)[:, None]
    tables = torch.where(live, to[table.clamp(min=0).long()], table)
    held = torch.zeros_like(shares).scatter(0, to.long(), torch.where(is_free, 0, shares), reduce="add")
    stack = torch.where(index < s["count"], (n - 1 - index).to(torch.int32), free)
    _copy(s["cache"], moves)
    return tables, stack, held, moves, far.sum().to(torch.int32)[None], s["cache"]


def run(state):
    return {"rows": _run_rows, "decode": _run_decode, "fork": _run_fork, "compact": _run_compact}[state["case"]["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    kind, page = case["kind"], case["page"]
    token = 2 * case["Hk"] * case["d"]                   # values of a token's keys and values
    if kind == "rows":
        spans = _spans(case)
        new = sum(b - a for a, b in spans)
        back = sum(b - a // BLOCK * BLOCK for a, b in spans)
        # new rows in, their codes out; codes of the rows that are read back in, their values out
        return {"bytes": new * token * (SIZES[case["dtype"]] + 1) + back * token * (SIZES[case["dtype"]] + 1) + 4 * (new + back),
                "flops": 2 * token * (new + back)}
    if kind == "decode":
        near = case["window"] + case["sinks"] if case["window"] else case["longest"]
        keys = sum(min(n, near) for n in _lengths(case["R"], case["longest"], empty=True))
        rows = case["R"] * case["Hq"]
        # every visible key once; of the values only those of a support, not counted here
        return {"bytes": keys * case["Hk"] * (case["d"] + 4 / BLOCK) + rows * (case["d"] * (SIZES[case["dtype"]] + 4) + 4),
                "flops": 2 * keys * case["Hq"] * case["d"]}
    page_bytes = case["Hk"] * _part_bytes(page, case["d"])
    if kind == "fork":
        old, new = _fork_lengths(case)
        n = case["samples"]
        forks = [m for r, m in enumerate(new) if r % n]
        copies = sum(1 for m in forks if m % page)
        # entries of the forks read and written, holders of their pages there and back; the copied pages in and out
        return {"bytes": copies * 2 * page_bytes + 24 * sum(-(-m // page) for m in forks) + 32 * len(new), "flops": 0}
    lens = _lengths(case["R"], case["longest"], empty=True)
    need = sum(-(-m // page) for m in lens)
    # a page lies behind the used ones with the chance that any page is free
    moved = need * (1 - case["used"])
    return {"bytes": moved * 2 * page_bytes + 8 * need + 16 * need / case["used"], "flops": 0}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_rows(case, seed):
    s = prepare(case, seed)
    page, d = case["page"], case["d"]
    kc, vc, ks, vs = (p.cpu() for p in _parts(s["cache"], page, d))
    slots, back = s["slots"].tolist(), s["back"].tolist()
    runs, t = [], 0
    while t < len(slots):                                # neighbouring rows of one block
        u = t + 1
        while u < len(slots) and slots[u] // BLOCK == slots[t] // BLOCK:
            u += 1
        runs.append((t, u))
        t = u

    def held(x, codes, scales):
        x = x.cpu().double()
        value = {}                                       # slot -> [Hk, d]
        for t, u in runs:
            pg, first = slots[t] // page, slots[t] % BLOCK
            at = slots[t] % page // BLOCK
            # (inputs are finite)
            unit = x[t:u].abs().amax((0, 2)).div(127.0).float().double()
            if first:
                unit = torch.maximum(unit, scales[pg, :, at].double().abs())
                was = scales[pg, :, at].double().abs()[:, None]
                for i in range(first):
                    c = codes[pg, :, at * BLOCK + i].double()
                    value[slots[t] - first + i] = torch.where(unit[:, None] > was, torch.round(c * was / unit[:, None]), c) * unit[:, None]
            q = torch.round(x[t:u] / unit[:, None])
            for i in range(t, u):
                value[slots[i]] = q[i - t] * unit[:, None]
        return torch.stack([value[j] for j in back])

    return held(s["k"], kc, ks), held(s["v"], vc, vs)


def _exact_decode(case, seed):
    s = prepare(case, seed)
    Hk, d, page, alpha = case["Hk"], case["d"], case["page"], case["alpha"]
    r = 1 / (alpha - 1)
    kc, vc, ks, vs = _parts(s["cache"], page, d)
    out, tau = [], []
    for k, n in enumerate(s["lens"].tolist()):
        if n == 0:
            out.append(torch.zeros(case["Hq"], d, dtype=torch.float64, device="cuda"))
            tau.append(torch.zeros(case["Hq"], dtype=torch.float64, device="cuda"))
            continue
        pages = s["table"][k, :-(-n // page)].long()
        keep = torch.arange(n, device="cuda")
        if case["window"]:
            keep = keep[(keep < case["sinks"]) | (keep >= n - case["window"])]

        def decoded(codes, scales):
            c = codes[pages].transpose(0, 1).flatten(1, 2)[:, keep]
            return c.double() * scales[pages].transpose(0, 1).flatten(1, 2)[:, keep // BLOCK].double()[..., None]

        x = (alpha - 1) / math.sqrt(d) * (s["q"][k].double().view(Hk, -1, d) @ decoded(kc, ks).mT)
        top = x.amax(-1, keepdim=True)
        lo, hi = top - 1, top.clone()
        for _ in range(56):
            mid = (lo + hi) / 2
            over = (x - mid).clamp(min=0).pow(r).sum(-1, keepdim=True) >= 1
            lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
        out.append(((x - lo).clamp(min=0).pow(r) @ decoded(vc, vs)).flatten(0, 1))
        tau.append(lo.flatten())
    return torch.stack(out), torch.stack(tau)


def _exact_fork(case, seed):
    s = prepare(case, seed)
    page = case["page"]
    table, stack = s["table"].tolist(), s["free"].tolist()
    free, cache = stack[:int(s["count"])], s["cache"].clone()
    holders = {}
    for row, n in zip(table, s["old"].tolist()):
        for p in row[:-(-n // page)]:
            holders[p] = holders.get(p, 0) + 1

    def step(lens, parents, new):
        R = len(lens)
        old = [row[:-(-n // page)] for row, n in zip(table, lens)]
        now = [old[parents[r]][:-(-new[r] // page)] for r in range(R)]
        for r in range(R):
            for p in now[r]:
                holders[p] += 1
            for p in old[r]:
                holders[p] -= 1
        for r in reversed(range(R)):
            for p in reversed(old[r]):
                if holders.get(p) == 0:
                    del holders[p]
                    stack[len(free)] = p
                    free.append(p)
        ends = {}
        for r in range(R):
            if new[r] % page:
                ends.setdefault(now[r][-1], []).append(r)
        whole = {p for pages, n in zip(now, new) for p in pages[:n // page]}
        moves = []
        for r in range(R):
            if new[r] % page == 0:
                continue
            p = now[r][-1]
            keeper = None if p in whole else min(ends[p], key=lambda i: (parents[i] != i, i))
            if (p in whole or len(ends[p]) > 1) and r != keeper:
                moves.append([p, free.pop()])
                now[r] = now[r][:-1] + [moves[-1][1]]
        for p, to in moves:
            holders[p] -= 1
            holders[to] = 1
        for r in range(R):
            table[r][:len(now[r])] = now[r]
        return new, moves + [[-1, -1]] * (R - len(moves)), [len(moves)]

    first = step(s["old"].tolist(), s["parents"].tolist(), s["new"].tolist())
    for a, b in first[1][:first[2][0]]:
        cache[b] = cache[a]
    back = step(first[0], s["itself"].tolist(), s["kept"].tolist())
    shares = [holders.get(p, 1) - 1 for p in range(len(stack))]
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return (*map(ints, (*first, back[0], back[1], table, stack, [len(free)], shares)), cache.cpu())


def _exact_compact(case, seed):
    s = prepare(case, seed)
    page, cache = case["page"], s["cache"].clone()
    table, stack, shares = s["table"].tolist(), s["free"].tolist(), s["shares"].tolist()
    n, free = len(stack), set(stack[:int(s["count"])])
    used = n - len(free)
    holes, far = [p for p in range(used) if p in free], [p for p in range(used, n) if p not in free]
    to = dict(zip(far, holes))
    tables = [[to.get(p, p) if b < -(-m // page) else p for b, p in enumerate(row)] for row, m in zip(table, s["lens"].tolist())]
    held = [0] * n
    for p in range(n):
        if p not in free:
            held[to.get(p, p)] = shares[p]
    moves = [[a, b] for a, b in zip(far, holes)]
    for a, b in moves:
        cache[b] = cache[a]
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return (ints(tables), ints([n - 1 - i if i < len(free) else p for i, p in enumerate(stack)]), ints(held),
            ints(moves + [[-1, -1]] * (n // 2 - len(moves))), ints([len(moves)]), cache.cpu())


def exact(case, seed):
    return {"rows": _exact_rows, "decode": _exact_decode, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](case, seed)
