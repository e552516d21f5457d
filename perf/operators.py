"""The operators beside the attention itself, as they are measured: what turns a layer's projections into the
queries and keys of the attention calls, and the cache of a serving program.

* "rope":   norm of each head's queries and keys and their rotation by one or several position axes, and its gradient;
* "tables": block tables, slots and positions of a step, made on the GPU from the requests' lengths;
* "cache":  keys and values written to the pages of a 4-bit cache and read back as the cache holds them;
* "decode": one query per head and request against the 4-bit cache.

`run` computes a case either with elementary torch operations (`own` false) or with the library (`own` true).

The 4-bit cache.  A page holds `page` tokens of every key/value head; a head's part of it is the codes of its keys
[page][d/2], their scale bytes [page][d/32], then the same two of its values.  32 neighbouring values share the scale
2^(byte - 127); a code is a sign bit above three bits that stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6; the value with the lower
index is in the lower half of a byte.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


# ---- the cases ----------------------------------------------------------------------------------------------------

def _rope(name, B, N, Hq, Hk, d, dtype="bf16", grad=False, rot=None, axes=1, interleaved=False):
    return dict(name=name, kind="rope", B=B, N=N, Hq=Hq, Hk=Hk, d=d, dtype=dtype, grad=grad, rot=rot or d, axes=axes,
                interleaved=interleaved)


def _decode(name, R, Hq, Hk, longest, d, alpha, sigma, dtype="bf16", page=64):
    return dict(name=name, kind="decode", R=R, Hq=Hq, Hk=Hk, longest=longest, d=d, alpha=alpha, sigma=sigma, dtype=dtype,
                page=page)


def listed():
    return [
        # the projections of one decoding step of eight requests: latency
        _rope("rope_step_8", 8, 1, 32, 8, 128),
        # a training batch of the benchmark's size, one position axis
        _rope("rope_16k", 2, 16384, 16, 16, 128),
        # the gradient of an ordinary training step with time, height and width positions
        _rope("rope_grad_4k_3axes", 4, 4096, 16, 16, 64, grad=True, axes=3),
        # fp32, an odd number of tokens, shared key heads, neighbours as pairs, half of each head rotated
        _rope("rope_grad_f32_1087", 2, 1087, 8, 2, 128, dtype="f32", grad=True, rot=64, interleaved=True),
        # one token more for each of 64 running requests, and the step taken back
        dict(name="tables_step_64", kind="tables", R=64, longest=4096, page=64, mix=False),
        # a scheduler's turn: requests end, start with their prompts and go on, with small pages
        dict(name="tables_turn_1000", kind="tables", R=1000, longest=8192, page=16, mix=True),
        # the new keys and values of a decoding step of 64 requests
        dict(name="cache_step_64", kind="cache", T=64, Hk=8, d=128, dtype="bf16", page=64),
        # the keys and values of a long prompt, as its attention and later steps will see them
        dict(name="cache_prompt_16k", kind="cache", T=16001, Hk=8, d=128, dtype="bf16", page=64),
        # one request at the start of a conversation: latency
        _decode("decode_1x1000", 1, 32, 8, 1000, 128, 1.5, 1.5),
        # an ordinary serving batch, ragged, alpha away from the closed forms, fp32 queries
        _decode("decode_24x8k_a125", 24, 16, 8, 8192, 64, 1.25, 1.5, dtype="f32", page=16),
        # one long context, every head with keys of its own (the heads of the benchmark's decode)
        _decode("decode_1x128k", 1, 32, 32, 131072, 128, 1.5, 2.0),
        # a large ragged batch with shared key heads
        _decode("decode_48x32k", 48, 32, 8, 32768, 128, 1.5, 1.5),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(("rope", "rope", "tables", "cache", "decode", "decode"))
    d, dtype = rng.choice((64, 128)), rng.choices(("bf16", "f32"), (3, 1))[0]
    page = rng.choice((16, 32, 64, 128, 256))
    if kind == "rope":
        grad = rng.random() < 0.5
        Hk = rng.choice((1, 2, 4, 8, 16))
        Hq = Hk * rng.choice((1, 2, 3, 4, 8)) if Hk < 16 else Hk
        tokens = _log_uniform(rng, 1, 32768 * 32 * 128 * 2 / ((Hq + Hk) * d * (4 if dtype == "f32" else 2) * (2 if grad else 1)))
        B = rng.choice((1, 2, 4))
        rot = rng.choices((d, d // 2, 24), (4, 2, 1))[0]
        return dict(kind=kind, B=B, N=max(1, min(int(tokens / B), 131072)), Hq=Hq, Hk=Hk, d=d, dtype=dtype, grad=grad, rot=rot,
                    axes=rng.choice((1, 1, 2, 3)), interleaved=rng.random() < 0.4)
    if kind == "tables":
        return dict(kind=kind, R=int(_log_uniform(rng, 1, 1001)), longest=int(_log_uniform(rng, 500, 8192)), page=page,
                    mix=rng.random() < 0.6)
    if kind == "cache":
        Hk = rng.choice((1, 2, 4, 8))
        return dict(kind=kind, T=int(_log_uniform(rng, 1, 16000 * 8 * 128 * 2 / (Hk * d * (4 if dtype == "f32" else 2)))), Hk=Hk,
                    d=d, dtype=dtype, page=page)
    Hk = rng.choice((1, 2, 4, 8))
    Hq = Hk * rng.choice((1, 2, 3, 4, 8, 16)) if Hk < 4 else Hk * rng.choice((1, 2, 4))
    R = int(_log_uniform(rng, 1, 65))
    longest = int(_log_uniform(rng, 100, min(131072, 48 * 32768 * 8 * 128 / (R * Hk * d), 48 * 32768 * 32 / (R * Hq))))
    return dict(kind=kind, R=R, Hq=Hq, Hk=Hk, longest=longest, d=d, alpha=rng.choice((1.25, 1.5, 1.5, 1.75, 2.0)),
                sigma=round(rng.uniform(1.2, 2.2), 2), dtype=dtype, page=page)


def _host_rng(seed):
    return torch.Generator().manual_seed(seed)


def _lengths(case):
    """The requests' lengths of a decode case: the longest, and others spread over the logarithm of the range, one empty.
    They belong to the case, not to the seed, so that every seed is the same work."""
    R, longest = case["R"], case["longest"]
    lens = [longest] + [int(longest ** (0.4 + 0.6 * ((k * 0.618034) % 1.0))) for k in range(1, R)]
    if R > 4:
        lens[2] = 0
    return lens


# ---- inputs -------------------------------------------------------------------------------------------------------

def _exponent(amax):
    """s of the scale 2^s of a block whose largest magnitude is `amax` (finite)."""
    _, e = torch.frexp(amax)
    s = e - 3                                          # floor(log2 amax) - 2
    s = s + (amax > torch.ldexp(torch.full_like(amax, 7.0), s)).to(s.dtype)
    return s.clamp(-126, 125)


def _quantise(x):
    """x [..., d] -> (codes as bytes [..., d/2], scale bytes [..., d/32])."""
    blocks = x.float().unflatten(-1, (-1, 32))
    s = _exponent(blocks.abs().amax(-1))
    y = torch.ldexp(blocks.double(), -s[..., None])
    m = y.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)).to(torch.uint8)
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (s + 127).to(torch.uint8)


def _pair_table(device):
    level = torch.tensor(LEVELS, device=device)
    signed = torch.cat([level, -level])
    low = torch.arange(256, device=device) % 16
    return torch.stack([signed[low], signed[torch.arange(256, device=device) // 16]], -1)


def _values(codes, scales):
    """What codes [..., d/2] and scale bytes [..., d/32] stand for, in 32 bits."""
    v = _pair_table(codes.device)[codes.int()].flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)[..., None]).flatten(-2)


def _parts(cache, page, d):
    """Views of a cache [pages, Hk, bytes]: key codes, key scales, value codes, value scales, each [pages, Hk, page, ...]."""
    a, b = page * d // 2, page * d // 32
    return [cache[..., o:o + n].unflatten(-1, (page, -1)) for o, n in ((0, a), (a, b), (a + b, a), (2 * a + b, b))]


def _prepare_rope(case, g):
    B, N, Hq, Hk, d = (case[k] for k in ("B", "N", "Hq", "Hk", "d"))
    dt = DTYPES[case["dtype"]]
    # queries, keys and values come out of one projection: queries and keys are views of its rows
    rows = torch.randn(B, N, Hq + 2 * Hk, d, generator=g, device="cuda").to(dt)
    start = torch.randint(0, 100000, (B, 1), generator=g, device="cuda", dtype=torch.int32)
    step = torch.arange(N, device="cuda", dtype=torch.int32)
    axes, pairs = case["axes"], case["rot"] // 2
    # one axis: text.  Several: a video, frames of 16 x 24 patches
    pos = [start + step] if axes == 1 else [start + step // 384, (step // 24 % 16).expand(B, N), (step % 24).expand(B, N)][:axes]
    sections = [pairs // axes + (1 if k < pairs % axes else 0) for k in range(axes)]
    state = dict(case=case, q=rows[:, :, :Hq], k=rows[:, :, Hq:Hq + Hk], pos=torch.stack(pos).contiguous(), sections=sections,
                 inv_freq=torch.pow(10000.0, -torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs).float(),
                 wq=1.0 + 0.2 * torch.randn(d, generator=g, device="cuda"), wk=1.0 + 0.2 * torch.randn(d, generator=g, device="cuda"),
                 axis=torch.repeat_interleave(torch.arange(axes), torch.tensor(sections)).cuda())
    if case["grad"]:
        state["dq"] = torch.randn(B, Hq, N, d, generator=g, device="cuda")
        state["dk"] = torch.randn(B, Hk, N, d, generator=g, device="cuda")
    return state


def _turn(case):
    """Lengths before and after a turn, on the host.  They belong to the case; the pages' order goes by the seed."""
    rng = _host_rng(case["R"] * 10007 + case["longest"])
    R, longest = case["R"], case["longest"]
    old = torch.exp(torch.rand(R, generator=rng) * math.log(longest)).int().clamp(1, longest - 1)
    new = old + 1
    if case["mix"]:
        what = torch.rand(R, generator=rng)
        prompt = torch.exp(torch.rand(R, generator=rng) * math.log(longest)).int().clamp(1, longest)
        new = torch.where(what < 0.05, 0, new)                             # ended
        starts = (what >= 0.05) & (what < 0.1)
        old, new = torch.where(starts, 0, old), torch.where(starts, prompt, new)
        new = torch.where((what >= 0.1) & (what < 0.15), old, new)         # waits
        new = torch.where((what >= 0.15) & (what < 0.2), old // 2, new)    # goes back
    return old.to(torch.int32), new.to(torch.int32)


def _prepare_tables(case, seed):
    R, page = case["R"], case["page"]
    old, new = _turn(case)
    blocks = -(-case["longest"] // page)
    have = (old + page - 1) // page
    need = (new + page - 1) // page
    # enough pages for most turns to be granted whole, now and then too few for the last requests
    pages = int(have.sum()) + max(1, int((need - have).clamp(min=0).sum() * 0.97)) + R % 7
    order = torch.randperm(pages, generator=_host_rng(seed + 1)).to(torch.int32)
    table = torch.full((R, blocks), -1, dtype=torch.int32)
    used = torch.arange(blocks)[None] < have[:, None]
    table[used] = order[:int(have.sum())]
    free = torch.full((pages,), -1, dtype=torch.int32)
    count = pages - int(have.sum())
    free[:count] = order[int(have.sum()):]
    # room for the new tokens of the turn, and for those that come back when it is taken back
    rows = int(torch.maximum((new - old).clamp(min=0).sum(), (old - new).clamp(min=0).sum()))
    return dict(case=case, old=old.cuda(), new=new.cuda(), table=table.cuda(), free=free.cuda(),
                count=torch.tensor([count], dtype=torch.int32, device="cuda"), rows=rows + 32)


def _prepare_cache(case, g, seed):
    T, Hk, d, page = (case[k] for k in ("T", "Hk", "d", "page"))
    rows = torch.randn(T, 2 * Hk, d, generator=g, device="cuda")
    # some channels of the keys are larger than the others, as in trained models
    rows[:, :Hk] *= torch.exp(0.7 * torch.randn(Hk, d, generator=g, device="cuda"))
    rows = rows.to(DTYPES[case["dtype"]])
    pages = T // page + 8
    slots = torch.arange(T, device="cuda")
    order = torch.randperm(pages, generator=_host_rng(seed)).cuda()
    slots = (order[slots // page] * page + slots % page).to(torch.int32)
    nbytes = page * d * 17 // 16
    return dict(case=case, k=rows[:, :Hk], v=rows[:, Hk:], slots=slots,
                cache=torch.zeros(pages, Hk, nbytes, dtype=torch.uint8, device="cuda"))


def _prepare_decode(case, g, seed):
    R, Hq, Hk, d, page = (case[k] for k in ("R", "Hq", "Hk", "d", "page"))
    lens = torch.tensor(_lengths(case), dtype=torch.int32)
    blocks = -(-case["longest"] // page)
    have = (lens + page - 1) // page
    total = int(have.sum())
    pages = total + 4
    table = torch.full((R, blocks), -1, dtype=torch.int32)
    table[torch.arange(blocks)[None] < have[:, None]] = torch.randperm(pages, generator=_host_rng(seed))[:total].to(torch.int32)
    cache = torch.empty(pages, Hk, page * d * 17 // 16, dtype=torch.uint8, device="cuda")
    for first in range(0, pages, 2048):                # in parts: the values before they are rounded take 15 times the cache
        part = cache[first:first + 2048]
        kc, ks, vc, vs = _parts(part, page, d)
        n = part.shape[0]
        kc[...], ks[...] = _quantise(case["sigma"] * torch.randn(n, Hk, page, d, generator=g, device="cuda"))
        vc[...], vs[...] = _quantise(torch.randn(n, Hk, page, d, generator=g, device="cuda"))
    q = (case["sigma"] * torch.randn(R, Hq, d, generator=g, device="cuda")).to(DTYPES[case["dtype"]])
    return dict(case=case, q=q, cache=cache, table=table.cuda(), lens=lens.cuda(), workspace=None)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    if kind == "rope":
        return _prepare_rope(case, g)
    if kind == "tables":
        return _prepare_tables(case, seed)
    return _prepare_cache(case, g, seed) if kind == "cache" else _prepare_decode(case, g, seed)


# ---- plain forms --------------------------------------------------------------------------------------------------

def _angles(s):
    turn = s["pos"].double()[s["axis"]] * s["inv_freq"].double()[:, None, None]       # [pairs, B, N]
    turn = turn.permute(1, 2, 0)[:, :, None]                                             # [B, N, 1, pairs]
    return torch.cos(turn).float(), torch.sin(turn).float()


def _rotate(x, cos, sin, rot, interleaved):
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(s):
    case = s["case"]
    cos, sin = _angles(s)

    def forward(x, w):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        y = _rotate(y, cos, sin, case["rot"], case["interleaved"])
        return y.to(DTYPES[case["dtype"]]).transpose(1, 2).contiguous()

    def backward(x, w, dy):
        x = x.float()
        g = _rotate(dy.transpose(1, 2), cos, -sin, case["rot"], case["interleaved"])
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xhat = x * rstd
        gw = g * w
        dx = rstd * (gw - xhat * (gw * xhat).mean(-1, keepdim=True))
        return dx.to(DTYPES[case["dtype"]]), (g * xhat).double().sum((0, 1, 2)).float()

    if not case["grad"]:
        return forward(s["q"], s["wq"]), forward(s["k"], s["wk"])
    dq, dwq = backward(s["q"], s["wq"], s["dq"])
    dk, dwk = backward(s["k"], s["wk"], s["dk"])
    return dq, dk, dwq, dwk


def _plain_tables(lens, new, table, free, count, page, rows):
    """One turn.  Pages that shrinking requests leave go back to the top of the stack `free`, the last request's last page
    first; growing requests then take theirs from its top, in their order, as long as they last."""
    R, blocks = table.shape
    have, need = (lens + page - 1) // page, (new + page - 1) // page
    b = torch.arange(blocks, device=table.device)[None]
    back = (b >= need[:, None]) & (b < have[:, None])
    place = back.flatten().flip(0).cumsum(0).flip(0).view(R, blocks) - 1 + count
    flat = torch.cat([free, free.new_zeros(1)])
    flat[torch.where(back, place, free.numel()).flatten()] = table.flatten()
    top = count + back.sum()
    tokens = (new - lens).clamp(min=0)
    fits = ((need - have).clamp(min=0).cumsum(0) <= top) | (need <= have)
    fits &= (tokens.cumsum(0) <= rows) | (tokens == 0)
    get = (b >= have[:, None]) & (b < need[:, None]) & fits[:, None]
    place = top - get.flatten().cumsum(0).view(R, blocks)
    table.copy_(torch.where(get, flat[torch.where(get, place, free.numel())], table))
    free.copy_(flat[:-1])
    count.copy_(top - get.sum())
    start = torch.cat([tokens.new_zeros(1), tokens.cumsum(0)]).to(torch.int32)
    t = torch.arange(rows, device=table.device, dtype=torch.int32)
    r = (torch.searchsorted(start, t, right=True) - 1).clamp(max=R - 1)
    live = t < start[R]
    position = torch.where(live, lens[r] + t - start[r], 0)
    page_of = table[r, (position // page).clamp(max=blocks - 1)]
    slots = torch.where(live & fits[r], page_of * page + position % page, -1)
    return torch.where(fits, new, lens), start, slots.to(torch.int32), position.to(torch.int32)


def _run_tables(s):
    page, rows = s["case"]["page"], s["rows"]
    if own:
        import paper_2604_15180_amd as ea
        after, start, slots, position, _ = ea.entmax_attn_cache_tables(s["old"], s["new"], s["table"], s["free"], s["count"], page, rows)
        back = ea.entmax_attn_cache_tables(after, s["old"], s["table"], s["free"], s["count"], page, rows)
        return after, start, slots, position, back[0], s["table"], s["free"], s["count"]
    after, start, slots, position = _plain_tables(s["old"], s["new"], s["table"], s["free"], s["count"], page, rows)
    back = _plain_tables(after, s["old"], s["table"], s["free"], s["count"], page, rows)
    return after, start, slots, position, back[0], s["table"], s["free"], s["count"]


def _run_cache(s):
    case = s["case"]
    page, d, cache = case["page"], case["d"], s["cache"]
    if own:
        import paper_2604_15180_amd as ea
        ea.entmax_attn_cache4_write(s["k"], s["v"], s["slots"], cache, page)
        return ea.entmax_attn_cache4_read(cache, s["slots"], page, d, s["k"].dtype)
    parts = _parts(cache, page, d)
    at, row = s["slots"] // page, s["slots"] % page
    (kc, ks), (vc, vs) = _quantise(s["k"]), _quantise(s["v"])
    parts[0][at, :, row], parts[1][at, :, row], parts[2][at, :, row], parts[3][at, :, row] = kc, ks, vc, vs
    k = _values(parts[0][at, :, row], parts[1][at, :, row])
    v = _values(parts[2][at, :, row], parts[3][at, :, row])
    return k.to(s["k"].dtype), v.to(s["k"].dtype)


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
    Hk, d, page, alpha = case["Hk"], case["d"], case["page"], case["alpha"]
    if own:
        import paper_2604_15180_amd as ea
        if s["workspace"] is None:
            nbytes = ea.entmax_attn_decode_cache4_workspace_bytes(case["R"], case["Hq"], Hk, d, case["longest"])
            s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device=s["q"].device)
        return ea.entmax_attn_decode_cache4(s["q"], s["cache"], s["table"], s["lens"], alpha, page, case["longest"],
                                            workspace=s["workspace"])[:2]
    R, blocks = s["table"].shape
    kc, ks, vc, vs = (p[s["table"].clamp(min=0)].transpose(1, 2).flatten(2, 3) for p in _parts(s["cache"], page, d))
    hidden = torch.arange(blocks * page, device=kc.device) >= s["lens"][:, None, None, None]
    z = torch.matmul(s["q"].float().view(R, Hk, -1, d), _values(kc, ks).transpose(-1, -2)) / math.sqrt(d)
    x = ((alpha - 1) * z).masked_fill(hidden, -math.inf)
    top = torch.where(s["lens"][:, None, None, None] > 0, x.amax(-1, keepdim=True), 0.0)
    x = x - top
    tau = torch.where(s["lens"][:, None, None, None] > 0, _threshold(x, alpha), 0.0)
    p = (x - tau).clamp(min=0).pow(1 / (alpha - 1)).float()
    o = torch.matmul(p, _values(vc, vs))
    return o.flatten(1, 2), (tau + top).float().flatten(1)


def run(state):
    kind = state["case"]["kind"]
    if kind == "rope":
        if not own:
            return _plain_rope(state)
        import paper_2604_15180_amd as ea
        s, case = state, state["case"]
        how = dict(q_weight=s["wq"], k_weight=s["wk"], eps=EPS, sections=s["sections"], interleaved=case["interleaved"])
        if case["grad"]:
            return ea.entmax_attn_qk_norm_rope_bwd(s["q"], s["k"], s["dq"], s["dk"], s["pos"], s["inv_freq"], **how)
        return ea.entmax_attn_qk_norm_rope_fwd(s["q"], s["k"], s["pos"], s["inv_freq"], **how)
    return {"tables": _run_tables, "cache": _run_cache, "decode": _run_decode}[kind](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "rope":
        values = case["B"] * case["N"] * (case["Hq"] + case["Hk"]) * case["d"]
        size = 4 if case["dtype"] == "f32" else 2
        tokens = case["B"] * case["N"] * case["axes"] * 4
        if case["grad"]:
            return {"bytes": values * (2 * size + 4) + tokens, "flops": 16 * values}
        return {"bytes": values * 2 * size + tokens, "flops": 8 * values}
    if kind == "tables":
        # lengths in and out twice, starts, slots and positions once each, twice; the tables' changes are small beside them
        old, new = _turn(case)
        rows = int((new - old).clamp(min=0).sum())
        return {"bytes": 2 * (16 * case["R"] + 8 * rows), "flops": 0}
    if kind == "cache":
        values = case["T"] * 2 * case["Hk"] * case["d"]
        return {"bytes": values * (2 * (4 if case["dtype"] == "f32" else 2) + 2 * 17 / 32) + 8 * case["T"], "flops": 4 * values}
    keys, size = sum(_lengths(case)), 4 if case["dtype"] == "f32" else 2
    rows = case["R"] * case["Hq"]
    # every key once; of the values only those of a support, not counted here
    return {"bytes": keys * case["Hk"] * case["d"] * 17 / 32 + rows * (case["d"] * (size + 4) + 4), "flops": 2 * keys * case["Hq"] * case["d"]}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_rope(case, seed):
    s = prepare(case, seed)
    rot, w64 = case["rot"], torch.float64
    angle = torch.stack([s["pos"][int(a)].to(w64) * s["inv_freq"][i].to(w64) for i, a in enumerate(s["axis"].tolist())], -1)
    wave = torch.polar(torch.ones_like(angle), angle)[:, :, None]          # exp(i angle), [B, N, 1, pairs]

    def turn(x, by):                                   # pairs as complex numbers
        if case["interleaved"]:
            z = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * by
            y = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * by
            y = torch.cat([z.real, z.imag], -1)
        return torch.cat([y, x[..., rot:]], -1)

    def forward(x, w):
        x = x.to(w64)
        return turn(x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.to(w64), wave).transpose(1, 2)

    if not case["grad"]:
        return forward(s["q"], s["wq"]).contiguous(), forward(s["k"], s["wk"]).contiguous()

    def backward(x, w, dy):                            # by automatic differentiation of the forward
        x, w = x.to(w64).requires_grad_(True), w.to(w64).requires_grad_(True)
        return torch.autograd.grad(forward(x, w), (x, w), dy.to(w64))

    (dq, dwq), (dk, dwk) = backward(s["q"], s["wq"], s["dq"]), backward(s["k"], s["wk"], s["dk"])
    return dq, dk, dwq, dwk


def _exact_tables(case, seed):
    s = prepare(case, seed)
    page, rows = case["page"], s["rows"]
    table, stack = s["table"].tolist(), s["free"].tolist()
    free, size = stack[:int(s["count"])], len(stack)

    def turn(lens, new):
        for r in reversed(range(len(lens))):           # pages that are left go back
            for b in reversed(range(-(-new[r] // page), -(-lens[r] // page))):
                stack[len(free)] = table[r][b]
                free.append(table[r][b])
        after, start, slots, position = [], [0], [], []
        wanted, top = 0, len(free)
        for r, (a, b) in enumerate(zip(lens, new)):
            pages = range(-(-a // page), -(-b // page))
            wanted += len(pages)
            ok = b <= a or ((wanted <= top or not pages) and start[-1] + b - a <= rows)
            if ok:
                for k in pages:
                    table[r][k] = free.pop()
            after.append(b if ok else a)
            start.append(start[-1] + max(0, b - a))
            position += range(a, b)
            slots += [table[r][p // page] * page + p % page if ok else -1 for p in range(a, b)]
        return after, start, (slots + [-1] * rows)[:rows], (position + [0] * rows)[:rows]

    first = turn(s["old"].tolist(), s["new"].tolist())
    back = turn(first[0], s["old"].tolist())
    return tuple(torch.tensor(x, dtype=torch.int32) for x in (*first, back[0], table, stack, [len(free)]))


def _exact_cache(case, seed):
    s = prepare(case, seed)

    def rounded(x):
        # the nearest level of the block's scale, of two as near the one with an even index
        blocks = x.double().unflatten(-1, (-1, 32))
        most = blocks.abs().amax(-1, keepdim=True)
        unit = torch.exp2(torch.floor(torch.log2(most)) - 2).clamp(2.0 ** -126, 2.0 ** 125)
        unit = torch.where(most > 7 * unit, 2 * unit, unit).clamp(max=2.0 ** 125)
        level = torch.tensor(LEVELS, device=x.device, dtype=torch.float64)
        odd = torch.tensor([0.0, 1.0] * 4, device=x.device, dtype=torch.float64)
        far = ((blocks.abs() / unit)[..., None] - level).abs() + 1e-12 * odd
        return (torch.copysign(level[far.argmin(-1)], blocks) * unit).flatten(-2)

    return rounded(s["k"]), rounded(s["v"])


def _exact_decode(case, seed):
    s = prepare(case, seed)
    Hk, d, page, alpha = case["Hk"], case["d"], case["page"], case["alpha"]
    r, level = 1 / (alpha - 1), torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device="cuda")
    out, tau = [], []

    def decoded(codes, scales):                        # [Hk, n, d/2], [Hk, n, d/32]
        v = torch.stack([level[(codes % 16).long()], level[(codes // 16).long()]], -1).flatten(-2)
        return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)

    for k, n in enumerate(_lengths(case)):
        if n == 0:
            out.append(torch.zeros(case["Hq"], d, dtype=torch.float64, device="cuda"))
            tau.append(torch.zeros(case["Hq"], dtype=torch.float64, device="cuda"))
            continue
        pages = s["table"][k, :-(-n // page)].long()
        kc, ks, vc, vs = (p[pages].transpose(0, 1).flatten(1, 2)[:, :n] for p in _parts(s["cache"], page, d))
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


def exact(case, seed):
    kind = case["kind"]
    return {"rope": _exact_rope, "tables": _exact_tables, "cache": _exact_cache, "decode": _exact_decode}[kind](case, seed)
