"""Host-only checks of the 8-bit cache and of shared pages: what their entry points refuse, their boundary under sanitizers, and the
definitions the GPU tests compare with against properties of their own."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2604_15180_amd as ea
from tests import paged_ref as ref
from tests.test_host_sanitizers import ENV, SAN, run

NULL, ALPHA, SHAPE, DTYPE, WORKSPACE, LAYOUT = -1, -2, -3, -4, -5, -8
A = 0x1000                                                   # never dereferenced: every call below is refused


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ea.lib_path()):
        from paper_2604_15180_amd import build
        build.build()
    return ea.lib()


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def rows(f, k=A, v=A, ks=(64, 64), vs=(64, 64), slots=A, cache=A, T=1, Hk=1, d=64, t=1, pages=4, page=16):
    a = (k, v, ks and i64(*ks), vs and i64(*vs), slots, cache)
    if f.__name__.endswith("read"):
        a = (cache, slots, k, v, ks and i64(*ks), vs and i64(*vs))
    return f(*a, T, Hk, d, t, pages, page, None)


def test_row_refusals(L):
    for f in (L.entmax_attn_cache8_write, L.entmax_attn_cache8_read):
        for missing in ("k", "v", "ks", "vs", "slots", "cache"):
            assert rows(f, **{missing: None}) == NULL, missing
        assert rows(f, t=9) == DTYPE
        for bad in (dict(T=-1), dict(Hk=0), dict(d=32), dict(page=24), dict(page=8), dict(pages=0), dict(pages=1 << 27), dict(T=1 << 30, Hk=64)):
            assert rows(f, **bad) == SHAPE, bad
        for bad in (dict(k=A + 8), dict(cache=A + 4), dict(ks=(4, 64)), dict(vs=(64, -64))):
            assert rows(f, **bad) == LAYOUT, bad
        assert rows(f, T=0, k=None, v=None, slots=None) == 0
    for bad in ((0, 64), (64, 64), (64, 0), (96, 64), (64, 100 * 8)):
        assert rows(L.entmax_attn_cache8_read, T=20, Hk=2, ks=bad) == LAYOUT, bad
    f = ea.entmax_attn_cache8_page_bytes
    for page in (16, 32, 64, 128, 256):
        assert f(8, 128, page) == 8 * ref.part_bytes(128, page) and f(3, 64, page) % 16 == 0
    assert f(8, 128, 60) == 0 and f(0, 128, 64) == 0 and f(1, 96, 64) == 0


def decode(L, q=A, cache=A, table=A, lens=A, O=A, tau=A, R=1, Hq=2, Hk=1, d=64, t=1, max_len=64, blocks=4, pages=8, page=16, window=0, sinks=0,
           alpha=1.5, ws=A, nbytes=1 << 40):
    return L.entmax_attn_decode_cache8(q, cache, table, lens, O, tau, None, R, Hq, Hk, d, t, max_len, blocks, pages, page, window, sinks, alpha, ws,
                                       nbytes, None)


def test_decode_refusals(L):
    for missing in ("q", "cache", "table", "lens", "O", "tau"):
        assert decode(L, **{missing: None}) == NULL, missing
    assert decode(L, t=5) == DTYPE
    for bad in (dict(R=0), dict(R=65536), dict(Hq=3, Hk=2), dict(Hk=0), dict(d=80), dict(max_len=0), dict(max_len=65), dict(blocks=0), dict(window=-1),
                dict(sinks=-1), dict(pages=0), dict(page=17), dict(pages=1 << 28), dict(max_len=(1 << 22) + 1, blocks=1 << 20)):
        assert decode(L, **bad) == SHAPE, bad
    for alpha in (1.0, 3.5, float("nan"), float("inf")):
        assert decode(L, alpha=alpha) == ALPHA
    assert decode(L, q=A + 8) == LAYOUT and decode(L, cache=A + 8) == LAYOUT
    assert decode(L, ws=None) == WORKSPACE and decode(L, ws=A + 128) == WORKSPACE and decode(L, nbytes=100) == WORKSPACE
    f = ea.entmax_attn_decode_cache8_workspace_bytes
    assert f(1, 32, 8, 128, 1000) >= 32 * 1000 * 4 and f(1, 32, 7, 128, 1000) == 0 and f(1, 32, 8, 128, 0) == 0
    assert f(1, 32, 8, 128, 100000, 1000, 4) < f(1, 32, 8, 128, 2000) and f(1, 1, 1, 64, 100, -1, 0) == 0
    assert f(1, 32, 8, 128, 1000, 1 << 40, 1 << 40) == f(1, 32, 8, 128, 1000)     # (a window of any length)


def fork(L, lens=A, parents=A, new=A, table=A, free=A, count=A, shares=A, out=A + 64, moves=A, status=A, R=1, blocks=4, page=16, pages=8, ws=A,
         nbytes=1 << 30):
    return L.entmax_attn_cache_fork(lens, parents, new, table, free, count, shares, out, moves, status, R, blocks, page, pages, ws, nbytes, None)


def compact(L, lens=A, table=A, free=A, count=A, shares=A, table_out=A, free_out=A, shares_out=A, moves=A, status=A, R=1, blocks=4, page=16, pages=8,
            ws=A, nbytes=1 << 30):
    return L.entmax_attn_cache_compact(lens, table, free, count, shares, table_out, free_out, shares_out, moves, status, R, blocks, page, pages, ws,
                                       nbytes, None)


def copy(L, src=A, dst=A, moves=A, count=A, n=1, nbytes=1024, a=4, b=4):
    return L.entmax_attn_cache_copy(src, dst, moves, count, n, nbytes, a, b, None)


SHAPES = (dict(R=0), dict(R=4097), dict(blocks=0), dict(page=8), dict(page=48), dict(page=512), dict(pages=0), dict(blocks=1 << 20, page=16),
          dict(pages=1 << 27, page=16))


def test_page_refusals(L):
    for missing in ("lens", "parents", "new", "table", "free", "count", "shares", "out", "moves", "status"):
        assert fork(L, **{missing: None}) == NULL, missing
    for missing in ("lens", "table", "free", "count", "table_out", "free_out", "shares_out", "shares", "moves", "status"):
        assert compact(L, **{missing: None}) == NULL, missing
    for missing in ("src", "dst", "moves", "count"):
        assert copy(L, **{missing: None}) == NULL, missing
    for bad in SHAPES:
        assert fork(L, **bad) == SHAPE and compact(L, **bad) == SHAPE, bad
    for bad in (dict(n=-1), dict(nbytes=0), dict(a=0), dict(b=0), dict(nbytes=1 << 36)):
        assert copy(L, **bad) == SHAPE, bad
    assert fork(L, out=A) == LAYOUT and fork(L, moves=A + 4) == LAYOUT and compact(L, moves=A + 4) == LAYOUT
    assert copy(L, nbytes=24) == LAYOUT and copy(L, src=A + 8) == LAYOUT and copy(L, dst=A + 4) == LAYOUT
    assert copy(L, n=0, moves=None) == 0
    for f in (fork, compact):
        assert f(L, ws=None) == WORKSPACE and f(L, ws=A + 128) == WORKSPACE and f(L, nbytes=100) == WORKSPACE
    assert ea.entmax_attn_cache_fork_workspace_bytes(0, 4) == 0 and ea.entmax_attn_cache_fork_workspace_bytes(3, 5) >= 2 * 3 * 5 * 4
    assert ea.entmax_attn_cache_compact_workspace_bytes(0) == 0 and ea.entmax_attn_cache_compact_workspace_bytes(1000) >= 1000 * 2


def test_bindings_refuse_cpu_tensors_and_wrong_types():
    x, i, c = torch.zeros(1, 1, 64), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 1, ref.part_bytes(64, 16), dtype=torch.uint8)
    m = torch.zeros(1, 2, dtype=torch.int32)
    for call in (lambda: ea.entmax_attn_cache8_write(x, x, i[0], c, 16), lambda: ea.entmax_attn_cache8_read(c, i[0], 16, 64),
                 lambda: ea.entmax_attn_decode_cache8(x, c, i, i[0], 1.5, 16), lambda: ea.entmax_attn_cache_copy(c, m, i[0]),
                 lambda: ea.entmax_attn_cache_fork(i[0], i[0], i[0], i, i[0], i[0], i[0], 16),
                 lambda: ea.entmax_attn_cache_compact(i[0], i, i[0], i[0], i[0], 16), lambda: ea.entmax_attn_cache8_empty(0, 1, 64, 16, device="cpu")):
        with pytest.raises(ValueError):
            call()
    assert ea.entmax_attn_cache8_empty(3, 2, 64, 16, device="cpu").shape == (3, 2, ref.part_bytes(64, 16))
    ws = torch.zeros(1, dtype=torch.uint8).expand(1 << 20)
    for call in (lambda: ea.entmax_attn_decode_cache8(x, c, i, i[0], 1.5, 16, workspace=ws),
                 lambda: ea.entmax_attn_cache_fork(i[0], i[0], i[0], i, i[0], i[0], i[0], 16, workspace=ws),
                 lambda: ea.entmax_attn_cache_compact(i[0], i, i[0], i[0], i[0], 16, workspace=ws)):
        with pytest.raises(ValueError, match="workspace"):
            call()
    with pytest.raises(ValueError, match="moves"):
        ea.entmax_attn_cache_fork(i[0], i[0], i[0], i, i[0], i[0], i[0], 16, out=(i[0],) * 2)
    with pytest.raises(ValueError, match="moves"):
        ea.entmax_attn_cache_compact(i[0], i, i[0], i[0], i[0], 16, out=(i[0],) * 4)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_boundary_under_sanitizers(tmp_path):
    from paper_2604_15180_amd import build as hip_build
    hip_build.build(force=False)
    mine = ("cache", "decode_cache8", "pages")
    objs = [os.path.join(hip_build.OBJDIR, u + ".o") for u in hip_build.UNITS if u not in mine]
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wno-unused-command-line-argument", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    sources = [os.path.join(hip_build.CSRC, u + ".hip") for u in mine] + [os.path.join(SAN, "paged_main.cpp")]
    outs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in sources]
    procs = [subprocess.Popen(["hipcc"] + flags + ["-c", s, "-o", o], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
             for s, o in zip(sources, outs)]
    for pr in procs:
        _, err = pr.communicate()
        assert pr.returncode == 0, err[-4000:]
    exe = str(tmp_path / "paged_san")
    run(["hipcc", "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize"] + outs + objs + ["-o", exe])
    res = run([exe], env=ENV)
    assert res.stdout.strip().endswith("ok") and "runtime error" not in res.stderr, res.stderr[-2000:]


# ---- the references against properties of their own ---------------------------------------------------------------

def test_reference_rows():
    rng = np.random.default_rng(3)
    d, page, Hk = 64, 32, 2
    c = ref.Cache8(rng.integers(0, 256, (3, Hk, ref.part_bytes(d, page)), dtype=np.uint8), d, page)
    assert (c.bytes() == c.raw).all()
    x = rng.standard_normal((40, Hk, d)).astype(np.float32)
    slots = np.concatenate([np.arange(64, 96), np.arange(0, 8)])
    c.write(x, 2 * x, slots)
    k, v = c.read(slots)
    for block in (slice(0, 16), slice(16, 32), slice(32, 40)):
        top = np.abs(x[block]).max((0, 2))[None, :, None].astype(np.float64)
        assert (np.abs(k[block] - x[block]) <= top / 254 * (1 + 1e-6)).all()
        assert (np.abs(v[block] - 2 * x[block]) <= top / 127 * (1 + 1e-6)).all()
    # appended rows: what stands in front is rounded once more where the scale grows, and stays where it does not
    before = c.read(np.arange(8))
    small = (x[:2] * 1e-3).astype(np.float32)
    c.write(small, small, [8, 9])
    assert all((a == b).all() for a, b in zip(before, c.read(np.arange(8))))
    big = (x[:1] * 1e2).astype(np.float32)
    c.write(big, big, [10])
    step = np.abs(big).max((0, 2))[None, :, None] / 127
    assert (np.abs(before[0] - c.read(np.arange(8))[0]) <= step / 2 * (1 + 1e-6)).all()
    # ties to even, not a number, zeros, tiny
    t = np.zeros((4, 1, d), np.float32)
    t[0, 0, :6] = [127, 0.5, 1.5, 2.5, -0.5, -3.5]
    t[1, 0, :2] = [np.inf, np.nan]
    c = ref.Cache8(np.zeros((1, 1, ref.part_bytes(d, 16)), np.uint8), d, 16)
    c.write(t, np.full_like(t, 1e-45), range(4))
    assert c.codes[0][0, 0, 0, :6].tolist() == [127, 0, 2, 2, 0, -4] and (c.codes[0][0, 0, 1, :2] == -128).all() and np.signbit(c.scales[0][0, 0, 0])
    assert c.scales[1][0, 0, 0] == 2.0 ** -126 and (c.codes[1] == 0).all()


def test_reference_forks_keep_account():
    rng = np.random.default_rng(5)
    page, R, blocks, n = 16, 9, 6, 40
    for trial in range(30):
        lens = [int(rng.integers(0, 40)) for _ in range(R)]
        need = [-(-m // page) for m in lens]
        order = rng.permutation(n)
        table, at = [[-1] * blocks for _ in range(R)], 0
        for r in range(R):
            table[r][:need[r]] = order[at:at + need[r]]
            at += need[r]
        p = ref.Pages(table, order[at:at + int(rng.integers(0, n - at + 1))], n, page)
        for step in range(6):
            parents, new = ref.random_fork(rng, lens)
            was = lens
            lens, moves, status = p.fork(lens, parents, new)
            held = [p.table[r][:p.size(lens[r])] for r in range(R)]
            free = p.stack[:p.count]
            for pg in range(n):
                k = sum(h.count(pg) for h in held)
                assert (pg in free) <= (k == 0) and p.shares[pg] == max(k - 1, 0)
            assert len(set(free)) == len(free) and status[0] == len(moves)
            for r in range(R):
                assert lens[r] == new[r] or (status[1] and lens[r] == new[r] // page * page)
                if lens[r] % page:                          # a page that will be written to is its request's own
                    assert sum(h.count(held[r][-1]) for h in held) == 1
            assert max(new[r] - was[parents[r]] for r in range(R)) <= 0
        moves, used = p.compact(lens)
        assert {pg for r in range(R) for pg in p.table[r][:p.size(lens[r])]} <= set(range(used)) and p.stack[:p.count] == list(range(n - 1, n - 1 - p.count, -1))
        assert all(a >= used > b for a, b in moves)
