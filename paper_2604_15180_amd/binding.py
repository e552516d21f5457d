"""ctypes binding of libentmax_attn.so (same names as the C entry points).

PyTorch is used for device memory and the current HIP stream only.  Outputs are allocated
here; every step of the path runs inside the library's kernels.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libentmax_attn.so")
_lib = None

EA_F32, EA_BF16 = 0, 1
EA_STATS_WORDS = 16
EA_STATS_COPIES = 64
STAT_NAMES = ("tau_subtiles", "out_subtiles", "delta_subtiles", "dq_subtiles", "dkdv_subtiles",
              "sweeps", "mask_subtiles", "out_pv_subtiles", "list_overflow_blocks", "gather_rows", "bwd_list_subtiles", "bwd_gather_rows",
              "f16_clamped")
EA_TIMER_SLOTS = 10
TIMER_NAMES = ("fwd_prep", "tau", "out", "mask", "bwd_prep", "dq", "dkdv", "decode_scores", "bwd_list", "bwd_gather")


class EntmaxAttnError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"entmax_attn error {code}: {text}")
        self.code = code


def lib_path():
    return _LIB_PATH


def lib():
    """Load the built library (build it first with __graft_entry__.build() or
    `python -m paper_2604_15180_amd.build`); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                f"{_LIB_PATH} is not built; run `python paper_2604_15180_amd/build.py` (needs hipcc). "
                "There is no fallback path.")
        L = ctypes.CDLL(_LIB_PATH)
        vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.entmax_attn_mask_tile.restype = ci
        L.entmax_attn_mask_tile.argtypes = []
        L.entmax_attn_histogram_bins.restype = ci
        L.entmax_attn_histogram_bins.argtypes = []
        L.entmax_attn_last_hip_error.restype = ci
        L.entmax_attn_last_hip_error.argtypes = []
        L.entmax_attn_workspace_bytes.restype = sz
        L.entmax_attn_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci, ci]
        L.entmax_attn_fwd.restype = ci
        L.entmax_attn_fwd.argtypes = [vp] * 7 + [ci, ci, ci, ci, ci, cf, ci, vp, sz, vp]
        L.entmax_attn_bwd.restype = ci
        L.entmax_attn_bwd.argtypes = [vp] * 10 + [ci, ci, ci, ci, ci, cf, ci, vp, sz, vp]
        L.entmax_attn_bwd_with_lists.restype = ci
        L.entmax_attn_bwd_with_lists.argtypes = [vp] * 8 + [sz] + [vp] * 3 + [ci, ci, ci, ci, ci, cf, ci, vp, sz, vp]
        L.entmax_attn_fwd_alpha_per_head.restype = ci
        L.entmax_attn_fwd_alpha_per_head.argtypes = [vp] * 7 + [ci, ci, ci, ci, ci, ctypes.POINTER(cf), ci, vp, sz, vp]
        L.entmax_attn_bwd_alpha_per_head.restype = ci
        L.entmax_attn_bwd_alpha_per_head.argtypes = [vp] * 10 + [ci, ci, ci, ci, ci, ctypes.POINTER(cf), ci, vp, sz, vp]
        L.entmax_attn_timer_enable.restype = ci
        L.entmax_attn_timer_enable.argtypes = [ci]
        L.entmax_attn_gather_enable.restype = ci
        L.entmax_attn_gather_enable.argtypes = [ci]
        L.entmax_attn_right_edge_enable.restype = ci
        L.entmax_attn_right_edge_enable.argtypes = [ci]
        L.entmax_attn_timer_read.restype = ci
        L.entmax_attn_timer_read.argtypes = [ctypes.POINTER(cf), ctypes.POINTER(ci), ci]
        L.entmax_attn_decode_workspace_bytes.restype = sz
        L.entmax_attn_decode_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
        L.entmax_attn_decode.restype = ci
        L.entmax_attn_decode.argtypes = [vp] * 7 + [ci, ci, ci, ci, ci, cf, vp, sz, vp]
        L.entmax_attn_decode_static_max_bytes.restype = sz
        L.entmax_attn_decode_static_max_bytes.argtypes = []
        L.entmax_attn_decode_static.restype = ci
        L.entmax_attn_decode_static.argtypes = [vp] * 7 + [ci, ci, ci, ci, ci, cf, vp]
        L.entmax_attn_fwd_histogram_bounds.restype = ci
        L.entmax_attn_fwd_histogram_bounds.argtypes = [vp, sz, ci, ci, ci, ci, ci, vp, vp, vp]
        L.entmax_attn_mfma_probe.restype = ci
        L.entmax_attn_mfma_probe.argtypes = [vp, vp, ci, ci, vp]
        L.entmax_attn_coissue_probe.restype = ci
        L.entmax_attn_coissue_probe.argtypes = [vp, ci, ci, ci, vp]
        L.entmax_attn_qk_norm_rope_fwd.restype = ci
        L.entmax_attn_qk_norm_rope_fwd.argtypes = [vp] * 10 + [ci] * 8 + [vp, ci, ci, cf, vp]
        L.entmax_attn_qk_norm_rope_workspace_bytes.restype = sz
        L.entmax_attn_qk_norm_rope_workspace_bytes.argtypes = [ci]
        L.entmax_attn_qk_norm_rope_bwd.restype = ci
        L.entmax_attn_qk_norm_rope_bwd.argtypes = [vp] * 16 + [ci] * 8 + [vp, ci, ci, cf, vp, sz, vp]
        L.entmax_attn_cache4_page_bytes.restype = sz
        L.entmax_attn_cache4_page_bytes.argtypes = [ci, ci, ci]
        L.entmax_attn_cache_tables.restype = ci
        L.entmax_attn_cache_tables.argtypes = [vp] * 10 + [ci] * 5 + [vp]
        L.entmax_attn_cache4_write.restype = ci
        L.entmax_attn_cache4_write.argtypes = [vp] * 6 + [ci] * 6 + [vp]
        L.entmax_attn_cache4_read.restype = ci
        L.entmax_attn_cache4_read.argtypes = [vp] * 6 + [ci] * 6 + [vp]
        L.entmax_attn_decode_cache4_workspace_bytes.restype = sz
        L.entmax_attn_decode_cache4_workspace_bytes.argtypes = [ci] * 5
        L.entmax_attn_decode_cache4.restype = ci
        L.entmax_attn_decode_cache4.argtypes = [vp] * 7 + [ci] * 9 + [cf, vp, sz, vp]
        L.entmax_attn_strerror.restype = ctypes.c_char_p
        L.entmax_attn_strerror.argtypes = [ci]
        _lib = L
    return _lib


def entmax_attn_mask_tile():
    return int(lib().entmax_attn_mask_tile())


def entmax_attn_histogram_bins():
    return int(lib().entmax_attn_histogram_bins())


def entmax_attn_strerror(code):
    return lib().entmax_attn_strerror(int(code)).decode()


def entmax_attn_workspace_bytes(B, H, N, d, dtype, causal, is_bwd):
    return int(lib().entmax_attn_workspace_bytes(B, H, N, d, _dtype_code(dtype), int(bool(causal)), int(bool(is_bwd))))


def _dtype_code(dtype):
    if dtype in (torch.float32, "f32", EA_F32):
        return EA_F32
    if dtype in (torch.bfloat16, "bf16", EA_BF16):
        return EA_BF16
    return 99   # the library answers EA_ERR_DTYPE


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _check(rc):
    if rc != 0:
        text = entmax_attn_strerror(rc)
        if rc == -6:
            text += f" (hipError {lib().entmax_attn_last_hip_error()})"
        raise EntmaxAttnError(rc, text)


def _workspace(nbytes, device):
    # torch's caching allocator returns 512-byte aligned blocks
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _prep(*tensors):
    first = tensors[0]
    for t in tensors:
        if not t.is_cuda:
            raise ValueError("entmax_attn: tensors must live on the GPU (there is no CPU path)")
        if not t.is_contiguous() or t.shape != first.shape or t.dtype != first.dtype:
            raise ValueError("entmax_attn: Q, K, V, dO must be contiguous [B,H,N,d] of one dtype")
    return first.shape


def _alpha_array(alpha, H):
    """None for a single alpha; else a ctypes array of H floats (one alpha per head)."""
    if isinstance(alpha, (int, float)):
        return None
    vals = [float(a) for a in (alpha.tolist() if hasattr(alpha, "tolist") else alpha)]
    if len(vals) != H:
        raise ValueError(f"entmax_attn: {len(vals)} alphas for {H} heads")
    return (ctypes.c_float * H)(*vals)


def entmax_attn_fwd(Q, K, V, alpha, causal, want_iters=False, workspace=None):
    """-> (O, tau, block_mask) or (O, tau, block_mask, iters).  `alpha`: one float, or a sequence of
    H floats (one per head).  The workspace used is kept in `entmax_attn_fwd.last_workspace` so
    that read_stats() can fetch the tile counters."""
    B, H, N, d = _prep(Q, K, V)
    dev = Q.device
    T = N // 64 if N % 64 == 0 else 0
    O = torch.empty((B, H, N, d), dtype=torch.float32, device=dev)
    tau = torch.empty((B, H, N), dtype=torch.float32, device=dev)
    mask = torch.empty((B, H, max(T, 1), max((T + 31) // 32, 1)), dtype=torch.int32, device=dev)
    iters = torch.empty((B, H, N), dtype=torch.int32, device=dev) if want_iters else None
    nbytes = entmax_attn_workspace_bytes(B, H, N, d, Q.dtype, causal, False)
    ws = workspace if workspace is not None else _workspace(nbytes, dev)
    stream = torch.cuda.current_stream(dev).cuda_stream
    per_head = _alpha_array(alpha, H)
    if per_head is None:
        rc = lib().entmax_attn_fwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(tau), _ptr(mask), _ptr(iters),
                                   B, H, N, d, _dtype_code(Q.dtype), float(alpha), int(bool(causal)),
                                   _ptr(ws), ws.numel(), ctypes.c_void_p(stream))
    else:
        rc = lib().entmax_attn_fwd_alpha_per_head(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(tau), _ptr(mask), _ptr(iters),
                                                  B, H, N, d, _dtype_code(Q.dtype), per_head, int(bool(causal)),
                                                  _ptr(ws), ws.numel(), ctypes.c_void_p(stream))
    _check(rc)
    entmax_attn_fwd.last_workspace = ws
    return (O, tau, mask, iters) if want_iters else (O, tau, mask)


def entmax_attn_fwd_histogram_bounds(workspace, B, H, N, d, dtype):
    """-> (tau0, upper) [B,H,N]: what the histogram stage alone gave in the last forward call that
    used `workspace` (start of the refinement and upper end of its bracket, raw convention)."""
    dev = workspace.device
    tau0 = torch.empty((B, H, N), dtype=torch.float32, device=dev)
    upper = torch.empty_like(tau0)
    _check(lib().entmax_attn_fwd_histogram_bounds(_ptr(workspace), workspace.numel(), B, H, N, d, _dtype_code(dtype),
                                                  _ptr(tau0), _ptr(upper), ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)))
    return tau0, upper


def entmax_attn_bwd(Q, K, V, O, dO, tau, alpha, causal, block_mask=None, workspace=None, fwd_workspace=None):
    """-> (dQ, dK, dV).  block_mask=None makes the library rebuild the mask from tau.  fwd_workspace:
    the forward call's workspace (entmax_attn_bwd_with_lists: the supports the forward listed are
    used instead of being found again; single alpha only)."""
    B, H, N, d = _prep(Q, K, V, dO)
    dev = Q.device
    dQ = torch.empty((B, H, N, d), dtype=torch.float32, device=dev)
    dK = torch.empty_like(dQ)
    dV = torch.empty_like(dQ)
    nbytes = entmax_attn_workspace_bytes(B, H, N, d, Q.dtype, causal, True)
    ws = workspace if workspace is not None else _workspace(nbytes, dev)
    stream = torch.cuda.current_stream(dev).cuda_stream
    per_head = _alpha_array(alpha, H)
    if fwd_workspace is not None:
        if per_head is not None:
            raise ValueError("entmax_attn_bwd: fwd_workspace goes with a single alpha")
        rc = lib().entmax_attn_bwd_with_lists(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(tau), _ptr(block_mask),
                                              _ptr(fwd_workspace), fwd_workspace.numel(), _ptr(dQ), _ptr(dK), _ptr(dV),
                                              B, H, N, d, _dtype_code(Q.dtype), float(alpha), int(bool(causal)),
                                              _ptr(ws), ws.numel(), ctypes.c_void_p(stream))
    elif per_head is None:
        rc = lib().entmax_attn_bwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(tau), _ptr(block_mask),
                                   _ptr(dQ), _ptr(dK), _ptr(dV), B, H, N, d, _dtype_code(Q.dtype), float(alpha),
                                   int(bool(causal)), _ptr(ws), ws.numel(), ctypes.c_void_p(stream))
    else:
        rc = lib().entmax_attn_bwd_alpha_per_head(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(tau), _ptr(block_mask),
                                                  _ptr(dQ), _ptr(dK), _ptr(dV), B, H, N, d, _dtype_code(Q.dtype), per_head,
                                                  int(bool(causal)), _ptr(ws), ws.numel(), ctypes.c_void_p(stream))
    _check(rc)
    entmax_attn_bwd.last_workspace = ws
    return dQ, dK, dV


def entmax_attn_decode_workspace_bytes(B, H, N, d, dtype):
    return int(lib().entmax_attn_decode_workspace_bytes(B, H, N, d, _dtype_code(dtype)))


def entmax_attn_decode_static_max_bytes():
    return int(lib().entmax_attn_decode_static_max_bytes())


def entmax_attn_decode_static(q, K, V, alpha, out=None):
    """entmax_attn_decode through the entry point that allocates nothing: the scratch is the
    library's own static array.  `out` = (O, tau, support, iters) tensors to write into (then this
    function allocates nothing either); without it they are made here with torch."""
    B, H, N, d = _check_decode_args(q, K, V)
    dev = K.device
    O, tau, support, iters = out if out is not None else _decode_outputs(B, H, d, dev)
    _check(lib().entmax_attn_decode_static(_ptr(q), _ptr(K), _ptr(V), _ptr(O), _ptr(tau), _ptr(support), _ptr(iters),
                                           B, H, N, d, _dtype_code(K.dtype), float(alpha),
                                           ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)))
    return O, tau, support, iters


def _decode_outputs(B, H, d, dev):
    return (torch.empty((B, H, d), dtype=torch.float32, device=dev), torch.empty((B, H), dtype=torch.float32, device=dev),
            torch.empty((B, H), dtype=torch.int32, device=dev), torch.empty((B, H), dtype=torch.int32, device=dev))


def _check_decode_args(q, K, V):
    for t in (q, K, V):
        if not t.is_cuda:
            raise ValueError("entmax_attn_decode: tensors must live on the GPU (there is no CPU path)")
    if K.dim() != 4 or K.shape != V.shape or q.shape != K.shape[:2] + K.shape[3:] or not (
            q.is_contiguous() and K.is_contiguous() and V.is_contiguous()) or not (q.dtype == K.dtype == V.dtype):
        raise ValueError("entmax_attn_decode: q [B,H,d], K, V [B,H,N,d], contiguous, of one dtype")
    return K.shape


def entmax_attn_decode(q, K, V, alpha, workspace=None):
    """One query per head against all cached keys: q [B,H,d], K, V [B,H,N,d] -> (O [B,H,d], tau [B,H],
    support [B,H], iters [B,H])."""
    B, H, N, d = _check_decode_args(q, K, V)
    dev = K.device
    O, tau, support, iters = _decode_outputs(B, H, d, dev)
    ws = workspace if workspace is not None else _workspace(entmax_attn_decode_workspace_bytes(B, H, N, d, K.dtype), dev)
    _check(lib().entmax_attn_decode(_ptr(q), _ptr(K), _ptr(V), _ptr(O), _ptr(tau), _ptr(support), _ptr(iters),
                                    B, H, N, d, _dtype_code(K.dtype), float(alpha), _ptr(ws), ws.numel(),
                                    ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)))
    return O, tau, support, iters


# ---- queries and keys from a layer's projections; the 4-bit cache --------------------------------

# These calls are made once a layer and token in a serving program, where a kernel takes a few microseconds: what the binding does
# around the library's call counts.  Devices are compared as integers, pointers passed as integers, and the stream is asked for without
# making a Stream object (entmax_attn_cache_tables: 14.6 -> 11.4 us of host time a call,
# of which the launch is 3).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on_gpu(call, first, *others):
    """Index of the one device of the tensors (None is skipped)."""
    dev = first.get_device()
    if dev < 0:
        raise ValueError(f"{call}: tensors must live on the GPU (there is no CPU path)")
    for t in others:
        if t is not None and t.get_device() != dev:
            if not t.is_cuda:
                raise ValueError(f"{call}: tensors must live on the GPU (there is no CPU path)")
            raise ValueError(f"{call}: tensors on GPU {dev} and GPU {t.get_device()}")
    return dev


def _launch(dev, function, *args):
    """Calls the library with `args` and the current stream of device `dev`, with that device current."""
    before = torch.cuda.current_device()
    if before == dev:
        rc = function(*args, _raw_stream(dev))
    else:
        torch.cuda.set_device(dev)
        try:
            rc = function(*args, _raw_stream(dev))
        finally:
            torch.cuda.set_device(before)
    if rc:
        _check(rc)


def _workspace_arg(call, t):
    """A caller's workspace is taken as all its bytes from its first one on: those of an expanded view are not there."""
    if t is not None and not t.is_contiguous():
        raise ValueError(f"{call}: workspace must be contiguous")


def _at(t):
    return None if t is None else t.data_ptr()


def _int32(call, name, t, shape):
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{call}: {name} must be contiguous int32 {list(shape)}, got {t.dtype} {list(t.shape)}")


_TwoStrides, _ThreeStrides = ctypes.c_int64 * 2, ctypes.c_int64 * 3


def _prep_args(call, q, k, positions, inv_freq, q_weight, k_weight, norm, sections):
    if q.dim() != 4 or k.dim() != 4 or q.shape[:2] != k.shape[:2] or q.shape[3] != k.shape[3] or q.dtype != k.dtype:
        raise ValueError(f"{call}: q [B,N,Hq,d], k [B,N,Hk,d] of one dtype")
    if q.stride(3) != 1 or k.stride(3) != 1:
        raise ValueError(f"{call}: the elements of a row of q and k must be contiguous")
    B, N, Hq, d = q.shape
    rot = axes = 0
    if inv_freq is not None and inv_freq.numel() > 0:
        rot = 2 * inv_freq.numel()
        if inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous():
            raise ValueError(f"{call}: inv_freq must be contiguous float32 [rot / 2]")
        if positions is None:
            raise ValueError(f"{call}: inv_freq without positions")
        axes = positions.shape[0] if positions.dim() == 3 else 1
        _int32(call, "positions", positions, (axes, B, N) if positions.dim() == 3 else (B, N))
        if sections is not None and len(sections) != axes:
            raise ValueError(f"{call}: {len(sections)} sections for {axes} position axes")
    for w in (q_weight, k_weight):
        if w is not None and (w.dtype != torch.float32 or w.shape != (d,) or not w.is_contiguous()):
            raise ValueError(f"{call}: a weight must be contiguous float32 [{d}]")
    if not norm and (q_weight is not None or k_weight is not None):
        raise ValueError(f"{call}: weights go with norm=True")
    sec = (ctypes.c_int * axes)(*sections) if rot and sections is not None else None
    return B, N, Hq, k.shape[2], d, rot, axes, sec


def _row_strides(t):
    a, b, c, _ = t.stride()
    if (a | b | c) & 7:     # (of a dimension of one torch keeps any stride; no row is a step along it away)
        a, b, c = (0 if n == 1 else s for n, s in zip(t.shape, (a, b, c)))
    return _ThreeStrides(a, b, c)


def entmax_attn_qk_norm_rope_fwd(q, k, positions, inv_freq, q_weight=None, k_weight=None, eps=1e-6, norm=True, sections=None,
                                 interleaved=False):
    """q [B,N,Hq,d], k [B,N,Hk,d] (any strides between rows) -> q_out [B,Hq,N,d], k_out [B,Hk,N,d], normed per head
    and rotated.  positions: int32 [B,N], or [axes,B,N] with `sections` pairs for each axis; inv_freq: float32 [rot / 2], None
    for no rotation."""
    call = "entmax_attn_qk_norm_rope_fwd"
    dev = _on_gpu(call, q, k, positions, inv_freq, q_weight, k_weight)
    B, N, Hq, Hk, d, rot, axes, sec = _prep_args(call, q, k, positions, inv_freq, q_weight, k_weight, norm, sections)
    q_out, k_out = q.new_empty((B, Hq, N, d)), q.new_empty((B, Hk, N, d))
    _launch(dev, lib().entmax_attn_qk_norm_rope_fwd, q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), _row_strides(q),
            _row_strides(k), _at(q_weight), _at(k_weight), _at(positions), _at(inv_freq), B, Hq, Hk, N, d, _dtype_code(q.dtype), rot, axes,
            sec, bool(interleaved), bool(norm), float(eps))
    return q_out, k_out


def entmax_attn_qk_norm_rope_workspace_bytes(d):
    return int(lib().entmax_attn_qk_norm_rope_workspace_bytes(d))


def entmax_attn_qk_norm_rope_bwd(q, k, dq_out, dk_out, positions, inv_freq, q_weight=None, k_weight=None, eps=1e-6, norm=True,
                                 sections=None, interleaved=False, out=None, workspace=None):
    """The gradient: dq_out [B,Hq,N,d], dk_out [B,Hk,N,d] float32 (entmax_attn_bwd's dQ, dK) -> (dq, dk, dq_weight, dk_weight),
    dq, dk like q, k (contiguous, or `out` = (dq, dk) views to write into), weight gradients float32 [d], None for a weight that
    was None."""
    call = "entmax_attn_qk_norm_rope_bwd"
    _workspace_arg(call, workspace)
    dev = _on_gpu(call, q, k, dq_out, dk_out, positions, inv_freq, q_weight, k_weight, workspace, *(out or ()))
    B, N, Hq, Hk, d, rot, axes, sec = _prep_args(call, q, k, positions, inv_freq, q_weight, k_weight, norm, sections)
    for g, H in ((dq_out, Hq), (dk_out, Hk)):
        if g.dtype != torch.float32 or g.shape != (B, H, N, d) or not g.is_contiguous():
            raise ValueError(f"{call}: dq_out, dk_out must be contiguous float32 [B,H,N,d]")
    if out is None:
        dq, dk = q.new_empty((B, N, Hq, d)), q.new_empty((B, N, Hk, d))
    else:
        dq, dk = out
        if dq.shape != q.shape or dk.shape != k.shape or dq.dtype != q.dtype or dk.dtype != q.dtype or dq.stride(3) != 1 or dk.stride(3) != 1:
            raise ValueError(f"{call}: out must be of q's and k's shapes and dtype, rows contiguous")
    dwq, dwk = (None if w is None else w.new_empty(d) for w in (q_weight, k_weight))
    ws = workspace
    if ws is None and (dwq is not None or dwk is not None):
        ws = _workspace(entmax_attn_qk_norm_rope_workspace_bytes(d), q.device)
    _launch(dev, lib().entmax_attn_qk_norm_rope_bwd, q.data_ptr(), k.data_ptr(), dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(),
            dk.data_ptr(), _row_strides(q), _row_strides(k), _row_strides(dq), _row_strides(dk), _at(q_weight), _at(k_weight),
            _at(positions), _at(inv_freq), _at(dwq), _at(dwk), B, Hq, Hk, N, d, _dtype_code(q.dtype), rot, axes, sec, bool(interleaved),
            bool(norm), float(eps), _at(ws), 0 if ws is None else ws.numel() * ws.element_size())
    return dq, dk, dwq, dwk


def entmax_attn_cache_tables(lens, new_lens, block_table, free_pages, free_count, page_size, max_tokens, out=None):
    """One scheduler step on the GPU: requests go from lens [R] to new_lens [R] tokens.  block_table [R,max_blocks], the stack
    free_pages [n_pages] and free_count [1] (all int32) are updated in place -> (lens_out [R], token_start [R+1], slots
    [max_tokens], positions [max_tokens], status [4]), int32; `out`: tensors to write them into (lens_out may be lens)."""
    call = "entmax_attn_cache_tables"
    if out is not None and len(out) != 5:       # (each goes to the library as a pointer of its own)
        raise ValueError(f"{call}: out must be (lens_out, token_start, slots, positions, status), got {len(out)} tensors")
    dev = _on_gpu(call, lens, new_lens, block_table, free_pages, free_count, *(out or ()))
    if block_table.dim() != 2 or free_pages.dim() != 1:
        raise ValueError(f"{call}: block_table [R,max_blocks], free_pages [n_pages]")
    R, blocks = block_table.shape
    shapes = ((R,), (R + 1,), (max_tokens,), (max_tokens,), (4,))
    for name, t, shape in (("lens", lens, (R,)), ("new_lens", new_lens, (R,)), ("block_table", block_table, (R, blocks)),
                           ("free_pages", free_pages, free_pages.shape), ("free_count", free_count, (1,))):
        _int32(call, name, t, shape)
    if out is None:
        if max_tokens < 0:
            raise ValueError(f"{call}: max_tokens must not be negative")
        out = torch.empty(2 * R + 5 + 2 * max_tokens, dtype=torch.int32, device=lens.device).split_with_sizes([R, R + 1, max_tokens, max_tokens, 4])
    else:
        for name, t, shape in zip(("lens_out", "token_start", "slots", "positions", "status"), out, shapes):
            _int32(call, name, t, shape)
    _launch(dev, lib().entmax_attn_cache_tables, lens.data_ptr(), new_lens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
            free_count.data_ptr(), *[t.data_ptr() for t in out], R, blocks, page_size, free_pages.numel(), max_tokens)
    return tuple(out)


def entmax_attn_cache4_page_bytes(Hk, d, page_size):
    return int(lib().entmax_attn_cache4_page_bytes(Hk, d, page_size))


def entmax_attn_cache4_empty(n_pages, Hk, d, page_size, device="cuda"):
    """A cache of n_pages pages: uint8 [n_pages, Hk, page_size * 17 d / 16], all values zero."""
    nbytes = entmax_attn_cache4_page_bytes(Hk, d, page_size)
    if nbytes == 0 or n_pages <= 0:
        raise ValueError("entmax_attn_cache4_empty: Hk, n_pages > 0, d 64 or 128, page_size 16, 32, 64, 128 or 256")
    return torch.zeros((n_pages, Hk, nbytes // Hk), dtype=torch.uint8, device=device)


def _cache_args(call, cache, d, page_size):
    if cache.dtype != torch.uint8 or cache.dim() != 3 or not cache.is_contiguous() or cache.shape[2] * 16 != page_size * d * 17:
        raise ValueError(f"{call}: cache must be contiguous uint8 [n_pages, Hk, page_size * 17 d / 16]")
    return cache.shape[0], cache.shape[1]


def _token_strides(t):
    a, b, _ = t.stride()
    if (a | b) & 7:         # (as in _row_strides)
        a, b = (0 if n == 1 else s for n, s in zip(t.shape, (a, b)))
    return _TwoStrides(a, b)


def _cache_rows(call, k, v, slots, Hk):
    if k.dim() != 3 or k.shape != v.shape or k.shape[1] != Hk or k.dtype != v.dtype:
        raise ValueError(f"{call}: K, V must be [T,Hk,d] of one dtype, with the cache's Hk")
    if k.numel() and (k.stride(2) != 1 or v.stride(2) != 1):
        raise ValueError(f"{call}: the elements of a row must be contiguous")
    _int32(call, "slots", slots, (k.shape[0],))
    return _token_strides(k), _token_strides(v)


def entmax_attn_cache4_write(K, V, slots, cache, page_size):
    """K, V [T,Hk,d] (any strides between rows) to the slots [T] (int32; negative: skipped) of a 4-bit cache."""
    call = "entmax_attn_cache4_write"
    dev = _on_gpu(call, K, V, slots, cache)
    d = K.shape[-1]
    pages, Hk = _cache_args(call, cache, d, page_size)
    ks, vs = _cache_rows(call, K, V, slots, Hk)
    _launch(dev, lib().entmax_attn_cache4_write, K.data_ptr(), V.data_ptr(), ks, vs, slots.data_ptr(), cache.data_ptr(), K.shape[0], Hk, d,
            _dtype_code(K.dtype), pages, page_size)


def entmax_attn_cache4_read(cache, slots, page_size, d, dtype=torch.bfloat16, out=None):
    """The rows of the slots [T] as the cache holds them -> (K, V) [T,Hk,d]; `out` = (K, V) to write into (any strides between
    rows; rows of negative slots are left as they were, and are undefined without `out`)."""
    call = "entmax_attn_cache4_read"
    dev = _on_gpu(call, cache, slots, *(out or ()))
    pages, Hk = _cache_args(call, cache, d, page_size)
    if out is None:
        out = (cache.new_empty((slots.numel(), Hk, d), dtype=dtype), cache.new_empty((slots.numel(), Hk, d), dtype=dtype))
    K, V = out
    if K.shape[-1] != d:
        raise ValueError(f"{call}: out must be [T,Hk,{d}]")
    ks, vs = _cache_rows(call, K, V, slots, Hk)
    _launch(dev, lib().entmax_attn_cache4_read, cache.data_ptr(), slots.data_ptr(), K.data_ptr(), V.data_ptr(), ks, vs, K.shape[0], Hk, d,
            _dtype_code(K.dtype), pages, page_size)
    return K, V


def entmax_attn_decode_cache4_workspace_bytes(R, Hq, Hk, d, max_len):
    return int(lib().entmax_attn_decode_cache4_workspace_bytes(R, Hq, Hk, d, max_len))


def entmax_attn_decode_cache4(q, cache, block_table, lens, alpha, page_size, max_len=None, workspace=None):
    """One query per head and request against a 4-bit cache: q [R,Hq,d], block_table [R,max_blocks], lens [R] (int32) ->
    (O [R,Hq,d], tau [R,Hq], support [R,Hq]).  max_len: the largest length there can be (default: all that the table's pages
    hold); launch and workspace go by it.  workspace: entmax_attn_decode_cache4_workspace_bytes bytes, about 4 R Hq max_len; without it
    they are allocated in every call."""
    call = "entmax_attn_decode_cache4"
    _workspace_arg(call, workspace)
    dev = _on_gpu(call, q, cache, block_table, lens, workspace)
    if q.dim() != 3 or not q.is_contiguous() or block_table.dim() != 2:
        raise ValueError(f"{call}: q contiguous [R,Hq,d], block_table [R,max_blocks]")
    R, Hq, d = q.shape
    pages, Hk = _cache_args(call, cache, d, page_size)
    _int32(call, "block_table", block_table, (R, block_table.shape[1]))
    _int32(call, "lens", lens, (R,))
    blocks = block_table.shape[1]
    if max_len is None:
        max_len = blocks * page_size
    O, tau, support = q.new_empty((R, Hq, d), dtype=torch.float32), q.new_empty((R, Hq), dtype=torch.float32), lens.new_empty((R, Hq))
    ws = workspace if workspace is not None else _workspace(entmax_attn_decode_cache4_workspace_bytes(R, Hq, Hk, d, max_len), q.device)
    _launch(dev, lib().entmax_attn_decode_cache4, q.data_ptr(), cache.data_ptr(), block_table.data_ptr(), lens.data_ptr(), O.data_ptr(),
            tau.data_ptr(), support.data_ptr(), R, Hq, Hk, d, _dtype_code(q.dtype), max_len, blocks, pages, page_size, float(alpha),
            ws.data_ptr(), ws.numel() * ws.element_size())
    return O, tau, support


def entmax_attn_mfma_probe(data, sink, groups, iters):
    """Enqueue the matrix-core rate probe on the current stream (data: >= 8192 fp16 values on the
    GPU, sink: >= groups * 256 floats). Returns the flops the launch performs."""
    if not (data.is_cuda and sink.is_cuda and data.dtype == torch.float16 and data.numel() >= 8192
            and sink.dtype == torch.float32 and sink.numel() >= groups * 256):
        raise ValueError("entmax_attn_mfma_probe: data = 8192 fp16 values, sink = groups * 256 floats, both on the GPU")
    _check(lib().entmax_attn_mfma_probe(_ptr(data), _ptr(sink), int(groups), int(iters),
                                         ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))
    return float(groups) * 4 * iters * 32 * 32768.0


def entmax_attn_coissue_probe(sink, iters, valu_per_round, with_mfma):
    """Enqueue the co-issue probe on the current stream (sink: >= 512 * 512 floats on the GPU)."""
    if not (sink.is_cuda and sink.dtype == torch.float32 and sink.numel() >= 512 * 512):
        raise ValueError("entmax_attn_coissue_probe: sink = 512 * 512 floats on the GPU")
    _check(lib().entmax_attn_coissue_probe(_ptr(sink), int(iters), int(valu_per_round), int(bool(with_mfma)),
                                            ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))


def entmax_attn_right_edge_enable(on):
    """Approximate forward from right-edge binning, no refinement (this thread's later forward calls)."""
    _check(lib().entmax_attn_right_edge_enable(int(bool(on))))


def entmax_attn_gather_enable(on):
    _check(lib().entmax_attn_gather_enable(int(bool(on))))


def entmax_attn_timer_enable(on):
    _check(lib().entmax_attn_timer_enable(int(bool(on))))


def entmax_attn_timer_read():
    """-> {kernel name: (summed ms, launches)} since the last read (waits for the events)."""
    ms = (ctypes.c_float * EA_TIMER_SLOTS)()
    cnt = (ctypes.c_int * EA_TIMER_SLOTS)()
    _check(lib().entmax_attn_timer_read(ms, cnt, EA_TIMER_SLOTS))
    return {TIMER_NAMES[k]: (float(ms[k]), int(cnt[k])) for k in range(EA_TIMER_SLOTS) if cnt[k]}


def read_stats(workspace):
    """Executed-tile counters of the last call that used `workspace` (synchronises)."""
    copies = workspace[: EA_STATS_COPIES * EA_STATS_WORDS * 8].view(torch.int64).view(EA_STATS_COPIES, EA_STATS_WORDS)
    return dict(zip(STAT_NAMES, copies.cpu().sum(0).tolist()))
