"""HiFA4 on MI355X: Python binding of libhifa4 (the C ABI in include/hifa4.h).

The binding only marshals arguments: torch tensors supply device memory and
the current HIP stream; every step of the computation runs in the library's
HIP kernels.  The shared library is loaded on first use from this package's
directory and a missing or stale build raises immediately -- there is no
fallback implementation.

Names mirror the C entry points:
  hifa4_calibrate_smooth_qk, hifa4_calibrate_smooth_qk_layers, hifa4_quantize_qk, hifa4_quantize_v,
  hifa4_attention_fwd, hifa4_workspace_bytes, hifa4_decode_fwd,
  hifa4_decode_workspace_bytes, hifa4_paged_page_bytes, hifa4_paged_append,
  hifa4_paged_gather, hifa4_paged_decode_fwd, hifa4_paged_decode_workspace_bytes,
  hifa4_paged_evict, hifa4_paged_chunk_fwd, hifa4_paged_chunk_workspace_bytes,
  hifa4_paged_extend, hifa4_paged_release, hifa4_rope, hifa4_selftest_exp2,
  hifa4_last_error.
"""
from __future__ import annotations

import ctypes
import os
import threading
from dataclasses import dataclass
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhifa4.so")

NORM_PREORDER, NORM_INCONSISTENT = 0, 1
OPERANDS_HIF4, OPERANDS_FP16, OPERANDS_P_ONLY = 0, 1, 2
STATUS = {0: "HIFA4_OK", -1: "HIFA4_ERR_INVALID_ARGUMENT", -2: "HIFA4_ERR_UNSUPPORTED",
          -3: "HIFA4_ERR_WORKSPACE", -4: "HIFA4_ERR_HIP"}

EXPORTED = ("hifa4_workspace_bytes", "hifa4_calibrate_workspace_bytes", "hifa4_calibrate_smooth_qk",
            "hifa4_calibrate_smooth_qk_layers",
            "hifa4_quantize_qk", "hifa4_quantize_v", "hifa4_attention_fwd", "hifa4_decode_workspace_bytes",
            "hifa4_decode_fwd", "hifa4_paged_page_bytes", "hifa4_paged_append", "hifa4_paged_gather",
            "hifa4_paged_decode_workspace_bytes", "hifa4_paged_decode_fwd", "hifa4_paged_evict",
            "hifa4_paged_chunk_workspace_bytes", "hifa4_paged_chunk_fwd", "hifa4_paged_extend",
            "hifa4_paged_release_workspace_bytes", "hifa4_paged_release", "hifa4_rope_frequencies", "hifa4_rope",
            "hifa4_selftest_exp2", "hifa4_last_error", "hifa4_attention_fwd_noalloc")
NOALLOC_SCRATCH_BYTES = 32 << 20
PAGE_TOKENS = 64


class Problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_heads_q", ctypes.c_int32),
                ("num_heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_seqlen", ctypes.c_int32), ("cu_seqlens", ctypes.c_void_p),
                ("total_tokens", ctypes.c_int32), ("causal", ctypes.c_int32)]


class FwdOptions(ctypes.Structure):
    _fields_ = [("norm", ctypes.c_int32), ("operands", ctypes.c_int32), ("smooth_qk", ctypes.c_int32),
                ("debug_p_codes", ctypes.c_void_p), ("debug_p_meta", ctypes.c_void_p),
                ("timing_events", ctypes.c_void_p), ("q_mean", ctypes.c_int32),
                ("test_decode_no_publish", ctypes.c_int32),
                ("debug_head_begin", ctypes.c_int32), ("debug_head_count", ctypes.c_int32),
                ("debug_token_begin", ctypes.c_int32), ("debug_token_count", ctypes.c_int32)]


class PagedCacheDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("operands", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("pool", ctypes.c_void_p), ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
                ("v_tail", ctypes.c_void_p)]


class CalibReport(ctypes.Structure):
    _fields_ = [("rho_k", ctypes.c_double), ("t_kq", ctypes.c_double), ("branch", ctypes.c_int32),
                ("alpha_used", ctypes.c_float)]


class Hifa4Error(RuntimeError):
    pass


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libhifa4.so (once).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"libhifa4.so not found at {path}; build it first "
                          "(python -m paper_2607_04302_amd.build or __graft_entry__.build())")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.hifa4_workspace_bytes.restype = sz
    lib.hifa4_workspace_bytes.argtypes = [P(Problem), P(FwdOptions)]
    lib.hifa4_calibrate_workspace_bytes.restype = sz
    lib.hifa4_calibrate_workspace_bytes.argtypes = [P(Problem), ctypes.c_int32]
    lib.hifa4_calibrate_smooth_qk.restype = ctypes.c_int
    lib.hifa4_calibrate_smooth_qk.argtypes = [P(Problem), ctypes.c_int32, vp, vp, ctypes.c_float, vp,
                                              P(CalibReport), vp, sz, vp]
    lib.hifa4_calibrate_smooth_qk_layers.restype = ctypes.c_int
    lib.hifa4_calibrate_smooth_qk_layers.argtypes = [P(Problem), ctypes.c_int32, ctypes.c_int32, vp, vp,
                                                     ctypes.c_float, vp, P(CalibReport), vp, sz, vp]
    lib.hifa4_quantize_qk.restype = ctypes.c_int
    lib.hifa4_quantize_qk.argtypes = [P(Problem), vp, vp, vp, vp, vp, vp, vp, vp]
    lib.hifa4_quantize_v.restype = ctypes.c_int
    lib.hifa4_quantize_v.argtypes = [P(Problem), vp, vp, vp, vp]
    lib.hifa4_attention_fwd.restype = ctypes.c_int
    lib.hifa4_attention_fwd.argtypes = [P(Problem), P(FwdOptions), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hifa4_attention_fwd_noalloc.restype = ctypes.c_int
    lib.hifa4_attention_fwd_noalloc.argtypes = [P(Problem), P(FwdOptions), vp, vp, vp, vp, vp, vp, vp]
    lib.hifa4_decode_workspace_bytes.restype = sz
    lib.hifa4_decode_workspace_bytes.argtypes = [P(Problem)]
    lib.hifa4_decode_fwd.restype = ctypes.c_int
    lib.hifa4_decode_fwd.argtypes = [P(Problem), P(FwdOptions), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    i32 = ctypes.c_int32
    lib.hifa4_paged_page_bytes.restype = sz
    lib.hifa4_paged_page_bytes.argtypes = [i32, i32, i32]
    lib.hifa4_paged_append.restype = ctypes.c_int
    lib.hifa4_paged_append.argtypes = [P(PagedCacheDesc), i32, i32, vp, vp, vp, vp, vp]
    lib.hifa4_paged_gather.restype = ctypes.c_int
    lib.hifa4_paged_gather.argtypes = [P(PagedCacheDesc), i32, i32, vp, vp, vp, vp, vp]
    lib.hifa4_paged_decode_workspace_bytes.restype = sz
    lib.hifa4_paged_decode_workspace_bytes.argtypes = [P(PagedCacheDesc), i32, i32]
    lib.hifa4_paged_decode_fwd.restype = ctypes.c_int
    lib.hifa4_paged_decode_fwd.argtypes = [P(PagedCacheDesc), i32, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, sz, vp]
    lib.hifa4_paged_evict.restype = ctypes.c_int
    lib.hifa4_paged_evict.argtypes = [i32, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    i64 = ctypes.c_int64
    lib.hifa4_paged_chunk_workspace_bytes.restype = sz
    lib.hifa4_paged_chunk_workspace_bytes.argtypes = [P(PagedCacheDesc), i32, i32, i32]
    lib.hifa4_paged_chunk_fwd.restype = ctypes.c_int
    lib.hifa4_paged_chunk_fwd.argtypes = [P(PagedCacheDesc), i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hifa4_paged_extend.restype = ctypes.c_int
    lib.hifa4_paged_extend.argtypes = [i32, i32, vp, vp, vp, vp, i32, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.hifa4_paged_release_workspace_bytes.restype = sz
    lib.hifa4_paged_release_workspace_bytes.argtypes = [i32]
    lib.hifa4_paged_release.restype = ctypes.c_int
    lib.hifa4_paged_release.argtypes = [i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.hifa4_rope_frequencies.restype = ctypes.c_int
    lib.hifa4_rope_frequencies.argtypes = [i32] + [ctypes.c_double, i32] + [ctypes.c_double] * 4 + [vp]
    lib.hifa4_rope.restype = ctypes.c_int
    lib.hifa4_rope.argtypes = [i32, i32, i32, i32, ctypes.c_float, vp, i32, vp, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, vp]
    lib.hifa4_selftest_exp2.restype = ctypes.c_int
    lib.hifa4_selftest_exp2.argtypes = [vp, vp, ctypes.c_int64, vp]
    lib.hifa4_last_error.restype = ctypes.c_char_p
    lib.hifa4_last_error.argtypes = []
    _lib = lib
    return lib


def hifa4_last_error() -> str:
    return load_library().hifa4_last_error().decode()


def _check(status: int, what: str):
    if status != 0:
        raise Hifa4Error(f"{what}: {STATUS.get(status, status)}: {hifa4_last_error()}")


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(device) -> int:
    # the handle of torch.cuda.current_stream(device) without the Stream object around it
    return _torch()._C._cuda_getCurrentRawStream(device.index)


def _require(t, dtype, name):
    if t is None:
        return
    if t.is_cuda and t.dtype == dtype and t.is_contiguous():
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must be contiguous")


@dataclass
class Shape:
    batch: int
    heads_q: int
    heads_kv: int
    head_dim: int
    max_seqlen: int
    tokens: int
    cu_seqlens: object = None

    def problem(self) -> Problem:
        return Problem(self.batch, self.heads_q, self.heads_kv, self.head_dim, self.max_seqlen,
                       _ptr(self.cu_seqlens), self.tokens if self.cu_seqlens is not None else 0, 1)


def shape_of(q, k, cu_seqlens=None, max_seqlen=None) -> Shape:
    """Problem shape from Q [B,S,Hq,D] (BSHD) or Q [T,Hq,D] + cu_seqlens (THD)."""
    if cu_seqlens is None:
        if q.dim() != 4:
            raise ValueError("fixed-length inputs are [batch, seqlen, heads, dim]")
        b, s, hq, d = q.shape
        return Shape(b, hq, k.shape[2], d, s, b * s)
    if q.dim() != 3:
        raise ValueError("variable-length inputs are [total_tokens, heads, dim] with cu_seqlens")
    if max_seqlen is None:
        raise ValueError("max_seqlen is required with cu_seqlens")
    _require(cu_seqlens, _torch().int32, "cu_seqlens")
    t, hq, d = q.shape
    return Shape(cu_seqlens.numel() - 1, hq, k.shape[1], d, int(max_seqlen), t, cu_seqlens)


def hifa4_workspace_bytes(shape: Shape, operands: int = OPERANDS_HIF4, q_mean: bool = False) -> int:
    lib = load_library()
    p = shape.problem()
    o = FwdOptions(NORM_PREORDER, operands, 0, None, None, None, 1 if q_mean else 0)
    return int(lib.hifa4_workspace_bytes(ctypes.byref(p), ctypes.byref(o)))


def hifa4_calibrate_smooth_qk(q_cal, k_cal, alpha: float):
    """q_cal [n, S, Hq, D], k_cal [n, S, Hkv, D] fp16 on the GPU.  Returns
    (s fp32 [Hkv, D] on the GPU, report dict).  Synchronizes the stream."""
    torch = _torch()
    _require(q_cal, torch.float16, "q_cal")
    _require(k_cal, torch.float16, "k_cal")
    lib = load_library()
    n, s, hq, d = q_cal.shape
    hkv = k_cal.shape[2]
    p = Problem(1, hq, hkv, d, s, None, 0, 1)
    ws_bytes = int(lib.hifa4_calibrate_workspace_bytes(ctypes.byref(p), n))
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=q_cal.device)
    out = torch.empty((hkv, d), dtype=torch.float32, device=q_cal.device)
    rep = CalibReport()
    _check(lib.hifa4_calibrate_smooth_qk(ctypes.byref(p), n, _ptr(q_cal), _ptr(k_cal), float(alpha),
                                         _ptr(out), ctypes.byref(rep), _ptr(ws), ws_bytes,
                                         _stream(q_cal.device)), "hifa4_calibrate_smooth_qk")
    return out, {"rho_k": rep.rho_k, "t_kq": rep.t_kq, "branch": rep.branch, "alpha_used": rep.alpha_used}


def hifa4_calibrate_smooth_qk_layers(q_cal, k_cal, alpha: float):
    """q_cal [L, n, S, Hq, D], k_cal [L, n, S, Hkv, D] fp16 on the GPU (L
    layers).  Returns (s fp32 [L, Hkv, D] on the GPU, list of L report dicts).
    Synchronizes the stream."""
    torch = _torch()
    _require(q_cal, torch.float16, "q_cal")
    _require(k_cal, torch.float16, "k_cal")
    lib = load_library()
    n_layers, n, s, hq, d = q_cal.shape
    hkv = k_cal.shape[3]
    p = Problem(1, hq, hkv, d, s, None, 0, 1)
    ws_bytes = int(lib.hifa4_calibrate_workspace_bytes(ctypes.byref(p), n))
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=q_cal.device)
    out = torch.empty((n_layers, hkv, d), dtype=torch.float32, device=q_cal.device)
    reps = (CalibReport * n_layers)()
    _check(lib.hifa4_calibrate_smooth_qk_layers(ctypes.byref(p), n_layers, n, _ptr(q_cal), _ptr(k_cal),
                                                float(alpha), _ptr(out), reps, _ptr(ws), ws_bytes,
                                                _stream(q_cal.device)), "hifa4_calibrate_smooth_qk_layers")
    return out, [{"rho_k": r.rho_k, "t_kq": r.t_kq, "branch": r.branch, "alpha_used": r.alpha_used} for r in reps]


def hifa4_quantize_qk(q, k, s=None, cu_seqlens=None, max_seqlen=None):
    """Canonical HIF4 codes of Smooth-QK'd Q and K.  Returns (q_codes uint8
    [T,Hq,D/64,32], q_meta int32 [T,Hq,D/64], k_codes, k_meta) -- meta words
    are uint32 bit patterns held in int32 tensors.  q=None quantizes K only
    (q_codes and q_meta are then None)."""
    torch = _torch()
    _require(q, torch.float16, "q")
    _require(k, torch.float16, "k")
    _require(s, torch.float32, "s")
    sh = shape_of(k if q is None else q, k, cu_seqlens, max_seqlen)
    lib = load_library()
    g = sh.head_dim // 64
    dev = k.device
    qc = qm = None
    if q is not None:
        qc = torch.empty((sh.tokens, sh.heads_q, g, 32), dtype=torch.uint8, device=dev)
        qm = torch.empty((sh.tokens, sh.heads_q, g), dtype=torch.int32, device=dev)
    kc = torch.empty((sh.tokens, sh.heads_kv, g, 32), dtype=torch.uint8, device=dev)
    km = torch.empty((sh.tokens, sh.heads_kv, g), dtype=torch.int32, device=dev)
    p = sh.problem()
    _check(lib.hifa4_quantize_qk(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(s), _ptr(qc), _ptr(qm), _ptr(kc),
                                 _ptr(km), _stream(dev)), "hifa4_quantize_qk")
    return qc, qm, kc, km


def hifa4_quantize_v(v, cu_seqlens=None, max_seqlen=None):
    """Canonical HIF4 codes of V along tokens: (codes uint8 [B, NB, Hkv, D, 32],
    meta int32 [B, NB, Hkv, D])."""
    torch = _torch()
    _require(v, torch.float16, "v")
    sh = shape_of(v, v, cu_seqlens, max_seqlen)
    lib = load_library()
    nb = (sh.max_seqlen + 63) // 64
    vc = torch.empty((sh.batch, nb, sh.heads_kv if cu_seqlens is None else v.shape[1], sh.head_dim, 32),
                     dtype=torch.uint8, device=v.device)
    sh.heads_kv = vc.shape[2]
    sh.heads_q = vc.shape[2]
    vm = torch.empty(vc.shape[:-1], dtype=torch.int32, device=v.device)
    p = sh.problem()
    _check(lib.hifa4_quantize_v(ctypes.byref(p), _ptr(v), _ptr(vc), _ptr(vm), _stream(v.device)), "hifa4_quantize_v")
    return vc, vm


class Workspace:
    """A reusable device workspace (grown on demand).  One call at a time may
    use it: calls on several streams or threads take one each, and a captured
    call keeps the buffer that it was captured with."""

    def __init__(self):
        self.buf = None

    def get(self, nbytes: int, device):
        buf = self.buf
        if buf is None or buf.numel() < nbytes or buf.device != device:
            torch = _torch()
            self.buf = buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        return buf


# Workspaces of calls that bring none: one buffer for each stream that a thread
# uses, since calls of two streams, or of two threads on one stream, may overlap
# between their launches.  A buffer is allocated on its own stream, so that the
# memory of one that is replaced or dropped is reused behind the calls that
# still read it.
_scratch_buffers = threading.local()
_MAX_SCRATCH_STREAMS = 16


def _capturing() -> bool:
    return _torch()._C._cuda_isCurrentStreamCapturing()


def _scratch(nbytes: int, device, stream: int):
    try:
        bufs = _scratch_buffers.by_stream
    except AttributeError:
        bufs = _scratch_buffers.by_stream = {}
    # captured: the graph's own memory, not a buffer that may be replaced before
    # a replay (the default stream, handle 0, cannot be captured)
    if stream and _capturing():
        return _torch().empty(max(nbytes, 256), dtype=_torch().uint8, device=device)
    key = (device.index, stream)
    buf = bufs.get(key)
    if buf is None or buf.numel() < nbytes:
        bufs.pop(key, None)
        while len(bufs) >= _MAX_SCRATCH_STREAMS:
            del bufs[next(iter(bufs))]
        buf = bufs[key] = _torch().empty(max(nbytes, 256), dtype=_torch().uint8, device=device)
    return buf


def hifa4_attention_fwd(q, k, v, s=None, cu_seqlens=None, max_seqlen=None, norm: int = NORM_PREORDER,
                        operands: int = OPERANDS_HIF4, smooth_qk: Optional[bool] = None, debug_p: bool = False,
                        out=None, lse=None, workspace: Optional[Workspace] = None, timing_events=None,
                        q_mean: bool = False, debug_heads=None, debug_tokens=None):
    """HiFA4 causal prefill forward.  Returns (o, lse) or, with debug_p,
    (o, lse, p_codes uint8 [NH,NT,NB,32], p_meta int32 [NH,NT,NB]) for the
    dump window debug_heads = (h0, NH) and debug_tokens = (t0, NT) (default:
    every head and token).  timing_events: optional three recorded
    torch.cuda.Event objects (before the pre-pass, before the attention
    kernel, after it).  q_mean: the Q-Mean auxiliary (HIF4 operands only)."""
    torch = _torch()
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.float16, n)
    _require(s, torch.float32, "s")
    sh = shape_of(q, k, cu_seqlens, max_seqlen)
    lib = load_library()
    dev = q.device
    if smooth_qk is None:
        smooth_qk = s is not None
    o = torch.empty_like(q) if out is None else out
    l = torch.empty((sh.heads_q, sh.tokens), dtype=torch.float32, device=dev) if lse is None else lse
    pc = pm = None
    h0, nh = debug_heads if debug_heads is not None else (0, 0)
    t0, nt = debug_tokens if debug_tokens is not None else (0, 0)
    if debug_p:
        nb = (sh.max_seqlen + 63) // 64
        pc = torch.zeros((nh or sh.heads_q, nt or sh.tokens, nb, 32), dtype=torch.uint8, device=dev)
        pm = torch.zeros((nh or sh.heads_q, nt or sh.tokens, nb), dtype=torch.int32, device=dev)
    ev_arr = None
    if timing_events is not None:
        ev_arr = (ctypes.c_void_p * 3)(*[e.cuda_event for e in timing_events])
    opt = FwdOptions(norm, operands, 1 if smooth_qk else 0, _ptr(pc), _ptr(pm),
                     ctypes.cast(ev_arr, ctypes.c_void_p) if ev_arr is not None else None, 1 if q_mean else 0,
                     0, h0, nh, t0, nt)
    p = sh.problem()
    need = int(lib.hifa4_workspace_bytes(ctypes.byref(p), ctypes.byref(opt)))
    stream = _stream(dev)
    ws = _scratch(need, dev, stream) if workspace is None else workspace.get(need, dev)
    _check(lib.hifa4_attention_fwd(ctypes.byref(p), ctypes.byref(opt), _ptr(q), _ptr(k), _ptr(v), _ptr(s),
                                   _ptr(o), _ptr(l), _ptr(ws), ws.numel(), stream), "hifa4_attention_fwd")
    if debug_p:
        return o, l, pc, pm
    return o, l


def hifa4_attention_fwd_noalloc(q, k, v, s=None, cu_seqlens=None, max_seqlen=None, norm: int = NORM_PREORDER,
                                operands: int = OPERANDS_HIF4, smooth_qk: Optional[bool] = None, out=None,
                                lse=None):
    """hifa4_attention_fwd with the library's static per-GPU scratch array as
    its workspace (no device allocation inside the call; at most
    NOALLOC_SCRATCH_BYTES of workspace).  Outputs are allocated here unless
    `out` and `lse` are given."""
    torch = _torch()
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.float16, n)
    _require(s, torch.float32, "s")
    sh = shape_of(q, k, cu_seqlens, max_seqlen)
    lib = load_library()
    dev = q.device
    if smooth_qk is None:
        smooth_qk = s is not None
    o = torch.empty_like(q) if out is None else out
    l = torch.empty((sh.heads_q, sh.tokens), dtype=torch.float32, device=dev) if lse is None else lse
    opt = FwdOptions(norm, operands, 1 if smooth_qk else 0, None, None, None, 0)
    p = sh.problem()
    _check(lib.hifa4_attention_fwd_noalloc(ctypes.byref(p), ctypes.byref(opt), _ptr(q), _ptr(k), _ptr(v), _ptr(s),
                                           _ptr(o), _ptr(l), _stream(dev)), "hifa4_attention_fwd_noalloc")
    return o, l


def decode_shape(q, k_codes, cu_seqlens=None, max_seqlen=None) -> Shape:
    """Problem shape of a decode step: q [B, Hq, D], K^ cache codes
    [T, Hkv, D/64, 32] (T = B * max_seqlen without cu_seqlens)."""
    if q.dim() != 3 or k_codes.dim() != 4:
        raise ValueError("decode takes q [batch, heads, dim] and k_codes [tokens, heads_kv, dim/64, 32]")
    b, hq, d = q.shape
    t, hkv = k_codes.shape[0], k_codes.shape[1]
    if cu_seqlens is None:
        if t % b:
            raise ValueError("without cu_seqlens the cache holds batch * max_seqlen tokens")
        return Shape(b, hq, hkv, d, t // b, t)
    if max_seqlen is None:
        raise ValueError("max_seqlen is required with cu_seqlens")
    _require(cu_seqlens, _torch().int32, "cu_seqlens")
    if cu_seqlens.numel() != b + 1:
        raise ValueError("cu_seqlens must hold batch + 1 entries")
    return Shape(b, hq, hkv, d, int(max_seqlen), t, cu_seqlens)


def hifa4_decode_workspace_bytes(shape: Shape) -> int:
    p = shape.problem()
    return int(load_library().hifa4_decode_workspace_bytes(ctypes.byref(p)))


def hifa4_decode_fwd(q, k_codes, k_meta, v_codes, v_meta, s=None, cu_seqlens=None, max_seqlen=None,
                     norm: int = NORM_PREORDER, smooth_qk: Optional[bool] = None, debug_p: bool = False,
                     out=None, lse=None, workspace: Optional[Workspace] = None, timing_events=None,
                     test_no_publish: int = 0):
    """One decode step over a packed HIF4 cache: q [B, Hq, D] fp16 is the query
    of each sequence's newest token; the cache is the output of
    hifa4_quantize_qk (K^, same s) and hifa4_quantize_v (V^) over the cached
    sequences.  Returns (o [B, Hq, D], lse [Hq, B]) or, with debug_p,
    (o, lse, p_codes uint8 [Hq, B, NB, 32], p_meta int32 [Hq, B, NB])."""
    torch = _torch()
    _require(q, torch.float16, "q")
    _require(k_codes, torch.uint8, "k_codes")
    _require(k_meta, torch.int32, "k_meta")
    _require(v_codes, torch.uint8, "v_codes")
    _require(v_meta, torch.int32, "v_meta")
    _require(s, torch.float32, "s")
    sh = decode_shape(q, k_codes, cu_seqlens, max_seqlen)
    nb = (sh.max_seqlen + 63) // 64
    g = sh.head_dim // 64
    if tuple(k_meta.shape) != (sh.tokens, sh.heads_kv, g) or tuple(k_codes.shape[2:]) != (g, 32):
        raise ValueError("k_codes/k_meta do not match [tokens, heads_kv, dim/64(, 32)]")
    if tuple(v_codes.shape) != (sh.batch, nb, sh.heads_kv, sh.head_dim, 32) or \
            tuple(v_meta.shape) != (sh.batch, nb, sh.heads_kv, sh.head_dim):
        raise ValueError("v_codes/v_meta do not match [batch, NB, heads_kv, dim(, 32)]")
    lib = load_library()
    dev = q.device
    if smooth_qk is None:
        smooth_qk = s is not None
    o = torch.empty_like(q) if out is None else out
    l = torch.empty((sh.heads_q, sh.batch), dtype=torch.float32, device=dev) if lse is None else lse
    pc = pm = None
    if debug_p:
        pc = torch.zeros((sh.heads_q, sh.batch, nb, 32), dtype=torch.uint8, device=dev)
        pm = torch.zeros((sh.heads_q, sh.batch, nb), dtype=torch.int32, device=dev)
    ev_arr = None
    if timing_events is not None:
        ev_arr = (ctypes.c_void_p * 3)(*[e.cuda_event for e in timing_events])
    opt = FwdOptions(norm, OPERANDS_HIF4, 1 if smooth_qk else 0, _ptr(pc), _ptr(pm),
                     ctypes.cast(ev_arr, ctypes.c_void_p) if ev_arr is not None else None, 0,
                     int(test_no_publish))
    p = sh.problem()
    need = int(lib.hifa4_decode_workspace_bytes(ctypes.byref(p)))
    stream = _stream(dev)
    ws = _scratch(need, dev, stream) if workspace is None else workspace.get(need, dev)
    _check(lib.hifa4_decode_fwd(ctypes.byref(p), ctypes.byref(opt), _ptr(q), _ptr(k_codes), _ptr(k_meta),
                                _ptr(v_codes), _ptr(v_meta), _ptr(s), _ptr(o), _ptr(l), _ptr(ws), ws.numel(),
                                stream), "hifa4_decode_fwd")
    if debug_p:
        return o, l, pc, pm
    return o, l


# ---------------------------------------------------------------------------
# The paged cache.
def _shaped(t, dtype, shape, device, name):
    if t.is_cuda and t.dtype is dtype and t.shape == shape and t.get_device() == device.index and t.is_contiguous():
        return
    _require(t, dtype, name)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")


def _row(t, dtype, n, device, name):
    """_shaped for one dimension of n."""
    if t.numel() == n and t.dtype is dtype and t.dim() == 1 and t.get_device() == device.index and t.is_contiguous():
        return
    _shaped(t, dtype, (n,), device, name)


def _count(x, name):
    """`x` where a 32-bit count goes (ctypes would cut a larger one without a word)."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must fit 32 bits, got {x}")
    return x


def _paged_call(name, device, *args):
    """Calls an entry point of the library with `device` current."""
    fn = getattr(_lib or load_library(), name)
    cuda = _torch_module._C
    back = cuda._cuda_getDevice()
    if back == device.index:
        status = fn(*args)
    else:
        cuda._cuda_setDevice(device.index)
        try:
            status = fn(*args)
        finally:
            cuda._cuda_setDevice(back)
    if status != 0:
        _check(status, name)


def hifa4_paged_page_bytes(heads_kv: int, head_dim: int, operands: int = OPERANDS_HIF4) -> int:
    """Bytes of a page: 64 tokens of K and V, every kv head."""
    n = int(load_library().hifa4_paged_page_bytes(_count(heads_kv, "heads_kv"), _count(head_dim, "head_dim"),
                                                  _count(operands, "operands")))
    if not n:
        raise Hifa4Error(f"hifa4_paged_page_bytes: {hifa4_last_error()}")
    return n


class PagedCache:
    """The handle of a paged K/V cache: pages of 64 tokens in one pool.

    pool         uint8 [num_pages, heads_kv, bytes] (bytes * heads_kv =
                 hifa4_paged_page_bytes; the contents are the library's)
    block_table  int32 [batch, max_pages], the page of each 64 tokens (an entry
                 that is no page of the pool, such as -1, holds no tokens)
    seq_lens     int32 [batch], cached tokens; 0 for an unused row
    v_tail       fp16 [batch, 64, heads_kv, head_dim], V of each sequence's
                 last page (hifa4_paged_append on HIF4 pages needs it)

    The tensors stay the caller's: tables and lengths are changed in place,
    also between replays of a captured call.  Before an append a length may be
    cut back within the page that the last append ended in, or to a multiple of
    64 (FP16 pages: anywhere; on HIF4 pages v_tail no longer holds V of an
    earlier page's tokens).  PagedCache.empty allocates them."""

    def __init__(self, pool, block_table, seq_lens, head_dim: int, operands: int = OPERANDS_HIF4, v_tail=None):
        torch = _torch()
        _require(pool, torch.uint8, "pool")
        if pool.dim() != 3:
            raise ValueError("pool is [num_pages, heads_kv, bytes]")
        heads_kv, dev = pool.shape[1], pool.device
        if hifa4_paged_page_bytes(heads_kv, head_dim, operands) != heads_kv * pool.shape[2]:
            raise ValueError(f"a page of {heads_kv} heads holds {hifa4_paged_page_bytes(heads_kv, head_dim, operands)} "
                             f"bytes, the pool has {heads_kv * pool.shape[2]}")
        if block_table.dim() != 2:
            raise ValueError("block_table is [batch, max_pages]")
        batch, max_pages = block_table.shape
        _shaped(block_table, torch.int32, (batch, max_pages), dev, "block_table")
        _shaped(seq_lens, torch.int32, (batch,), dev, "seq_lens")
        if v_tail is not None:
            _shaped(v_tail, torch.float16, (batch, PAGE_TOKENS, heads_kv, head_dim), dev, "v_tail")
        self._tensors = (pool, block_table, seq_lens, v_tail)
        self.device, self.batch, self.heads_kv, self.head_dim = dev, batch, heads_kv, head_dim
        self.operands, self.max_pages = operands, max_pages
        self._desc = PagedCacheDesc(batch, heads_kv, head_dim, operands, pool.shape[0], max_pages, _ptr(pool),
                                    _ptr(block_table), _ptr(seq_lens), _ptr(v_tail))
        self._ref = ctypes.byref(self._desc)
        self._workspace_bytes = {}

    pool = property(lambda self: self._tensors[0])
    block_table = property(lambda self: self._tensors[1])
    seq_lens = property(lambda self: self._tensors[2])
    v_tail = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, num_pages: int, batch: int, max_pages: int, heads_kv: int, head_dim: int,
              operands: int = OPERANDS_HIF4, device="cuda"):
        """A cache whose rows are all empty (no pages, length 0)."""
        torch = _torch()
        record = hifa4_paged_page_bytes(heads_kv, head_dim, operands) // heads_kv
        pool = torch.empty((num_pages, heads_kv, record), dtype=torch.uint8, device=device)
        table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=device)
        lens = torch.zeros(batch, dtype=torch.int32, device=device)
        tail = None
        if operands == OPERANDS_HIF4:
            tail = torch.zeros((batch, PAGE_TOKENS, heads_kv, head_dim), dtype=torch.float16, device=device)
        return cls(pool, table, lens, head_dim, operands, tail)


def hifa4_paged_append(cache: PagedCache, k, v, s=None, cu_new=None, max_new: Optional[int] = None):
    """Appends new tokens: k, v fp16 [total, heads_kv, head_dim]; without
    cu_new one token per row of the batch, else sequence b gets the rows
    [cu_new[b], cu_new[b+1]).  cache.seq_lens counts the new tokens already.
    s: the Smooth-QK scales (the pages then hold k/s).  max_new: an upper bound
    of the tokens per sequence (default: all of them; it sizes the launch for
    every row, so large batches give it)."""
    torch, dev = _torch(), cache.device
    if k.dim() != 3:
        raise ValueError("k is [total, heads_kv, head_dim]")
    total = _count(k.shape[0], "the rows of k")
    _shaped(k, torch.float16, (total, cache.heads_kv, cache.head_dim), dev, "k")
    _shaped(v, torch.float16, (total, cache.heads_kv, cache.head_dim), dev, "v")
    if s is not None:
        _shaped(s, torch.float32, (cache.heads_kv, cache.head_dim), dev, "s")
    if cu_new is not None:
        _shaped(cu_new, torch.int32, (cache.batch + 1,), dev, "cu_new")
    if max_new is None:
        max_new = total if cu_new is not None else 1
    _paged_call("hifa4_paged_append", dev, cache._ref, total, _count(max_new, "max_new"), _ptr(cu_new), k.data_ptr(), v.data_ptr(), _ptr(s),
                _stream(dev))


def hifa4_paged_gather(cache: PagedCache, cu_tokens, total_tokens: int, max_tokens: Optional[int] = None, starts=None,
                       k=None, v=None):
    """Reads tokens back: of sequence b the tokens from starts[b] (default 0)
    on into the rows [cu_tokens[b], cu_tokens[b+1]).  Returns (k, v) fp16
    [total_tokens, heads_kv, head_dim] (allocated unless given), K as it is
    cached.  max_tokens: an upper bound of the rows per sequence (default: all
    of them)."""
    torch, dev = _torch(), cache.device
    shape = (_count(total_tokens, "total_tokens"), cache.heads_kv, cache.head_dim)
    max_tokens = total_tokens if max_tokens is None else _count(max_tokens, "max_tokens")
    _shaped(cu_tokens, torch.int32, (cache.batch + 1,), dev, "cu_tokens")
    if starts is not None:
        _shaped(starts, torch.int32, (cache.batch,), dev, "starts")
    if k is None:
        k = torch.empty(shape, dtype=torch.float16, device=dev)
    else:
        _shaped(k, torch.float16, shape, dev, "k")
    if v is None:
        v = torch.empty_like(k)
    else:
        _shaped(v, torch.float16, shape, dev, "v")
    _paged_call("hifa4_paged_gather", dev, cache._ref, total_tokens, max_tokens, cu_tokens.data_ptr(),
                _ptr(starts), k.data_ptr(), v.data_ptr(), _stream(dev))
    return k, v


def hifa4_paged_decode_workspace_bytes(cache: PagedCache, heads_q: int, page_weights: bool = False) -> int:
    n = int(load_library().hifa4_paged_decode_workspace_bytes(cache._ref, _count(heads_q, "heads_q"),
                                                              1 if page_weights else 0))
    if not n:
        raise Hifa4Error(f"hifa4_paged_decode_workspace_bytes: {hifa4_last_error()}")
    return n


def hifa4_paged_decode_fwd(cache: PagedCache, q, s=None, page_weights=None, decay: float = 1.0, weights_out=None,
                           out=None, lse=None, workspace: Optional[Workspace] = None):
    """One decode step over the pages: q [batch, heads_q, head_dim] fp16, the
    query of each sequence's newest token.  Returns (o like q, lse fp32
    [heads_q, batch]); empty rows get 0 and -inf.  page_weights fp32 [batch,
    max_pages]: becomes decay * page_weights + this step's attention weight of
    each page (in place, or in weights_out)."""
    torch, dev = _torch(), cache.device
    if q.dim() != 3:
        raise ValueError("q is [batch, heads_q, head_dim]")
    hq = q.shape[1]
    _shaped(q, torch.float16, (cache.batch, hq, cache.head_dim), dev, "q")
    if s is not None:
        _shaped(s, torch.float32, (cache.heads_kv, cache.head_dim), dev, "s")
    weighs = page_weights is not None
    if weighs:
        _shaped(page_weights, torch.float32, (cache.batch, cache.max_pages), dev, "page_weights")
        if weights_out is None:
            weights_out = page_weights
        else:
            _shaped(weights_out, torch.float32, (cache.batch, cache.max_pages), dev, "weights_out")
    elif weights_out is not None:
        raise ValueError("weights_out needs page_weights")
    if out is None:
        out = torch.empty_like(q)
    else:
        _shaped(out, torch.float16, q.shape, dev, "out")
    if lse is None:
        lse = torch.empty((hq, cache.batch), dtype=torch.float32, device=dev)
    else:
        _shaped(lse, torch.float32, (hq, cache.batch), dev, "lse")
    need = cache._workspace_bytes.get((hq, weighs))
    if need is None:
        need = cache._workspace_bytes[hq, weighs] = hifa4_paged_decode_workspace_bytes(cache, hq, weighs)
    stream = _stream(dev)
    ws = _scratch(need, dev, stream) if workspace is None else workspace.get(need, dev)
    _paged_call("hifa4_paged_decode_fwd", dev, cache._ref, hq, q.data_ptr(), _ptr(s), out.data_ptr(), lse.data_ptr(),
                _ptr(page_weights), _ptr(weights_out), decay, ws.data_ptr(), ws.numel(), stream)
    return out, lse


def hifa4_paged_evict(block_table, seq_lens, page_weights, budget: int, first: int = 0, last: int = 1, out_table=None,
                      out_lens=None, out_weights=None, freed=None, num_freed=None):
    """Evicts the pages of the least weight from every sequence that holds more
    than `budget`; its `first` first and `last` last pages stay.  Works in place
    unless out_table, out_lens, out_weights are given.  Returns (freed int32
    [batch, max_pages]: the evicted pages in order, then -1; num_freed int32
    [batch])."""
    torch, dev = _torch(), block_table.device
    if block_table.dim() != 2:
        raise ValueError("block_table is [batch, max_pages]")
    for x, name in ((budget, "budget"), (first, "first"), (last, "last")):
        _count(x, name)
    i32, f32 = torch.int32, torch.float32
    shape = block_table.shape
    rows = shape[:1]
    _shaped(block_table, i32, shape, dev, "block_table")
    _shaped(seq_lens, i32, rows, dev, "seq_lens")
    _shaped(page_weights, f32, shape, dev, "page_weights")
    if out_table is None:
        out_table = block_table
    else:
        _shaped(out_table, i32, shape, dev, "out_table")
    if out_lens is None:
        out_lens = seq_lens
    else:
        _shaped(out_lens, i32, rows, dev, "out_lens")
    if out_weights is None:
        out_weights = page_weights
    else:
        _shaped(out_weights, f32, shape, dev, "out_weights")
    if freed is None:
        freed = torch.empty(shape, dtype=i32, device=dev)
    else:
        _shaped(freed, i32, shape, dev, "freed")
    if num_freed is None:
        num_freed = torch.empty(rows, dtype=i32, device=dev)
    else:
        _shaped(num_freed, i32, rows, dev, "num_freed")
    _paged_call("hifa4_paged_evict", dev, shape[0], shape[1], block_table.data_ptr(), seq_lens.data_ptr(),
                page_weights.data_ptr(), budget, first, last, out_table.data_ptr(), out_lens.data_ptr(),
                out_weights.data_ptr(), freed.data_ptr(), num_freed.data_ptr(), _stream(dev))
    return freed, num_freed


def hifa4_paged_chunk_workspace_bytes(cache: PagedCache, heads_q: int, total_new: int, max_new: int) -> int:
    n = int(load_library().hifa4_paged_chunk_workspace_bytes(cache._ref, _count(heads_q, "heads_q"),
                                                             _count(total_new, "total_new"), _count(max_new, "max_new")))
    if not n:
        raise Hifa4Error(f"hifa4_paged_chunk_workspace_bytes: {hifa4_last_error()}")
    return n


def hifa4_paged_chunk_fwd(cache: PagedCache, q, cu_new, s=None, max_new: Optional[int] = None, out=None, lse=None,
                          workspace: Optional[Workspace] = None):
    """The attention of each sequence's last tokens over the pages: q [total,
    heads_q, head_dim] fp16, of sequence b the rows [cu_new[b], cu_new[b+1]), whose
    tokens are the last ones of its cached tokens (appended before); a token sees
    the cached ones up to its own.  max_new: an upper bound of the tokens per
    sequence (default: all of them; it sizes the launch, so batches give it).
    Returns (o like q, lse fp32 [heads_q, total]); rows that see nothing get 0 and
    -inf, rows that no sequence has are left as they are (uninitialized where out
    and lse are not given)."""
    torch, dev = _torch(), cache.device
    if q.dim() != 3:
        raise ValueError("q is [total, heads_q, head_dim]")
    total, hq = _count(q.shape[0], "the rows of q"), q.shape[1]
    _shaped(q, torch.float16, (total, hq, cache.head_dim), dev, "q")
    _shaped(cu_new, torch.int32, (cache.batch + 1,), dev, "cu_new")
    if s is not None:
        _shaped(s, torch.float32, (cache.heads_kv, cache.head_dim), dev, "s")
    if out is None:
        out = torch.empty_like(q)
    else:
        _shaped(out, torch.float16, q.shape, dev, "out")
    if lse is None:
        lse = torch.empty((hq, total), dtype=torch.float32, device=dev)
    else:
        _shaped(lse, torch.float32, (hq, total), dev, "lse")
    max_new = total if max_new is None else _count(max_new, "max_new")
    key = (hq, total, max_new)
    need = cache._workspace_bytes.get(key)
    if need is None:
        if len(cache._workspace_bytes) >= 4096:
            cache._workspace_bytes.clear()
        need = cache._workspace_bytes[key] = hifa4_paged_chunk_workspace_bytes(cache, hq, total, max_new)
    stream = _stream(dev)
    ws = _scratch(need, dev, stream) if workspace is None else workspace.get(need, dev)
    _paged_call("hifa4_paged_chunk_fwd", dev, cache._ref, hq, total, max_new, cu_new.data_ptr(), q.data_ptr(), _ptr(s),
                out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    return out, lse


def hifa4_paged_extend(block_table, seq_lens, counts, free_pages, num_free, max_total: int, max_new: Optional[int] = None,
                       shift=None, out_lens=None, out_free=None, cu_new=None, positions=None, slots=None):
    """Deals out the pages of counts[b] new tokens for each row of block_table
    [batch, max_pages] from the stack free_pages (int32, num_free[0] of them free,
    the last on top).  Rows are served in order; one whose tokens would go beyond
    max_total, or its pages beyond the free ones, gets none.  Works in place on
    block_table and, unless out_lens and out_free are given, on seq_lens and
    num_free.  Returns (cu_new int32 [batch+1], positions int32 [max_total], slots
    int64 [max_total]): the prefix sums of the tokens that the rows got, and of each
    its position (plus shift[b], the tokens that evictions took out) and its slot
    (64 * page + place); -1 behind the last one.  max_new: an upper bound of the
    tokens per row (default: max_total)."""
    torch, dev = _torch(), block_table.device
    if block_table.dim() != 2:
        raise ValueError("block_table is [batch, max_pages]")
    if free_pages.dim() != 1:
        raise ValueError("free_pages is [capacity]")
    i32 = torch.int32
    batch, max_pages = shape = block_table.shape
    capacity = _count(free_pages.shape[0], "the free pages")
    if _count(max_total, "max_total") < 0:
        raise ValueError("max_total must be >= 0")
    max_new = max_total if max_new is None else _count(max_new, "max_new")
    _shaped(block_table, i32, shape, dev, "block_table")
    _row(seq_lens, i32, batch, dev, "seq_lens")
    _row(counts, i32, batch, dev, "counts")
    _row(free_pages, i32, capacity, dev, "free_pages")
    _row(num_free, i32, 1, dev, "num_free")
    if shift is not None:
        _row(shift, i32, batch, dev, "shift")
    if out_lens is None:
        out_lens = seq_lens
    else:
        _row(out_lens, i32, batch, dev, "out_lens")
    if out_free is None:
        out_free = num_free
    else:
        _row(out_free, i32, 1, dev, "out_free")
    if cu_new is None:
        cu_new = torch.empty(batch + 1, dtype=i32, device=dev)
    else:
        _row(cu_new, i32, batch + 1, dev, "cu_new")
    if positions is None:
        positions = torch.empty(max_total, dtype=i32, device=dev)
    else:
        _row(positions, i32, max_total, dev, "positions")
    if slots is None:
        slots = torch.empty(max_total, dtype=torch.int64, device=dev)
    else:
        _row(slots, torch.int64, max_total, dev, "slots")
    _paged_call("hifa4_paged_extend", dev, batch, max_pages, block_table.data_ptr(), seq_lens.data_ptr(), counts.data_ptr(),
                free_pages.data_ptr(), capacity, num_free.data_ptr(), None if shift is None else shift.data_ptr(), max_total, max_new,
                out_lens.data_ptr(), out_free.data_ptr(), cu_new.data_ptr(), positions.data_ptr(), slots.data_ptr(), _stream(dev))
    return cu_new, positions, slots


def hifa4_paged_release(table, to, free_pages, num_free, first=None, out_free=None, workspace: Optional[Workspace] = None):
    """Puts the entries at the places [first[b], to[b]) (first: default 0) of each
    row of table [batch, max_pages] back on the stack free_pages, the first row's
    first entry on top; negative entries are no pages.  num_free counts them
    afterwards, unless out_free is given.  Returns out_free.  For the pages that
    hifa4_paged_evict took out: hifa4_paged_release(freed, num_freed, ...)."""
    torch, dev = _torch(), table.device
    if table.dim() != 2:
        raise ValueError("table is [batch, max_pages]")
    if free_pages.dim() != 1:
        raise ValueError("free_pages is [capacity]")
    i32 = torch.int32
    batch, max_pages = shape = table.shape
    capacity = _count(free_pages.shape[0], "the free pages")
    _shaped(table, i32, shape, dev, "table")
    _row(to, i32, batch, dev, "to")
    if first is not None:
        _row(first, i32, batch, dev, "first")
    _row(free_pages, i32, capacity, dev, "free_pages")
    _row(num_free, i32, 1, dev, "num_free")
    if out_free is None:
        out_free = num_free
    else:
        _row(out_free, i32, 1, dev, "out_free")
    need = 4 * (batch + 1)
    stream = _stream(dev)
    ws = _scratch(need, dev, stream) if workspace is None else workspace.get(need, dev)
    _paged_call("hifa4_paged_release", dev, batch, max_pages, table.data_ptr(), None if first is None else first.data_ptr(), to.data_ptr(),
                free_pages.data_ptr(), capacity, num_free.data_ptr(), out_free.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    return out_free


# ---------------------------------------------------------------------------
# Rotary positions.
ROPE_SCALINGS = ("none", "linear", "ntk", "parts")


class Rope:
    """Frequencies of the rotary positions of heads of head_dim channels, of which
    the first rot_dim (default: all; a multiple of 8) are rotated.

    base         w_i = base^(-2i/rot_dim) is the angle of pair i per position
    interleaved  pairs are neighbouring channels (else i and i + rot_dim/2)
    scaling      of the frequencies, for contexts longer than the trained one:
                 "none"; "linear": w / factor; "ntk": base * factor^(r/(r-2));
                 "parts": w (g + (1-g)/factor), where g goes from 0 to 1 as the
                 turns over original_len positions go from low to high
    magnitude    factor of the rotated values"""

    def __init__(self, head_dim: int, rot_dim: Optional[int] = None, base: float = 10000.0, interleaved: bool = False,
                 scaling: str = "none", factor: float = 1.0, original_len: float = 0.0, low: float = 1.0, high: float = 32.0,
                 magnitude: float = 1.0, device="cuda"):
        torch = _torch()
        if scaling not in ROPE_SCALINGS:
            raise ValueError(f"scaling must be one of {ROPE_SCALINGS}, got {scaling!r}")
        if head_dim not in (64, 128, 256):
            raise ValueError(f"head_dim must be 64, 128 or 256, got {head_dim}")
        rot_dim = head_dim if rot_dim is None else rot_dim
        if rot_dim <= 0 or rot_dim > head_dim or rot_dim % 8:
            raise ValueError(f"rot_dim must be a multiple of 8 between 8 and head_dim, got {rot_dim}")
        turns = (ctypes.c_uint64 * (rot_dim // 2))()
        _check(load_library().hifa4_rope_frequencies(rot_dim, base, ROPE_SCALINGS.index(scaling), factor, original_len, low, high,
                                                     turns), "hifa4_rope_frequencies")
        # uint64 bit patterns in an int64 tensor
        signed = [t - 2 ** 64 if t >= 2 ** 63 else t for t in turns]
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self.device = self.turns.device
        self.head_dim, self.rot_dim, self.interleaved, self.magnitude = head_dim, rot_dim, bool(interleaved), float(magnitude)
        self._interleaved, self._turns = int(self.interleaved), self.turns.data_ptr()


def _rope_rows(t, tokens, head_dim, device, name):
    """(heads, pointer, elements from token to token) of [tokens, heads, head_dim], each token's heads contiguous."""
    torch = _torch()
    if t is None:
        return 0, None, 0
    if t.dim() == 3 and t.dtype is torch.float16 and t.get_device() == device.index:
        rows, heads, d = t.shape
        if rows == tokens and d == head_dim:
            a, b, c = t.stride()
            if tokens <= 1:
                a = heads * d               # (there is no next token: the tensor's own stride says nothing)
            if c == 1 and (b == d or heads <= 1) or not tokens:
                return _count(heads, "heads"), t.data_ptr(), a
            raise ValueError(f"{name}: a token's heads must be contiguous")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype is not torch.float16:
        raise ValueError(f"{name} must be {torch.float16}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    raise ValueError(f"{name} must be [{tokens}, heads, {head_dim}], got {list(t.shape)}")


def _rope_out(x, y, heads, tokens, head_dim, device, name):
    """The output for x (y, or a new tensor): (it, pointer, elements from token to token)."""
    if x is None:
        if y is not None:
            raise ValueError(f"{name}_out needs a {name} of its shape")
        return None, None, 0
    if y is None:
        y = _torch().empty((tokens, heads, head_dim), dtype=x.dtype, device=device)
        return y, y.data_ptr(), heads * head_dim
    if y.shape != x.shape:
        raise ValueError(f"{name}_out needs a {name} of its shape")
    _, at, stride = _rope_rows(y, tokens, head_dim, device, name + "_out")
    return y, at, stride


def hifa4_rope(rope: Rope, positions, q=None, k=None, q_out=None, k_out=None, transposed: bool = False):
    """Rotates q [tokens, heads_q, head_dim] and k [tokens, heads_k, head_dim] (fp16;
    either may be None; a token's heads are contiguous, tokens any multiple of 8
    elements apart, so parts of one projection's rows will do) by the positions
    int32 [tokens].  Rows of negative positions are no tokens: their outputs are
    left as they are.  Returns (q_out, k_out), allocated unless given; q_out=q and
    k_out=k work in place.  transposed: the transposed rotation, the gradient of q
    and k from that of q_out and k_out (the inverse, where the magnitude is 1)."""
    torch, dev = _torch(), rope.device
    if positions.dim() != 1:
        raise ValueError("positions is [tokens]")
    tokens = _count(positions.shape[0], "the tokens")
    _row(positions, torch.int32, tokens, dev, "positions")
    d = rope.head_dim
    hq, qp, qs = _rope_rows(q, tokens, d, dev, "q")
    hk, kp, ks = _rope_rows(k, tokens, d, dev, "k")
    q_out, qo, qos = _rope_out(q, q_out, hq, tokens, d, dev, "q")
    k_out, ko, kos = _rope_out(k, k_out, hk, tokens, d, dev, "k")
    _paged_call("hifa4_rope", dev, d, rope.rot_dim, rope._interleaved, 1 if transposed else 0, rope.magnitude, rope._turns, tokens,
                positions.data_ptr(), hq, qp, qs, qo, qos, hk, kp, ks, ko, kos, _stream(dev))
    return q_out, k_out


def hifa4_selftest_exp2(x):
    """y = fp16(2^x) through the kernels' exponential routine (x fp16 on GPU)."""
    torch = _torch()
    _require(x, torch.float16, "x")
    y = torch.empty_like(x)
    _check(load_library().hifa4_selftest_exp2(_ptr(x), _ptr(y), x.numel(), _stream(x.device)), "hifa4_selftest_exp2")
    return y
