"""Python binding of libviscache (include/viscache.h, include/viscache_step.h): argument marshalling only.

Every function here has the name of the C entry point it calls.  torch is used
for device memory (outputs and workspaces) and for the current CUDA stream;
every step of the compression pass runs in the library's kernels.  There is no
fallback: if ``_lib/libviscache.so`` is missing or fails to load, importing
the functions raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import List, Optional, Sequence, Tuple

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lib", "libviscache.so")

VC_OK = 0
VC_ERR_INVALID_ARG = 1
VC_ERR_INFEASIBLE = 2
VC_ERR_WORKSPACE = 3
VC_ERR_CUDA = 4
VC_ERR_DEVICE_TIMEOUT = 5
VC_ERR_UNSUPPORTED = 6
VC_ERR_DEVICE_INDEX = 7
VC_BF16, VC_F32 = 0, 1
VC_RANK_SHARED, VC_RANK_PER_LAYER = 0, 1
VC_SCHED_PARABOLA, VC_SCHED_FIXED, VC_SCHED_ARITHMETIC, VC_SCHED_GEOMETRIC = 0, 1, 2, 3
VC_DROP_SURVIVORS, VC_DROP_ALL = 0, 1
VC_PATH_AUTO, VC_PATH_SIMT = 0, 1
VC_ROPE_SECTIONED, VC_ROPE_INTERLEAVED = 0, 1
VC_ROPE_HALVES, VC_ROPE_ADJACENT = 0, 1
VC_TEST_WAIT_SCORE_LSE, VC_TEST_WAIT_SCORE_COLSUM, VC_TEST_WAIT_FUSE = 1, 2, 4

_ERR_NAMES = {1: "VC_ERR_INVALID_ARG", 2: "VC_ERR_INFEASIBLE", 3: "VC_ERR_WORKSPACE",
              4: "VC_ERR_CUDA", 5: "VC_ERR_DEVICE_TIMEOUT", 6: "VC_ERR_UNSUPPORTED",
              7: "VC_ERR_DEVICE_INDEX"}

EXPORTED = ("viscache_plan_budgets", "viscache_plan_budgets_ex", "prunekv_score_workspace_size", "prunekv_score",
            "prunekv_select_workspace_size", "prunekv_select", "prunekv_fuse_workspace_size",
            "prunekv_fuse_compact", "prunekv_workspace_size", "prunekv_compress",
            "prunekv_get_status", "viscache_version", "viscache_profile_enable",
            "viscache_profile_read", "prunekv_score_static", "prunekv_score_static_capacity",
            "prunekv_score_static_status", "viscache_set_kernel_path", "viscache_set_dependent_launch",
            "viscache_test_inject_wait",
            "viscache_device_accessible", "viscache_scout_workspace_size", "viscache_scout_sizes", "viscache_scout_mmr",
            "viscache_decode_workspace_size", "viscache_decode_attention",
            "viscache_kv4_sizes", "viscache_kv4_quantize", "viscache_kv4_dequantize",
            "viscache_decode_attention_kv4", "viscache_mrope", "viscache_kv8_workspace_size",
            "viscache_kv8_append", "viscache_kv8_read", "viscache_kv8_attention")

# the entry points of include/viscache_step.h
EXPORTED_STEP = ("viscache_norm_mrope", "viscache_norm_mrope_grad_workspace_size", "viscache_norm_mrope_grad",
                 "viscache_kv8_weigh", "viscache_kv8_evict_workspace_size", "viscache_kv8_evict", "viscache_sample")


class VisCacheError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__("%s failed: %s (%d)" % (fn, _ERR_NAMES.get(code, "unknown"), code))
        self.code = code


class vc_batch(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int32), ("n_vis", ctypes.POINTER(ctypes.c_int32)),
                ("W", ctypes.POINTER(ctypes.c_int32)), ("rr_num", ctypes.POINTER(ctypes.c_uint32)),
                ("rr_den", ctypes.POINTER(ctypes.c_uint32))]


class vc_params(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("h", ctypes.c_int32),
                ("m_num", ctypes.c_uint32), ("m_den", ctypes.c_uint32), ("mu", ctypes.c_float),
                ("tau", ctypes.c_float), ("scale", ctypes.c_float), ("rank_mode", ctypes.c_int32),
                ("schedule", ctypes.c_int32), ("drop_mode", ctypes.c_int32)]


class vc_rope(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("sections", ctypes.c_int32 * 4), ("order", ctypes.c_int32),
                ("pairing", ctypes.c_int32), ("theta", ctypes.c_double)]


class vc_kv8(ctypes.Structure):
    _fields_ = [("K_codes", ctypes.c_void_p), ("V_codes", ctypes.c_void_p), ("K_scale", ctypes.c_void_p),
                ("V_scale", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("page", ctypes.c_int32), ("d", ctypes.c_int32)]


class vc_kv8_step(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("block_table", ctypes.c_void_p),
                ("seq_lens", ctypes.c_void_p), ("row_start", ctypes.c_void_p), ("n_rows", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library (loads on first use; raises if it was never built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("libviscache.so is not built (%s); run __graft_entry__.build()" % _LIB_PATH)
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, u32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_float, ctypes.c_size_t
        pi32 = ctypes.POINTER(ctypes.c_int32)
        L.viscache_plan_budgets.argtypes = [i32, i32, u32, u32, i32, u32, u32, pi32, pi32, pi32]
        L.viscache_plan_budgets_ex.argtypes = [i32, i32, u32, u32, i32, u32, u32, i32, i32, pi32, pi32,
                                               pi32]
        L.viscache_scout_workspace_size.argtypes = [i32, pi32, i32]
        L.viscache_scout_workspace_size.restype = sz
        L.viscache_scout_sizes.argtypes = [i32, pi32, u32, u32, pi32]
        L.viscache_scout_mmr.argtypes = [vp, vp, i32, pi32, i32, f32, u32, u32, vp, vp, vp, pi32, vp, sz, vp]
        L.viscache_kv4_sizes.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params),
                                         ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
        L.viscache_kv4_quantize.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params), vp, vp,
                                            vp, vp, vp, vp, vp]
        L.viscache_kv4_dequantize.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params), vp, vp,
                                              vp, vp, vp, vp, vp]
        L.viscache_decode_attention_kv4.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params), i32,
                                                    vp, vp, vp, vp, vp, vp, vp, pi32, vp, vp, sz, vp]
        L.viscache_decode_workspace_size.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params), pi32]
        L.viscache_decode_workspace_size.restype = sz
        L.viscache_decode_attention.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params), i32,
                                                vp, vp, vp, vp, vp, pi32, vp, vp, sz, vp]
        i64 = ctypes.c_int64
        L.viscache_mrope.argtypes = [ctypes.POINTER(vc_rope), vp, i32, i64, i32, i32, i32, vp, i64, vp, i64, i32,
                                     vp, i64, vp, i64, vp]
        L.viscache_kv8_workspace_size.argtypes = [i32, i32, i32, i32]
        L.viscache_kv8_workspace_size.restype = sz
        pc8, ps8 = ctypes.POINTER(vc_kv8), ctypes.POINTER(vc_kv8_step)
        L.viscache_kv8_append.argtypes = [pc8, ps8, i32, vp, i64, i64, vp, i64, i64, vp, sz, vp]
        L.viscache_kv8_read.argtypes = [pc8, ps8, i32, vp, vp, vp, sz, vp]
        L.viscache_kv8_attention.argtypes = [pc8, ps8, i32, i32, vp, i64, f32, i32, vp, vp, vp, sz, vp]
        pr = ctypes.POINTER(vc_rope)
        L.viscache_norm_mrope.argtypes = [pr, vp, i32, i64, i32, i32, i32, vp, i64, vp, i64, vp, vp, f32, vp, i64, vp,
                                          i64, vp]
        L.viscache_norm_mrope_grad_workspace_size.argtypes = [i64, i32, i32, i32]
        L.viscache_norm_mrope_grad_workspace_size.restype = sz
        L.viscache_norm_mrope_grad.argtypes = [pr, vp, i32, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp,
                                               vp, f32, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.viscache_kv8_weigh.argtypes = [pc8, ps8, i32, i32, vp, i64, vp, f32, i32, vp, vp, sz, vp]
        L.viscache_kv8_evict_workspace_size.argtypes = [i32, i32]
        L.viscache_kv8_evict_workspace_size.restype = sz
        L.viscache_kv8_evict.argtypes = [pc8, ps8, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.viscache_sample.argtypes = [i32, i64, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
        L.prunekv_score_workspace_size.argtypes = [i32, i32, i32]
        L.prunekv_score_workspace_size.restype = sz
        L.prunekv_score.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, i32, vp, vp,
                                    vp, sz, vp]
        L.prunekv_score_static.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, i32, vp,
                                           vp, vp]
        L.prunekv_score_static_capacity.argtypes = []
        L.prunekv_score_static_capacity.restype = sz
        L.prunekv_score_static_status.argtypes = [vp]
        L.prunekv_select_workspace_size.argtypes = [i32, i32, i32, i32]
        L.prunekv_select_workspace_size.restype = sz
        L.prunekv_select.argtypes = [vp, i32, i32, i32, pi32, i32, i32, vp, vp, vp, vp, sz, vp]
        L.prunekv_fuse_workspace_size.argtypes = [pi32, i32, i32, i32, i32, i32]
        L.prunekv_fuse_workspace_size.restype = sz
        L.prunekv_fuse_compact.argtypes = [vp, vp, i32, i32, i32, i32, i32, pi32, i32, vp, vp, f32,
                                           f32, vp, vp, vp, sz, vp]
        L.prunekv_workspace_size.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params)]
        L.prunekv_workspace_size.restype = sz
        L.prunekv_compress.argtypes = [ctypes.POINTER(vc_batch), ctypes.POINTER(vc_params), vp, vp,
                                       vp, vp, vp, vp, vp, sz, vp]
        L.prunekv_get_status.argtypes = [vp, vp]
        L.viscache_version.restype = ctypes.c_char_p
        L.viscache_profile_enable.argtypes = [i32]
        L.viscache_set_kernel_path.argtypes = [i32]
        L.viscache_set_dependent_launch.argtypes = [i32]
        L.viscache_test_inject_wait.argtypes = [i32]
        L.viscache_device_accessible.argtypes = [vp]
        L.viscache_profile_read.argtypes = [ctypes.c_char_p, i32, ctypes.POINTER(ctypes.c_float),
                                            pi32, i32]
        _lib = L
    return _lib


def _check(fn: str, rc: int) -> None:
    if rc != VC_OK:
        raise VisCacheError(fn, rc)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return VC_BF16
    if t.dtype == torch.float32:
        return VC_F32
    raise TypeError("unsupported dtype %s (bf16 or fp32)" % t.dtype)


def _on(stream):
    """Where a call allocates: its own stream.  A block of another stream's pool may still be in use
    there, and one that the call drops on return would be handed out again before its kernels ran."""
    if stream is None:
        return contextlib.nullcontext()
    if not hasattr(stream, "device"):           # a stream of another library: its handle is enough
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    return torch.cuda.stream(stream)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _on(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _workspace(nbytes: int, device, ws: Optional[torch.Tensor], stream) -> torch.Tensor:
    return ws if ws is not None else _empty(max(nbytes, 256), torch.uint8, device, stream)


def _i32(seq):
    arr = (ctypes.c_int32 * len(seq))(*[int(x) for x in seq])
    return arr


# ---------------------------------------------------------------------------

def viscache_version() -> str:
    return lib().viscache_version().decode()


def viscache_device_accessible(t: torch.Tensor) -> bool:
    """True if the current CUDA device can read the tensor's memory directly."""
    rc = lib().viscache_device_accessible(ctypes.c_void_p(t.data_ptr()))
    if rc < 0:
        raise VisCacheError("viscache_device_accessible", -rc)
    return rc == 1


def viscache_plan_budgets(L: int, n_vis: int, rr_num: int, rr_den: int, h: int = 0,
                          m_num: int = 3, m_den: int = 4) -> Tuple[List[int], int, int]:
    """Host planner (Eq. parabolic): returns (B[L], Nq, h)."""
    B = (ctypes.c_int32 * L)()
    nq, hh = ctypes.c_int32(), ctypes.c_int32()
    _check("viscache_plan_budgets",
           lib().viscache_plan_budgets(L, n_vis, rr_num, rr_den, h, m_num, m_den, B,
                                       ctypes.byref(nq), ctypes.byref(hh)))
    return list(B), nq.value, hh.value


def viscache_plan_budgets_ex(L: int, n_vis: int, rr_num: int, rr_den: int, h: int = 0,
                             m_num: int = 3, m_den: int = 4, schedule: int = VC_SCHED_PARABOLA,
                             drop_mode: int = VC_DROP_SURVIVORS) -> Tuple[List[int], int, int]:
    """Host planner with a budget schedule and drop-set choice: returns (B[L], Nq, h)."""
    B = (ctypes.c_int32 * L)()
    nq, hh = ctypes.c_int32(), ctypes.c_int32()
    _check("viscache_plan_budgets_ex",
           lib().viscache_plan_budgets_ex(L, n_vis, rr_num, rr_den, h, m_num, m_den, schedule,
                                          drop_mode, B, ctypes.byref(nq), ctypes.byref(hh)))
    return list(B), nq.value, hh.value


def viscache_scout_mmr(H: torch.Tensor, prompt: torch.Tensor, n_frames: Sequence[int], lam: float = 0.7,
                       p: Tuple[int, int] = (3, 4), with_gains: bool = True, stream=None,
                       out: Optional[Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]] = None,
                       ws: Optional[torch.Tensor] = None):
    """Keyframe selection, Eq. (mmr): returns (order, keyframes, gains, k per video).

    H: device fp32 [sum F][D], prompt: device fp32 [n_req][D].  ``out`` may
    hold preallocated (order, keyframes, gains) int32/int32/fp32 [sum k]
    tensors and ``ws`` a workspace, so repeated calls allocate nothing.
    """
    n_req = len(n_frames)
    D = H.shape[1]
    nf = (ctypes.c_int32 * n_req)(*n_frames)
    need = lib().viscache_scout_workspace_size(n_req, nf, D)
    if need == 0:
        raise VisCacheError("viscache_scout_workspace_size", VC_ERR_INVALID_ARG)
    kk = (ctypes.c_int32 * n_req)()
    _check("viscache_scout_sizes", lib().viscache_scout_sizes(n_req, nf, p[0], p[1], kk))
    ks = list(kk)
    dev = H.device
    if out is not None:
        order, keys, gains = out
    else:
        order = _empty(sum(ks), torch.int32, dev, stream)
        keys = _empty(sum(ks), torch.int32, dev, stream)
        gains = _empty(sum(ks), torch.float32, dev, stream) if with_gains else None
    ws = _workspace(need, dev, ws, stream)
    k_out = (ctypes.c_int32 * n_req)()
    if H.dtype != torch.float32 or prompt.dtype != torch.float32 or not H.is_contiguous() \
            or not prompt.is_contiguous() or prompt.shape != (n_req, D) or H.shape[0] != sum(n_frames):
        raise VisCacheError("viscache_scout_mmr", VC_ERR_INVALID_ARG)
    _check("viscache_scout_mmr", lib().viscache_scout_mmr(
        _ptr(H), _ptr(prompt), n_req, nf, D, float(lam), p[0], p[1], _ptr(order), _ptr(keys),
        _ptr(gains), k_out, _ptr(ws), ws.numel(), _stream(stream)))
    assert list(k_out) == ks
    return order, keys, gains, ks


def prunekv_score_workspace_size(L: int, Hq: int, W: int) -> int:
    return lib().prunekv_score_workspace_size(L, Hq, W)


def prunekv_score(Qw: torch.Tensor, K: torch.Tensor, scale: float = 0.0,
                  rank_mode: int = VC_RANK_SHARED, row_lse: Optional[torch.Tensor] = None,
                  scores: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """Eq. (token_score): scores [Hkv][n] (shared) or [L][Hkv][n] (per layer), fp32."""
    L, Hq, W, d = Qw.shape
    _, Hkv, n, _ = K.shape
    if scores is None:
        shape = (Hkv, n) if rank_mode == VC_RANK_SHARED else (L, Hkv, n)
        scores = _empty(shape, torch.float32, K.device, stream)
    ws = _workspace(prunekv_score_workspace_size(L, Hq, W), K.device, ws, stream)
    _check("prunekv_score", lib().prunekv_score(
        _ptr(Qw), _ptr(K), _dtype_code(K), L, Hq, Hkv, d, n, W, float(scale), rank_mode,
        _ptr(row_lse), _ptr(scores), _ptr(ws), ws.numel(), _stream(stream)))
    return scores


def prunekv_score_static_capacity() -> int:
    """Bytes of the library's fixed scratch array (VC_STATIC_SCRATCH_BYTES)."""
    return lib().prunekv_score_static_capacity()


def prunekv_score_static_status(stream=None) -> int:
    """Device status of the last prunekv_score_static call (synchronises `stream`)."""
    return lib().prunekv_score_static_status(_stream(stream))


def prunekv_score_static(Qw: torch.Tensor, K: torch.Tensor, scale: float = 0.0,
                         rank_mode: int = VC_RANK_SHARED, row_lse: Optional[torch.Tensor] = None,
                         scores: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """prunekv_score with the library's fixed scratch array instead of a workspace.

    For callers that cannot allocate device memory: the C entry point
    allocates nothing (pass ``scores`` to keep this wrapper allocation-free
    too).  Calls overlapping on the GPU race on the shared scratch.
    """
    L, Hq, W, d = Qw.shape
    _, Hkv, n, _ = K.shape
    if scores is None:
        shape = (Hkv, n) if rank_mode == VC_RANK_SHARED else (L, Hkv, n)
        scores = _empty(shape, torch.float32, K.device, stream)
    _check("prunekv_score_static", lib().prunekv_score_static(
        _ptr(Qw), _ptr(K), _dtype_code(K), L, Hq, Hkv, d, n, W, float(scale), rank_mode,
        _ptr(row_lse), _ptr(scores), _stream(stream)))
    return scores


def prunekv_select_workspace_size(L: int, Hkv: int, n_vis: int, rank_mode: int = VC_RANK_SHARED) -> int:
    return lib().prunekv_select_workspace_size(L, Hkv, n_vis, rank_mode)


def drop_rows(B: Sequence[int], Nq: int, Hkv: int) -> int:
    return Hkv * sum(Nq - b for b in B if b > 0)


def prunekv_select(scores: torch.Tensor, B: Sequence[int], Nq: int, rank_mode: int = VC_RANK_SHARED,
                   ws: Optional[torch.Tensor] = None, stream=None):
    """Ranking and keep/drop lists: returns (rank, keep_idx, drop_idx), int32 device tensors."""
    L = len(B)
    Hkv, n = scores.shape[-2], scores.shape[-1]
    dev = scores.device
    rank = _empty(scores.shape, torch.int32, dev, stream)
    keep = _empty(max(1, Hkv * sum(B)), torch.int32, dev, stream)
    drop = _empty(max(1, drop_rows(B, Nq, Hkv)), torch.int32, dev, stream)
    ws = _workspace(prunekv_select_workspace_size(L, Hkv, n, rank_mode), dev, ws, stream)
    _check("prunekv_select", lib().prunekv_select(
        _ptr(scores), L, Hkv, n, _i32(B), Nq, rank_mode, _ptr(rank), _ptr(keep), _ptr(drop),
        _ptr(ws), ws.numel(), _stream(stream)))
    return rank, keep[:Hkv * sum(B)], drop[:drop_rows(B, Nq, Hkv)]


def prunekv_fuse_workspace_size(B: Sequence[int], Hkv: int, d: int, n_vis: int, Nq: int) -> int:
    return lib().prunekv_fuse_workspace_size(_i32(B), len(B), Hkv, d, n_vis, Nq)


def prunekv_fuse_compact(K: torch.Tensor, V: torch.Tensor, B: Sequence[int], Nq: int,
                         keep_idx: torch.Tensor, drop_idx: torch.Tensor, mu: float = 0.7,
                         tau: float = 1.0, K_out: Optional[torch.Tensor] = None,
                         V_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                         stream=None):
    """Prune keys / fuse values (Eq. redistribution, Eq. weight_fusion): returns (K_out, V_out)."""
    L, Hkv, n, d = K.shape
    rows = Hkv * sum(B)
    if K_out is None:
        K_out = _empty((max(rows, 1), d), K.dtype, K.device, stream)
    if V_out is None:
        V_out = _empty((max(rows, 1), d), V.dtype, V.device, stream)
    with _on(stream):
        keep_idx = keep_idx if keep_idx.numel() else torch.zeros(1, dtype=torch.int32, device=K.device)
        drop_idx = drop_idx if drop_idx.numel() else torch.zeros(1, dtype=torch.int32, device=K.device)
    ws = _workspace(prunekv_fuse_workspace_size(B, Hkv, d, n, Nq), K.device, ws, stream)
    _check("prunekv_fuse_compact", lib().prunekv_fuse_compact(
        _ptr(K), _ptr(V), _dtype_code(K), L, Hkv, d, n, _i32(B), Nq, _ptr(keep_idx),
        _ptr(drop_idx), float(mu), float(tau), _ptr(K_out), _ptr(V_out), _ptr(ws), ws.numel(),
        _stream(stream)))
    return K_out[:rows], V_out[:rows]


class Batch:
    """Host description of a batch (vc_batch) kept alive with its arrays."""

    def __init__(self, n_vis: Sequence[int], W: Sequence[int], rr: Sequence[Tuple[int, int]]):
        k = len(n_vis)
        self._n = (ctypes.c_int32 * k)(*n_vis)
        self._w = (ctypes.c_int32 * k)(*W)
        self._a = (ctypes.c_uint32 * k)(*[a for a, _ in rr])
        self._b = (ctypes.c_uint32 * k)(*[b for _, b in rr])
        self.c = vc_batch(k, self._n, self._w, self._a, self._b)
        self.n_vis, self.W, self.rr = list(n_vis), list(W), list(rr)


def make_params(L: int, Hq: int, Hkv: int, d: int, dtype: int, h: int = 0, m=(3, 4),
                mu: float = 0.7, tau: float = 1.0, scale: float = 0.0,
                rank_mode: int = VC_RANK_SHARED, schedule: int = VC_SCHED_PARABOLA,
                drop_mode: int = VC_DROP_SURVIVORS) -> vc_params:
    return vc_params(L, Hq, Hkv, d, dtype, h, m[0], m[1], mu, tau, scale, rank_mode, schedule,
                     drop_mode)


def prunekv_workspace_size(batch: Batch, params: vc_params) -> int:
    return lib().prunekv_workspace_size(ctypes.byref(batch.c), ctypes.byref(params))


def compressed_rows(batch: Batch, params: vc_params) -> int:
    rows = 0
    for n, (a, b) in zip(batch.n_vis, batch.rr):
        B, _, _ = viscache_plan_budgets_ex(params.L, n, a, b, params.h, params.m_num, params.m_den,
                                           params.schedule, params.drop_mode)
        rows += params.Hkv * sum(B)
    return rows


def prunekv_compress(batch: Batch, params: vc_params, Qw: torch.Tensor, K: torch.Tensor,
                     V: torch.Tensor, K_out: Optional[torch.Tensor] = None,
                     V_out: Optional[torch.Tensor] = None, idx_out: Optional[torch.Tensor] = None,
                     ws: Optional[torch.Tensor] = None, stream=None):
    """The whole pass over a packed batch: returns (K_out, V_out, idx_out)."""
    rows = compressed_rows(batch, params)
    dev = K.device
    if K_out is None:
        K_out = _empty((max(rows, 1), params.d), K.dtype, dev, stream)
    if V_out is None:
        V_out = _empty((max(rows, 1), params.d), V.dtype, dev, stream)
    if idx_out is None:
        idx_out = _empty(max(rows, 1), torch.int32, dev, stream)
    ws = _workspace(prunekv_workspace_size(batch, params), dev, ws, stream)
    _check("prunekv_compress", lib().prunekv_compress(
        ctypes.byref(batch.c), ctypes.byref(params), _ptr(Qw), _ptr(K), _ptr(V), _ptr(K_out),
        _ptr(V_out), _ptr(idx_out), _ptr(ws), ws.numel(), _stream(stream)))
    return K_out[:rows], V_out[:rows], idx_out[:rows]


def viscache_decode_workspace_size(batch: Batch, params: vc_params,
                                   n_text: Optional[Sequence[int]] = None) -> int:
    return lib().viscache_decode_workspace_size(ctypes.byref(batch.c), ctypes.byref(params),
                                                _i32(n_text) if n_text is not None else None)


def viscache_decode_attention(batch: Batch, params: vc_params, layer: int, q: torch.Tensor,
                              K_out: torch.Tensor, V_out: torch.Tensor,
                              K_text: Optional[torch.Tensor] = None, V_text: Optional[torch.Tensor] = None,
                              n_text: Optional[Sequence[int]] = None, out: Optional[torch.Tensor] = None,
                              ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One decode step's attention in `layer` over the compressed cache: q [n_req][Hq][d] -> out."""
    if out is None:
        with _on(stream):
            out = torch.empty_like(q)
    nt = _i32(n_text) if n_text is not None else None
    if ws is None:
        need = lib().viscache_decode_workspace_size(ctypes.byref(batch.c), ctypes.byref(params), nt)
        if need == 0:
            raise VisCacheError("viscache_decode_workspace_size", VC_ERR_INVALID_ARG)
        ws = _workspace(need, q.device, None, stream)
    _check("viscache_decode_attention", lib().viscache_decode_attention(
        ctypes.byref(batch.c), ctypes.byref(params), int(layer), _ptr(q), _ptr(K_out), _ptr(V_out),
        _ptr(K_text), _ptr(V_text), nt, _ptr(out), _ptr(ws), ws.numel(), _stream(stream)))
    return out


def viscache_decode_attention_kv4(batch: Batch, params: vc_params, layer: int, q: torch.Tensor,
                                  kv4, K_text: Optional[torch.Tensor] = None,
                                  V_text: Optional[torch.Tensor] = None, n_text: Optional[Sequence[int]] = None,
                                  out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                                  stream=None) -> torch.Tensor:
    """Decode step in `layer` over the 4-bit cache kv4 = (K_codes, V_codes, K_params, V_params)."""
    if out is None:
        with _on(stream):
            out = torch.empty_like(q)
    nt = _i32(n_text) if n_text is not None else None
    if ws is None:
        need = lib().viscache_decode_workspace_size(ctypes.byref(batch.c), ctypes.byref(params), nt)
        if need == 0:
            raise VisCacheError("viscache_decode_workspace_size", VC_ERR_INVALID_ARG)
        ws = _workspace(need, q.device, None, stream)
    kc, vc_, kp, vp_ = kv4
    _check("viscache_decode_attention_kv4", lib().viscache_decode_attention_kv4(
        ctypes.byref(batch.c), ctypes.byref(params), int(layer), _ptr(q), _ptr(kc), _ptr(vc_), _ptr(kp),
        _ptr(vp_), _ptr(K_text), _ptr(V_text), nt, _ptr(out), _ptr(ws), ws.numel(), _stream(stream)))
    return out


def viscache_kv4_sizes(batch: Batch, params: vc_params) -> Tuple[int, int]:
    """(rows, key groups) of the compacted cache's 4-bit form."""
    rows, groups = ctypes.c_int64(0), ctypes.c_int64(0)
    _check("viscache_kv4_sizes", lib().viscache_kv4_sizes(ctypes.byref(batch.c), ctypes.byref(params),
                                                          ctypes.byref(rows), ctypes.byref(groups)))
    return rows.value, groups.value


def viscache_kv4_quantize(batch: Batch, params: vc_params, K_out: torch.Tensor, V_out: torch.Tensor,
                          out=None, stream=None):
    """4-bit codes and (scale, min) parameters of the compacted cache:
    returns (K_codes [rows][d/2], V_codes [rows][d/2], K_params [groups][d][2], V_params [rows][d/32][2])."""
    rows, groups = viscache_kv4_sizes(batch, params)
    d, dev = params.d, K_out.device
    if out is None:
        out = (_empty((max(rows, 1), d // 2), torch.uint8, dev, stream),
               _empty((max(rows, 1), d // 2), torch.uint8, dev, stream),
               _empty((max(groups, 1), d, 2), torch.float32, dev, stream),
               _empty((max(rows, 1), d // 32, 2), torch.float32, dev, stream))
    kc, vc_, kp, vp_ = out
    _check("viscache_kv4_quantize", lib().viscache_kv4_quantize(
        ctypes.byref(batch.c), ctypes.byref(params), _ptr(K_out), _ptr(V_out), _ptr(kc), _ptr(vc_),
        _ptr(kp), _ptr(vp_), _stream(stream)))
    return kc[:rows], vc_[:rows], kp[:groups], vp_[:rows]


def viscache_kv4_dequantize(batch: Batch, params: vc_params, K_codes: torch.Tensor, V_codes: torch.Tensor,
                            K_params: torch.Tensor, V_params: torch.Tensor, dtype=torch.bfloat16,
                            out=None, stream=None):
    """Reconstruction (K_hat, V_hat) [rows][d] of the 4-bit cache in `dtype`."""
    rows = K_codes.shape[0]
    if out is None:
        out = (_empty((max(rows, 1), params.d), dtype, K_codes.device, stream),
               _empty((max(rows, 1), params.d), dtype, K_codes.device, stream))
    kh, vh = out
    _check("viscache_kv4_dequantize", lib().viscache_kv4_dequantize(
        ctypes.byref(batch.c), ctypes.byref(params), _ptr(K_codes), _ptr(V_codes), _ptr(K_params),
        _ptr(V_params), _ptr(kh), _ptr(vh), _stream(stream)))
    return kh[:rows], vh[:rows]


# ---------------------------------------------------------------------------
# Rotary positions with several axes and the 8-bit paged cache

def make_rope(sections: Sequence[int], theta: float = 10000.0, interleaved: bool = False,
              adjacent: bool = False) -> vc_rope:
    """Rotary description: frequencies of each axis, their order and how values are paired."""
    if not 1 <= len(sections) <= 4:
        raise VisCacheError("make_rope", VC_ERR_INVALID_ARG)
    return vc_rope(len(sections), (ctypes.c_int32 * 4)(*sections),
                   VC_ROPE_INTERLEAVED if interleaved else VC_ROPE_SECTIONED,
                   VC_ROPE_ADJACENT if adjacent else VC_ROPE_HALVES, theta)


_current_device = torch._C._cuda_getDevice
_TYPE = {torch.bfloat16: VC_BF16, torch.float32: VC_F32}


def _rows(fn: str, t: torch.Tensor, dtype, dev: int, rows: int, heads: int, d: int) -> Tuple[int, int]:
    """Row and head stride of [rows][heads][d] rows with dense d on the current device (a step's calls
    are a few microseconds, so the checks read each attribute once)."""
    if t.dtype != dtype or t.get_device() != dev or t.shape != (rows, heads, d):
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    r, h, e = t.stride()
    if heads == 1:
        h = d                    # a stride along a single entry means nothing
    if rows == 1:
        r = max(heads * h, heads * d)
    if e != 1 and d != 1:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    return r, h


def _type(t: torch.Tensor) -> int:
    code = _TYPE.get(t.dtype)
    return _dtype_code(t) if code is None else code       # raises TypeError


def _raw_stream(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def viscache_mrope(rope: vc_rope, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None,
                   inverse: bool = False, q_out: Optional[torch.Tensor] = None,
                   k_out: Optional[torch.Tensor] = None, stream=None):
    """Rotary positions with several axes: q [rows][Hq][d], k [rows][Hkv][d] -> (q_out, k_out).

    positions: device int32 [n_axes][rows].  Rows may be strided (a slice of a
    fused projection); ``q_out``/``k_out`` may be ``q``/``k`` themselves.
    """
    fn = "viscache_mrope"
    code, dt, dev = _type(q), q.dtype, _current_device()
    if q.dim() != 3:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rows, Hq, d = q.shape
    if q_out is None:
        q_out = _empty((rows, Hq, d), dt, q.device, stream)
    qs, qh = _rows(fn, q, dt, dev, rows, Hq, d)
    qos, qoh = _rows(fn, q_out, dt, dev, rows, Hq, d)
    Hkv, ks, kos, kp, kop, kh, koh = 0, 0, 0, None, None, d, d
    if k is not None:
        Hkv = k.shape[1]
        if k_out is None:
            k_out = _empty((rows, Hkv, d), dt, q.device, stream)
        ks, kh = _rows(fn, k, dt, dev, rows, Hkv, d)
        kos, koh = _rows(fn, k_out, dt, dev, rows, Hkv, d)
        kp, kop = k.data_ptr(), k_out.data_ptr()
    else:
        k_out = None
    if qh != d or qoh != d or kh != d or koh != d or positions.dtype != torch.int32 or \
            positions.shape != (rope.n_axes, rows) or not positions.is_contiguous() or positions.get_device() != dev:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rc = lib().viscache_mrope(rope, positions.data_ptr(), code, rows, Hq, Hkv, d, q.data_ptr(), qs, kp, ks,
                              1 if inverse else 0, q_out.data_ptr(), qos, kop, kos, _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return q_out, k_out


class Kv8Cache:
    """One layer's 8-bit pool (vc_kv8) kept alive with its tensors: codes uint8 (or
    float8_e4m3fn) [n_pages][Hkv][page][d], scales fp32 [n_pages][Hkv]."""

    def __init__(self, K_codes: torch.Tensor, V_codes: torch.Tensor, K_scale: torch.Tensor, V_scale: torch.Tensor):
        n, Hkv, page, d = K_codes.shape
        for t in (K_codes, V_codes):
            if t.dtype not in (torch.uint8, torch.float8_e4m3fn) or t.shape != (n, Hkv, page, d) or \
                    not t.is_contiguous():
                raise VisCacheError("Kv8Cache", VC_ERR_INVALID_ARG)
        for t in (K_scale, V_scale):
            if t.dtype != torch.float32 or t.shape != (n, Hkv) or not t.is_contiguous():
                raise VisCacheError("Kv8Cache", VC_ERR_INVALID_ARG)
        if len({t.device for t in (K_codes, V_codes, K_scale, V_scale)}) != 1:
            raise VisCacheError("Kv8Cache", VC_ERR_INVALID_ARG)
        self.tensors = (K_codes, V_codes, K_scale, V_scale)
        self.n_pages, self.Hkv, self.page, self.d = n, Hkv, page, d
        self.device, self.index = K_codes.device, K_codes.get_device()
        self.c = vc_kv8(K_codes.data_ptr(), V_codes.data_ptr(), K_scale.data_ptr(), V_scale.data_ptr(), n, Hkv,
                        page, d)

    @classmethod
    def empty(cls, n_pages: int, Hkv: int, page: int, d: int, device="cuda") -> "Kv8Cache":
        """A pool with nothing in it (what unwritten slots hold is never used)."""
        return cls(torch.empty((n_pages, Hkv, page, d), dtype=torch.uint8, device=device),
                   torch.empty((n_pages, Hkv, page, d), dtype=torch.uint8, device=device),
                   torch.empty((n_pages, Hkv), dtype=torch.float32, device=device),
                   torch.empty((n_pages, Hkv), dtype=torch.float32, device=device))


class Kv8Step:
    """The requests of one step (vc_kv8_step) kept alive with their device arrays: block_table int32
    [n_req][max_pages], seq_lens int32 [n_req], row_start int32 [n_req + 1], and the packed rows."""

    def __init__(self, block_table: torch.Tensor, seq_lens: torch.Tensor, row_start: torch.Tensor, n_rows: int):
        n = seq_lens.shape[0]
        for t, shape in ((block_table, (n, block_table.shape[-1])), (seq_lens, (n,)), (row_start, (n + 1,))):
            if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous() or t.device != seq_lens.device:
                raise VisCacheError("Kv8Step", VC_ERR_INVALID_ARG)
        self.tensors = (block_table, seq_lens, row_start)
        self.n_rows, self.device, self.index = int(n_rows), seq_lens.device, seq_lens.get_device()
        self.c = vc_kv8_step(n, block_table.shape[1], block_table.data_ptr(), seq_lens.data_ptr(),
                             row_start.data_ptr(), self.n_rows)


def viscache_kv8_workspace_size(n_rows: int, Hq: int, Hkv: int, d: int) -> int:
    return lib().viscache_kv8_workspace_size(n_rows, Hq, Hkv, d)


def _kv8_ws(fn: str, cache: Kv8Cache, step: Kv8Step, Hq: int, ws: Optional[torch.Tensor], stream):
    # the device of the call, and the workspace on it
    dev = _current_device()
    if cache.index != dev or step.index != dev:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    if ws is None:
        need = viscache_kv8_workspace_size(step.n_rows, Hq, cache.Hkv, cache.d)
        if need == 0:
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
        ws = _workspace(need, cache.device, None, stream)
    elif ws.get_device() != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    return dev, ws


def viscache_kv8_append(cache: Kv8Cache, step: Kv8Step, K: torch.Tensor, V: torch.Tensor,
                        ws: Optional[torch.Tensor] = None, stream=None) -> None:
    """Write the step's rows K, V [rows][Hkv][d] into the cache (row and head strides of at least d,
    multiples of 16 bytes: slices of a fused projection and transposed blocks are read in place)."""
    fn = "viscache_kv8_append"
    dev, ws = _kv8_ws(fn, cache, step, cache.Hkv, ws, stream)
    code, dt = _type(K), K.dtype
    kr, kh = _rows(fn, K, dt, dev, step.n_rows, cache.Hkv, cache.d)
    vr, vh = _rows(fn, V, dt, dev, step.n_rows, cache.Hkv, cache.d)
    rc = lib().viscache_kv8_append(cache.c, step.c, code, K.data_ptr(), kr, kh, V.data_ptr(), vr, vh, ws.data_ptr(),
                                   ws.numel(), _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)


def viscache_kv8_read(cache: Kv8Cache, step: Kv8Step, dtype=torch.bfloat16, out=None,
                      ws: Optional[torch.Tensor] = None, stream=None):
    """The step's rows back from the cache: (K_hat, V_hat) [rows][Hkv][d] in `dtype` (or `out`'s)."""
    fn = "viscache_kv8_read"
    dev, ws = _kv8_ws(fn, cache, step, cache.Hkv, ws, stream)
    if out is None:
        shape = (step.n_rows, cache.Hkv, cache.d)
        out = (_empty(shape, dtype, cache.device, stream),
               _empty(shape, dtype, cache.device, stream))
    kh, vh = out
    code = _type(kh)
    for t in out:
        _rows(fn, t, kh.dtype, dev, step.n_rows, cache.Hkv, cache.d)
        if not t.is_contiguous():
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rc = lib().viscache_kv8_read(cache.c, step.c, code, kh.data_ptr(), vh.data_ptr(), ws.data_ptr(), ws.numel(),
                                 _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return kh, vh


def viscache_kv8_attention(cache: Kv8Cache, step: Kv8Step, q: torch.Tensor, scale: float = 0.0,
                           causal: bool = True, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """The step's query rows q [rows][Hq][d] over their requests' pages: out [rows][Hq][d]; ``lse`` fp32
    [rows][Hq] takes the log of each softmax's normaliser."""
    fn = "viscache_kv8_attention"
    code, dt = _type(q), q.dtype
    if q.dim() != 3:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rows, Hq, d = step.n_rows, q.shape[1], cache.d
    dev, ws = _kv8_ws(fn, cache, step, Hq, ws, stream)
    qs, qh = _rows(fn, q, dt, dev, rows, Hq, d)
    if out is None:
        out = _empty((rows, Hq, d), dt, q.device, stream)
    _rows(fn, out, dt, dev, rows, Hq, d)
    lp = None
    if lse is not None:
        if lse.dtype != torch.float32 or lse.shape != (rows, Hq) or not lse.is_contiguous() or lse.get_device() != dev:
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
        lp = lse.data_ptr()
    if qh != d or not out.is_contiguous():
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rc = lib().viscache_kv8_attention(cache.c, step.c, code, Hq, q.data_ptr(), qs, scale, 1 if causal else 0,
                                      out.data_ptr(), lp, ws.data_ptr(), ws.numel(), _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return out


# ---------------------------------------------------------------------------
# The rest of a decode step around the 8-bit paged cache

def _flat(fn: str, t: torch.Tensor, dtype, dev: int, shape) -> int:
    """Address of a dense tensor of that type and shape on the current device."""
    if t.dtype != dtype or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    return t.data_ptr()


def _heads(fn: str, t: torch.Tensor, dtype, dev: int, rows: int, heads: int, d: int) -> int:
    """Row stride of rows whose heads are dense."""
    r, h = _rows(fn, t, dtype, dev, rows, heads, d)
    if h != d:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    return r


def viscache_norm_mrope(rope: vc_rope, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor],
                        q_weight: torch.Tensor, k_weight: Optional[torch.Tensor], eps: float = 1e-6,
                        q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """Heads normed by their root mean square, times q_weight / k_weight [d], and rotated as by
    viscache_mrope: q [rows][Hq][d], k [rows][Hkv][d] (or None, with None for its weight) -> (q_out, k_out).

    Rows may be strided; ``q_out``/``k_out`` may be ``q``/``k`` themselves.
    """
    fn = "viscache_norm_mrope"
    code, dt, dev = _type(q), q.dtype, _current_device()
    if q.dim() != 3:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rows, Hq, d = q.shape
    if q_out is None:
        q_out = _empty((rows, Hq, d), dt, q.device, stream)
    qs, qos = _heads(fn, q, dt, dev, rows, Hq, d), _heads(fn, q_out, dt, dev, rows, Hq, d)
    Hkv, ks, kos, kp, kop, kw = 0, 0, 0, None, None, None
    if k is not None:
        if k.dim() != 3 or k_weight is None:
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
        Hkv = k.shape[1]
        if k_out is None:
            k_out = _empty((rows, Hkv, d), dt, q.device, stream)
        ks, kos = _heads(fn, k, dt, dev, rows, Hkv, d), _heads(fn, k_out, dt, dev, rows, Hkv, d)
        kp, kop, kw = k.data_ptr(), k_out.data_ptr(), _flat(fn, k_weight, dt, dev, (d,))
    else:
        k_out = None
    rc = lib().viscache_norm_mrope(rope, _flat(fn, positions, torch.int32, dev, (rope.n_axes, rows)), code, rows, Hq,
                                   Hkv, d, q.data_ptr(), qs, kp, ks, _flat(fn, q_weight, dt, dev, (d,)), kw, eps,
                                   q_out.data_ptr(), qos, kop, kos, _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return q_out, k_out


def viscache_norm_mrope_grad_workspace_size(n_rows: int, Hq: int, Hkv: int, d: int) -> int:
    return lib().viscache_norm_mrope_grad_workspace_size(n_rows, Hq, Hkv, d)


def viscache_norm_mrope_grad(rope: vc_rope, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor],
                             q_out_grad: torch.Tensor, k_out_grad: Optional[torch.Tensor], q_weight: torch.Tensor,
                             k_weight: Optional[torch.Tensor], eps: float = 1e-6,
                             q_grad: Optional[torch.Tensor] = None, k_grad: Optional[torch.Tensor] = None,
                             q_weight_grad: Optional[torch.Tensor] = None,
                             k_weight_grad: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                             stream=None):
    """Gradient of viscache_norm_mrope: (q_grad, k_grad) rows and (q_weight_grad, k_weight_grad) fp32 [d].

    q, k are the forward call's inputs, q_out_grad, k_out_grad the gradients of its outputs; the weights'
    gradients are written, not added to.
    """
    fn = "viscache_norm_mrope_grad"
    code, dt, dev = _type(q), q.dtype, _current_device()
    if q.dim() != 3:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rows, Hq, d = q.shape
    if q_grad is None:
        q_grad = _empty((rows, Hq, d), dt, q.device, stream)
    if q_weight_grad is None:
        q_weight_grad = _empty((d,), torch.float32, q.device, stream)
    qs, qgs = _heads(fn, q, dt, dev, rows, Hq, d), _heads(fn, q_grad, dt, dev, rows, Hq, d)
    qys = _heads(fn, q_out_grad, dt, dev, rows, Hq, d)
    Hkv, ks, kys, kgs, kp, kyp, kgp, kw, kwg = 0, 0, 0, 0, None, None, None, None, None
    if k is not None:
        if k.dim() != 3 or k_weight is None or k_out_grad is None:
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
        Hkv = k.shape[1]
        if k_grad is None:
            k_grad = _empty((rows, Hkv, d), dt, q.device, stream)
        if k_weight_grad is None:
            k_weight_grad = _empty((d,), torch.float32, q.device, stream)
        ks, kgs = _heads(fn, k, dt, dev, rows, Hkv, d), _heads(fn, k_grad, dt, dev, rows, Hkv, d)
        kys = _heads(fn, k_out_grad, dt, dev, rows, Hkv, d)
        kp, kyp, kgp = k.data_ptr(), k_out_grad.data_ptr(), k_grad.data_ptr()
        kw, kwg = _flat(fn, k_weight, dt, dev, (d,)), _flat(fn, k_weight_grad, torch.float32, dev, (d,))
    else:
        k_grad = k_weight_grad = None
    if ws is None:
        need = viscache_norm_mrope_grad_workspace_size(rows, Hq, Hkv, d)
        if need == 0:
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
        ws = _workspace(need, q.device, None, stream)
    elif ws.get_device() != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rc = lib().viscache_norm_mrope_grad(
        rope, _flat(fn, positions, torch.int32, dev, (rope.n_axes, rows)), code, rows, Hq, Hkv, d, q.data_ptr(), qs,
        kp, ks, q_out_grad.data_ptr(), qys, kyp, kys, _flat(fn, q_weight, dt, dev, (d,)), kw, eps, q_grad.data_ptr(),
        qgs, kgp, kgs, _flat(fn, q_weight_grad, torch.float32, dev, (d,)), kwg, ws.data_ptr(), ws.numel(),
        _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return q_grad, k_grad, q_weight_grad, k_weight_grad


def viscache_kv8_weigh(cache: Kv8Cache, step: Kv8Step, q: torch.Tensor, lse: torch.Tensor, weights: torch.Tensor,
                       scale: float = 0.0, causal: bool = True, ws: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """Adds the attention that the step's rows q [rows][Hq][d] pay each cached token to `weights` fp32
    [n_pages][Hkv][page]; ``lse`` fp32 [rows][Hq] is viscache_kv8_attention's.  Returns `weights`."""
    fn = "viscache_kv8_weigh"
    code, dt = _type(q), q.dtype
    if q.dim() != 3:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rows, Hq, d = step.n_rows, q.shape[1], cache.d
    dev, ws = _kv8_ws(fn, cache, step, Hq, ws, stream)
    qs = _heads(fn, q, dt, dev, rows, Hq, d)
    rc = lib().viscache_kv8_weigh(cache.c, step.c, code, Hq, q.data_ptr(), qs,
                                  _flat(fn, lse, torch.float32, dev, (rows, Hq)), scale, 1 if causal else 0,
                                  _flat(fn, weights, torch.float32, dev, (cache.n_pages, cache.Hkv, cache.page)),
                                  ws.data_ptr(), ws.numel(), _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return weights


def viscache_kv8_evict_workspace_size(n_req: int, Hkv: int) -> int:
    return lib().viscache_kv8_evict_workspace_size(n_req, Hkv)


def viscache_kv8_evict(cache: Kv8Cache, step: Kv8Step, weights: torch.Tensor, keep: torch.Tensor, max_keep: int,
                       sink: int = 0, recent: int = 0, kept: Optional[torch.Tensor] = None,
                       new_lens: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Holds each request to its keep[r] (int32, on the device, at most max_keep) heaviest tokens of each
    KV head, in place: (kept int32 [n_req][Hkv][max_keep], new_lens int32 [n_req]).  ``new_lens`` may be
    the step's seq_lens."""
    fn = "viscache_kv8_evict"
    dev, n = _current_device(), step.c.n_req
    if cache.index != dev or step.index != dev or max_keep < 1:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    if kept is None:
        kept = _empty((n, cache.Hkv, max_keep), torch.int32, cache.device, stream)
    if new_lens is None:
        new_lens = _empty((n,), torch.int32, cache.device, stream)
    if ws is None:
        need = viscache_kv8_evict_workspace_size(n, cache.Hkv)
        if need == 0:
            raise VisCacheError(fn, VC_ERR_INVALID_ARG)
        ws = _workspace(need, cache.device, None, stream)
    elif ws.get_device() != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    rc = lib().viscache_kv8_evict(cache.c, step.c,
                                  _flat(fn, weights, torch.float32, dev, (cache.n_pages, cache.Hkv, cache.page)),
                                  _flat(fn, keep, torch.int32, dev, (n,)), max_keep, sink, recent,
                                  _flat(fn, kept, torch.int32, dev, (n, cache.Hkv, max_keep)),
                                  _flat(fn, new_lens, torch.int32, dev, (n,)), ws.data_ptr(), ws.numel(),
                                  _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return kept, new_lens


def viscache_sample(logits: torch.Tensor, u: torch.Tensor, temperature: torch.Tensor,
                    top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                    min_p: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None,
                    logprob: Optional[torch.Tensor] = None, stream=None):
    """The next token of each row of logits [rows][vocab] from random numbers u [rows] in [0, 1):
    (token int32 [rows], logprob fp32 [rows]).  temperature, top_p, min_p fp32 [rows], top_k int32 [rows];
    a filter that is None keeps everything.  Rows of logits may be strided."""
    fn = "viscache_sample"
    code, dev = _type(logits), _current_device()
    if logits.dim() != 2 or logits.get_device() != dev:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    n, vocab = logits.shape
    stride = logits.stride(0) if n > 1 else vocab
    if vocab > 1 and logits.stride(1) != 1:
        raise VisCacheError(fn, VC_ERR_INVALID_ARG)
    if token is None:
        token = _empty((n,), torch.int32, logits.device, stream)
    if logprob is None:
        logprob = _empty((n,), torch.float32, logits.device, stream)
    row = lambda t, dt: None if t is None else _flat(fn, t, dt, dev, (n,))
    rc = lib().viscache_sample(code, n, vocab, logits.data_ptr(), stride, row(u, torch.float32),
                               row(temperature, torch.float32), row(top_k, torch.int32), row(top_p, torch.float32),
                               row(min_p, torch.float32), row(token, torch.int32), row(logprob, torch.float32),
                               _raw_stream(stream, dev))
    if rc != VC_OK:
        raise VisCacheError(fn, rc)
    return token, logprob


def viscache_set_kernel_path(path: int) -> None:
    """VC_PATH_AUTO (tensor cores for bf16, d=128) or VC_PATH_SIMT (CUDA cores everywhere)."""
    _check("viscache_set_kernel_path", lib().viscache_set_kernel_path(path))


def viscache_set_dependent_launch(on: bool) -> None:
    """True (default): kernels after a call's first are dependent launches; False: ordinary launches."""
    _check("viscache_set_dependent_launch", lib().viscache_set_dependent_launch(1 if on else 0))


def viscache_test_inject_wait(kernel_mask: int) -> None:
    """Test support: the named tensor-core kernels add one wait that gives up (0 = off)."""
    _check("viscache_test_inject_wait", lib().viscache_test_inject_wait(kernel_mask))


def viscache_profile_enable(on: bool) -> None:
    _check("viscache_profile_enable", lib().viscache_profile_enable(1 if on else 0))


def viscache_profile_read(max_kernels: int = 32):
    """{kernel name: (total ms, launches)} recorded since profiling was enabled / last read."""
    names = ctypes.create_string_buffer(4096)
    ms = (ctypes.c_float * max_kernels)()
    cnt = (ctypes.c_int32 * max_kernels)()
    k = lib().viscache_profile_read(names, 4096, ms, cnt, max_kernels)
    if k < 0:
        raise VisCacheError("viscache_profile_read", -k)
    keys = names.value.decode().split("\n")[:k]
    return {keys[i]: (ms[i], cnt[i]) for i in range(k)}


def prunekv_get_status(ws: torch.Tensor, stream=None) -> int:
    return lib().prunekv_get_status(_ptr(ws), _stream(stream))
