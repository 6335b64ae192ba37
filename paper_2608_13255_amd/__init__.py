"""MI355X-native GeoCache cross-view delta transport.

Python binding of libgeocache.so (hand-written HIP kernels for gfx950 behind
the C ABI declared in include/geocache.h).  Every function here has the name
of the C entry point it wraps and only marshals arguments: it checks torch
tensors (device, dtype, contiguity, shape), allocates outputs the caller did
not supply, passes raw device pointers and the current HIP stream, and turns
a negative status into GeoCacheError.  All computation runs in the library's
kernels; there is no CPU fallback, and importing the package fails if the
library has not been built.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgeocache.so")
ABI_VERSION = 4   # GC_ABI_VERSION the binding is written for

# constants mirrored from include/geocache.h
GC_OK = 0
GC_F32, GC_BF16, GC_E4M3 = 0, 1, 2
GC_DDIM, GC_FLOW_EULER = 0, 1
GC_PRED_NONE, GC_PRED_EPS, GC_PRED_V, GC_PRED_VEL = 0, 1, 2, 3
GC_FULL_PERIODIC, GC_FULL_HEAD_MID_TAIL, GC_FULL_HEAD_TAIL_E = 0, 1, 2
GC_MAX_VIEWS, GC_MAX_ANCHORS, GC_MAX_GRID = 64, 8, 4094
GC_NOALLOC_SCRATCH_BYTES = 1 << 20
GC_MAX_HEAD_DIM, GC_MAX_HEADS, GC_MAX_AXES = 256, 1024, 4
GC_ROPE_HALF, GC_ROPE_INTERLEAVED = 0, 1
GC_ATTENTION_ITEM_WORDS = 12
GC_MAX_WIDTH, GC_MAX_INNER = 32768, 1 << 20
GC_ACT_NONE, GC_ACT_SILU, GC_ACT_GELU, GC_ACT_GELU_TANH = 0, 1, 2, 3
ERRORS = {-1: "GC_ERR_ARG", -2: "GC_ERR_SHAPE", -3: "GC_ERR_DTYPE", -4: "GC_ERR_ALIGN",
          -5: "GC_ERR_ALIAS", -6: "GC_ERR_CAPACITY", -7: "GC_ERR_HIP"}

# gc_camera: int32 model, float R[9], float t[3], fx, fy, cx, cy (68 bytes)
CAMERA_DTYPE = np.dtype([("model", "<i4"), ("R", "<f4", (9,)), ("t", "<f4", (3,)), ("fx", "<f4"),
                         ("fy", "<f4"), ("cx", "<f4"), ("cy", "<f4")])
assert CAMERA_DTYPE.itemsize == 68


class GeoCacheError(RuntimeError):
    def __init__(self, func: str, code: int, msg: str):
        super().__init__(f"{func} failed with {ERRORS.get(code, code)}: {msg}")
        self.code = code


class _Sampler(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("pred_out", ctypes.c_int32), ("T", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("beta_start", ctypes.c_double), ("beta_end", ctypes.c_double)]


class UniPCStep(ctypes.Structure):
    """gc_unipc_step: coefficients of one UniPC step (gc_unipc_coeffs)."""
    _fields_ = [("use_corrector", ctypes.c_int32), ("corrector_order", ctypes.c_int32),
                ("predictor_order", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("c_xprev", ctypes.c_double), ("c_mk2", ctypes.c_double), ("c_mk1", ctypes.c_double),
                ("c_mk", ctypes.c_double), ("p_xc", ctypes.c_double), ("p_mk1", ctypes.c_double),
                ("p_mk", ctypes.c_double)]


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


class RopeScaling(ctypes.Structure):
    """gc_rope_scaling: rotary frequencies for contexts longer than the trained one."""
    _fields_ = [("factor", ctypes.c_double), ("original_len", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double), ("amplitude", ctypes.c_double)]

    def __init__(self, factor: float, original_len: float, low: float = 1.0, high: float = 32.0,
                 amplitude: float = 1.0):
        super().__init__(factor, original_len, low, high, amplitude)


class AttentionInfo(ctypes.Structure):
    """gc_attention_info: sizes of a plan (gc_attention_plan)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "dim", "dtype", "causal", "n_seq", "total_q",
                                              "total_k", "kind", "tile_rows", "n_items", "n_slots", "n_groups")]
    _fields_ += [("reserved", ctypes.c_int32 * 3), ("workspace_bytes", ctypes.c_int64)]


@dataclass(frozen=True)
class Sampler:
    """gc_sampler: kind GC_DDIM (linear betas over T steps) or GC_FLOW_EULER."""
    kind: int = GC_DDIM
    pred_out: int = GC_PRED_NONE
    T: int = 1000
    beta_start: float = 1e-4
    beta_end: float = 0.02

    def c(self) -> _Sampler:
        """The C form, made anew: the caller's own to write to, from what the
        fields hold now."""
        return _Sampler(self.kind, self.pred_out, self.T, 0, self.beta_start, self.beta_end)


_LIB = None
_vp = ctypes.c_void_p
_i32p = ctypes.POINTER(ctypes.c_int32)
_i = ctypes.c_int
_i64 = ctypes.c_int64
_headsp = ctypes.POINTER(_Heads)
_rowsp = ctypes.POINTER(_Rows)


def lib() -> ctypes.CDLL:
    """The loaded libgeocache.so (raises if it has not been built)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it (python -c 'import __graft_entry__ as g; g.build()' "
                              "or make -C paper_2608_13255_amd)")
        L = ctypes.CDLL(LIB_PATH)
        sig = {
            "gc_abi_version": ([], _i),
            "gc_last_error": ([], ctypes.c_char_p),
            "gc_posmap_downsample": ([_vp, _i64, _i, _i, _i, _vp, _vp], _i),
            "gc_posmap_bbox": ([_vp, _i, _i, _i, _i, ctypes.c_float, _vp, _vp], _i),
            "gc_build_correspondence": ([_vp, _vp, _i, _i, _i, _i, _i32p, _i, _i, _vp, _vp, _vp, _vp, _vp], _i),
            "gc_index_workspace_bytes": ([_i64], ctypes.c_size_t),
            "gc_index_correspondence": ([_vp, _i64, _i, _i, _i, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp], _i),
            "gc_index_correspondence_noalloc": ([_vp, _i64, _i, _i, _i, _vp, _vp, _vp, _vp], _i),
            "gc_index_foreground": ([_vp, _i64, _i, _i, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp], _i),
            "gc_transport_step": ([_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _i32p, _i, _i, _i, _vp,
                                   _vp], _i),
            "gc_sampler_reconstruct": ([_vp, _vp, _vp, _vp, _i64, _i, ctypes.POINTER(_Sampler), ctypes.c_double,
                                        ctypes.c_double, _vp], _i),
            "gc_transport_reconstruct": ([_vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i, _i, _i, _i, _i, _i32p, _i,
                                          _i, _i, ctypes.POINTER(_Sampler), ctypes.c_double, ctypes.c_double, _vp,
                                          _vp, _vp, _vp], _i),
            "gc_unipc_coeffs": ([ctypes.POINTER(_Sampler), _i, _i, _i, _i, ctypes.POINTER(UniPCStep)], _i),
            "gc_unipc_update": ([_vp, _vp, _vp, _vp, _vp, _i64, _i, ctypes.POINTER(UniPCStep), _vp, _vp, _vp], _i),
            "gc_transport_unipc": ([_vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i32p,
                                    _i, _i, _i, ctypes.POINTER(UniPCStep), _vp, _vp, _vp, _vp], _i),
            "gc_transport_step_geom": ([_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _i32p, _i, _i,
                                        _i, _vp, _vp], _i),
            "gc_transport_reconstruct_geom": ([_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i, _i, _i, _i, _i,
                                               _i32p, _i, _i, _i, ctypes.POINTER(_Sampler), ctypes.c_double,
                                               ctypes.c_double, _vp, _vp, _vp, _vp], _i),
            "gc_transport_unipc_geom": ([_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i, _i, _i, _i, _i,
                                         _i32p, _i, _i, _i, ctypes.POINTER(UniPCStep), _vp, _vp, _vp, _vp], _i),
            "gc_coverage_pair_words": ([_i, _i, _i, _i], _i64),
            "gc_coverage_pairs": ([_vp, _vp, _vp, _i, _i, _i, _i, _vp, _vp], _i),
            "gc_coverage_init": ([_vp, _i, _i, _i, _i, _vp, _vp], _i),
            "gc_coverage_update": ([_vp, _i, _i, _i, _i, _i32p, _i, _i, _vp, _vp, _vp], _i),
            "gc_coverage_workspace_bytes": ([], ctypes.c_size_t),
            "gc_coverage_select": ([_vp, _vp, _i, _i, _i, _i, _i, _i32p, _i, _vp, _vp, ctypes.c_size_t, _vp], _i),
            "gc_schedule_refresh_due": ([_vp, _i, _i, ctypes.c_double, ctypes.POINTER(ctypes.c_int)], _i),
            "gc_coverage_score": ([_vp, _vp, _i, _i, _i, _i, _i32p, _i, _i, _vp, _vp, ctypes.c_size_t, _vp], _i),
            "gc_coverage_update_select": ([_vp, _i, _i, _i, _i, _i32p, _i, _i, _vp, _vp, _i, _i32p, _i, _vp, _vp,
                                           ctypes.c_size_t, _vp], _i),
            "gc_coverage_update_score": ([_vp, _i, _i, _i, _i, _i32p, _i, _i, _vp, _vp, _i32p, _i, _i, _vp, _vp,
                                          ctypes.c_size_t, _vp], _i),
            "gc_schedule_forced_views": ([_i32p, _i, _i, _i, _i32p, ctypes.POINTER(ctypes.c_int)], _i),
            "gc_schedule_advance_gaps": ([_i32p, _i, _i32p, _i, _i], _i),
            "gc_schedule_anchors": ([_i, _i, _i64, _i32p], _i),
            "gc_schedule_full_steps": ([_i, _i, _i, ctypes.POINTER(ctypes.c_uint8)], _i),
            "gc_sampler_step_times": ([ctypes.POINTER(_Sampler), _i, _i, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_double)], _i),
            "gc_sampler_alpha_bar": ([ctypes.POINTER(_Sampler), _i, ctypes.POINTER(ctypes.c_double)], _i),
            "gc_rope_table": ([_vp, _i64, _i32p, _i, ctypes.c_double, ctypes.POINTER(RopeScaling), _vp], _i),
            "gc_rope": ([_headsp, _i64, _i, _i, _i, _vp, _vp, _i64, _i32p, _i, _i, _headsp, _vp], _i),
            "gc_qk_norm_rope": ([_headsp, _i, _headsp, _i, _i64, _i, _i, _vp, _vp, ctypes.c_double, _vp, _vp, _i64,
                                 _i32p, _i, _i, _headsp, _headsp, _vp], _i),
            "gc_attention_plan": ([_i32p, _i32p, _i, _i, _i, _i, _i, _i, ctypes.POINTER(AttentionInfo), _i32p, _i64],
                                  _i),
            "gc_attention": ([_headsp, _headsp, _headsp, _headsp, _vp, ctypes.POINTER(AttentionInfo), _vp,
                              ctypes.c_double, _vp, ctypes.c_size_t, _vp], _i),
            "gc_add_rms_norm": ([_rowsp, _rowsp, _i64, _i, _i, _vp, ctypes.c_double, _rowsp, _rowsp, _i, _vp, _vp], _i),
            "gc_quantize_rows": ([_rowsp, _i64, _i, _i, _rowsp, _vp, _vp], _i),
            "gc_linear_workspace_bytes": ([_i64, _i, _i, _i, _i], _i64),
            "gc_linear": ([_rowsp, _vp, _rowsp, _vp, _i64, _i, _i, _i, _vp, _i, _i, _rowsp, _rowsp, _i, _vp,
                           ctypes.c_size_t, _vp], _i),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        if L.gc_abi_version() != ABI_VERSION:
            raise ImportError(f"libgeocache ABI {L.gc_abi_version()} != {ABI_VERSION}")
        _LIB = L
    return _LIB


def _check(rc: int, func: str) -> None:
    if rc != GC_OK:
        raise GeoCacheError(func, rc, lib().gc_last_error().decode(errors="replace"))


def _current_raw_stream() -> int:
    """Handle of torch's current stream on the current device, without the
    Stream object that torch.cuda.current_stream() builds on the way (a few
    microseconds of a step's host time)."""
    if _RAW_STREAM is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _RAW_STREAM(torch._C._cuda_getDevice())


# what torch's own generated code calls for the same purpose
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None) if hasattr(torch._C, "_cuda_getDevice") else None
_GET_DEVICE = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_raw_stream()
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _side_stream(stream) -> Optional[torch.cuda.Stream]:
    """The stream of an explicit `stream` argument when it is not torch's
    current stream (None otherwise)."""
    if stream is None:
        return None
    handle = _stream(stream)
    if handle == _current_raw_stream():
        return None
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(handle)


def _keep(stream, tensors) -> None:
    """Outputs handed to work on a side stream, the caller's among them: tell
    torch's caching allocator, so that their memory is not given to other
    work before the side stream's kernels are done with it."""
    if stream is None:
        return
    s = _side_stream(stream)
    if s is not None:
        for t in tensors:
            t.record_stream(s)


def _empty(stream, shape, dtype: torch.dtype, device) -> torch.Tensor:
    """Memory for work on `stream`.  Of a side stream's own, since current-stream
    work that has yet to end may still use what torch's allocator hands out
    here: nothing orders the side stream after it.  What the current stream
    reads of it later keeps it from being handed out again, too."""
    side = None if stream is None else _side_stream(stream)
    if side is None:
        return torch.empty(shape, dtype=dtype, device=device)
    here = torch.cuda.current_stream()
    torch.cuda.set_stream(side)             # (3.7 us with its way back; torch.cuda.stream() takes 6.1)
    try:
        t = torch.empty(shape, dtype=dtype, device=device)
    finally:
        torch.cuda.set_stream(here)
    if t.is_cuda:
        t.record_stream(here if t.device == here.device else torch.cuda.current_stream(t.device))
    return t


def _empty_like(stream, x: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """_empty of x's shape (and type), contiguous."""
    if stream is None:
        return torch.empty_like(x, dtype=dtype, memory_format=_CONTIGUOUS)
    return _empty(stream, x.shape, x.dtype if dtype is None else dtype, x.device)


def _after_side(stream) -> None:
    """Order torch's current stream (and so a following host read-back)
    after the work just enqueued on a side stream."""
    s = _side_stream(stream)
    if s is not None:
        torch.cuda.current_stream().wait_stream(s)


def _dev(t: torch.Tensor, name: str) -> int:
    if isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    raise ValueError(f"{name} must be contiguous")


def _opt(t: Optional[torch.Tensor], name: str) -> Optional[int]:
    return None if t is None else _dev(t, name)


def dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GC_F32
    if t.dtype == torch.bfloat16:
        return GC_BF16
    raise ValueError(f"latents must be float32 or bfloat16 (got {t.dtype})")


# int32 array types by length (an array type made anew for each call costs
# more than the array)
_I32 = [ctypes.c_int32 * n for n in range(GC_MAX_VIEWS + 1)]


def _anchors(anchors: Sequence[int]):
    n = len(anchors)
    return (_I32[n] if n <= GC_MAX_VIEWS else ctypes.c_int32 * n)(*map(int, anchors)), n


def camera_tensor(cams: Dict[str, np.ndarray], device="cuda") -> torch.Tensor:
    """Pack camera arrays (keys model, R, t, fx, fy, cx, cy with a common
    leading shape, e.g. [B][N]) into a device uint8 tensor of gc_camera."""
    lead = np.shape(cams["model"])
    rec = np.zeros(lead, CAMERA_DTYPE)
    rec["model"] = cams["model"]
    rec["R"] = np.reshape(cams["R"], lead + (9,))
    rec["t"] = cams["t"]
    for k in ("fx", "fy", "cx", "cy"):
        rec[k] = cams[k]
    raw = np.ascontiguousarray(rec).view(np.uint8).reshape(lead + (68,))
    return torch.from_numpy(raw.copy()).to(device)


# ---------------------------------------------------------------------------
# entry points
# ---------------------------------------------------------------------------

def gc_posmap_downsample(pos_hi: torch.Tensor, f: int, pos_lat: torch.Tensor = None, stream=None) -> torch.Tensor:
    """pos_hi float32 [..., Hr, Wr, 3] -> pos_lat float32 [..., Hr/f, Wr/f, 3]."""
    if pos_hi.dtype != torch.float32 or pos_hi.dim() < 3 or pos_hi.shape[-1] != 3:
        raise ValueError("pos_hi must be float32 [..., Hr, Wr, 3]")
    Hr, Wr = pos_hi.shape[-3], pos_hi.shape[-2]
    lead = tuple(pos_hi.shape[:-3])
    n = int(np.prod(lead)) if lead else 1
    if pos_lat is None:
        pos_lat = _empty(stream, lead + (Hr // f, Wr // f, 3), torch.float32, pos_hi.device)
    _check(lib().gc_posmap_downsample(_dev(pos_hi, "pos_hi"), n, Hr, Wr, f, _dev(pos_lat, "pos_lat"),
                                      _stream(stream)), "gc_posmap_downsample")
    return pos_lat


def gc_posmap_bbox(pos: torch.Tensor, tol_frac: float = 0.01, bbox: torch.Tensor = None, stream=None) -> torch.Tensor:
    """pos float32 [B, N, H, W, 3] -> bbox float32 [B, 8]."""
    if pos.dtype != torch.float32 or pos.dim() != 5 or pos.shape[-1] != 3:
        raise ValueError("pos must be float32 [B, N, H, W, 3]")
    B, N, H, W, _ = pos.shape
    if bbox is None:
        bbox = _empty(stream, (B, 8), torch.float32, pos.device)
    _check(lib().gc_posmap_bbox(_dev(pos, "pos"), B, N, H, W, float(tol_frac), _dev(bbox, "bbox"),
                                _stream(stream)), "gc_posmap_bbox")
    return bbox


def gc_build_correspondence(pos: torch.Tensor, cams: torch.Tensor, anchors: Sequence[int], K: int,
                            bbox: torch.Tensor, corr: torch.Tensor = None, weights: torch.Tensor = None,
                            stats: torch.Tensor = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """pos float32 [B, N, H, W, 3], cams uint8 [B, N, 68] (camera_tensor),
    bbox float32 [B, 8] -> (corr int32 [B, N-a, H, W, a], weights float32
    [B, N-a, H, W, a, K]); stats (optional) int32/uint32 [B, 4]."""
    if pos.dtype != torch.float32 or pos.dim() != 5 or pos.shape[-1] != 3:
        raise ValueError("pos must be float32 [B, N, H, W, 3]")
    B, N, H, W, _ = pos.shape
    if cams.dtype != torch.uint8 or tuple(cams.shape) != (B, N, 68):
        raise ValueError(f"cams must be uint8 [B={B}, N={N}, 68]")
    arr, a = _anchors(anchors)
    NT = N - a
    dev = pos.device
    if corr is None:
        corr = _empty(stream, (B, NT, H, W, a), torch.int32, dev)
    if weights is None:
        weights = _empty(stream, (B, NT, H, W, a, K), torch.float32, dev)
    if tuple(corr.shape) != (B, NT, H, W, a) or corr.dtype != torch.int32:
        raise ValueError("corr must be int32 [B, N-a, H, W, a]")
    if tuple(weights.shape) != (B, NT, H, W, a, K) or weights.dtype != torch.float32:
        raise ValueError("weights must be float32 [B, N-a, H, W, a, K]")
    if stats is not None and (tuple(stats.shape) != (B, 4) or stats.element_size() != 4):
        raise ValueError("stats must be a 32-bit [B, 4] tensor")
    _check(lib().gc_build_correspondence(_dev(pos, "pos"), _dev(cams, "cams"), B, N, H, W, arr, a, K,
                                         _dev(bbox, "bbox"), _dev(corr, "corr") if corr.numel() else None,
                                         _dev(weights, "weights") if weights.numel() else None,
                                         _opt(stats, "stats"), _stream(stream)), "gc_build_correspondence")
    return corr, weights


@dataclass
class VisibleIndex:
    """Output of gc_index_correspondence: vis_bits (int32 view of the uint32
    words), vis_list (int32) and the host count n_vis."""
    vis_bits: torch.Tensor
    vis_list: torch.Tensor
    n_vis: int


def gc_index_correspondence(corr: torch.Tensor, workspace: torch.Tensor = None, stream=None) -> VisibleIndex:
    """Visible-token index of a correspondence (corr int32 [B, N-a, H, W, a]),
    its list in tile order.  Reads the visible count back to the host (one
    synchronisation)."""
    if corr.dtype != torch.int32 or corr.dim() != 5:
        raise ValueError("corr must be int32 [B, N-a, H, W, a]")
    a = corr.shape[-1]
    n_tok = int(corr.numel() // a) if a else 0
    n_views = corr.shape[0] * corr.shape[1] if n_tok else 0
    H, W = max(corr.shape[2], 1), max(corr.shape[3], 1)
    dev = corr.device
    need = int(lib().gc_index_workspace_bytes(n_tok))
    if workspace is None:
        workspace = _empty(stream, need, torch.uint8, dev)
    if workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace must hold at least {need} bytes")
    bits = _empty(stream, max(1, (n_tok + 31) // 32), torch.int32, dev)
    lst = _empty(stream, max(1, n_tok), torch.int32, dev)
    nv = _empty(stream, 1, torch.int32, dev)
    _check(lib().gc_index_correspondence(_dev(corr, "corr") if n_tok else None, n_views, H, W, a,
                                         _dev(bits, "vis_bits"), _dev(lst, "vis_list"), _dev(nv, "n_vis"),
                                         _dev(workspace, "workspace"),
                                         workspace.numel() * workspace.element_size(), _stream(stream)),
           "gc_index_correspondence")
    _keep(stream, (bits, lst))
    _after_side(stream)          # the count is read on the current stream
    return VisibleIndex(bits, lst, int(nv.item()))


def gc_index_correspondence_noalloc(corr: torch.Tensor, stream=None) -> VisibleIndex:
    """gc_index_correspondence with the library's own scratch instead of a
    workspace (the C call allocates nothing; this wrapper allocates the
    outputs).  Reads the visible count back to the host."""
    if corr.dtype != torch.int32 or corr.dim() != 5:
        raise ValueError("corr must be int32 [B, N-a, H, W, a]")
    a = corr.shape[-1]
    n_tok = int(corr.numel() // a) if a else 0
    n_views = corr.shape[0] * corr.shape[1] if n_tok else 0
    H, W = max(corr.shape[2], 1), max(corr.shape[3], 1)
    dev = corr.device
    bits = _empty(stream, max(1, (n_tok + 31) // 32), torch.int32, dev)
    lst = _empty(stream, max(1, n_tok), torch.int32, dev)
    nv = _empty(stream, 1, torch.int32, dev)
    _check(lib().gc_index_correspondence_noalloc(_dev(corr, "corr") if n_tok else None, n_views, H, W, a,
                                                 _dev(bits, "vis_bits"), _dev(lst, "vis_list"), _dev(nv, "n_vis"),
                                                 _stream(stream)), "gc_index_correspondence_noalloc")
    _keep(stream, (bits, lst))
    _after_side(stream)
    return VisibleIndex(bits, lst, int(nv.item()))


@dataclass
class ForegroundIndex:
    """Output of gc_index_foreground: fg_bits (int32 view of the uint32
    words), fg_recs (int32 [capacity, 4] records {token, x, y, z}) and the
    host count n_fg."""
    fg_bits: torch.Tensor
    fg_recs: torch.Tensor
    n_fg: int


def gc_index_foreground(pos: torch.Tensor, workspace: torch.Tensor = None, stream=None) -> ForegroundIndex:
    """Foreground index of position maps (float32 [..., H, W, 3], e.g.
    [B, N, H, W, 3]), once per asset batch; its records in tile order.  Reads
    the foreground count back to the host (one synchronisation)."""
    if pos.dtype != torch.float32 or pos.dim() < 3 or pos.shape[-1] != 3:
        raise ValueError("pos must be float32 [..., H, W, 3]")
    H, W = pos.shape[-3], pos.shape[-2]
    n_tok = int(pos.numel() // 3)
    n_views = n_tok // (H * W) if H * W else 0
    dev = pos.device
    need = int(lib().gc_index_workspace_bytes(n_tok))
    if workspace is None:
        workspace = _empty(stream, need, torch.uint8, dev)
    if workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace must hold at least {need} bytes")
    bits = _empty(stream, max(1, (n_tok + 31) // 32), torch.int32, dev)
    recs = _empty(stream, (max(1, n_tok), 4), torch.int32, dev)
    nf = _empty(stream, 1, torch.int32, dev)
    _check(lib().gc_index_foreground(_dev(pos, "pos") if n_tok else None, n_views, max(H, 1), max(W, 1),
                                     _dev(bits, "fg_bits"),
                                     _dev(recs, "fg_recs"), _dev(nf, "n_fg"), _dev(workspace, "workspace"),
                                     workspace.numel() * workspace.element_size(), _stream(stream)),
           "gc_index_foreground")
    _keep(stream, (bits, recs))
    _after_side(stream)          # the count is read on the current stream
    return ForegroundIndex(bits, recs, int(nf.item()))


def _fg_args(fg_index: Optional[ForegroundIndex]):
    if fg_index is None:
        return None, None, 0
    return _dev(fg_index.fg_bits, "fg_bits"), _dev(fg_index.fg_recs, "fg_recs"), int(fg_index.n_fg)


def _index_args(index: Optional[VisibleIndex]):
    if index is None:
        return None, None, 0
    return _dev(index.vis_bits, "vis_bits"), _dev(index.vis_list, "vis_list"), int(index.n_vis)


def _latent_shape(x0_prev: torch.Tensor):
    if x0_prev.dim() != 5:
        raise ValueError("latents must be [B, N, H, W, C]")
    return tuple(x0_prev.shape)


def gc_transport_step(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, corr: torch.Tensor,
                      weights: torch.Tensor, anchors: Sequence[int], x0_out: torch.Tensor = None,
                      index: VisibleIndex = None, stream=None) -> torch.Tensor:
    """Eq. 1 over one cached step; returns x0_out [B, N, H, W, C].  `index`
    (gc_index_correspondence of corr) selects the split launch."""
    B, N, H, W, C = _latent_shape(x0_prev)
    arr, a = _anchors(anchors)
    if tuple(x0_anchor_new.shape) != (B, a, H, W, C) or x0_anchor_new.dtype != x0_prev.dtype:
        raise ValueError(f"x0_anchor_new must be [B, a={a}, H, W, C] of the same dtype as x0_prev")
    K = weights.shape[-1]
    if x0_out is None:
        x0_out = _empty_like(stream, x0_prev)
    _check(lib().gc_transport_step(_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
                                   _dev(corr, "corr") if corr.numel() else None,
                                   _dev(weights, "weights") if weights.numel() else None, *_index_args(index),
                                   B, N, H, W, C, arr, a, K, dtype_code(x0_prev), _dev(x0_out, "x0_out"),
                                   _stream(stream)), "gc_transport_step")
    _keep(stream, (x0_out,))
    return x0_out


def gc_sampler_reconstruct(x_t: torch.Tensor, x0: torch.Tensor, sampler: Sampler, t: float, t_next: float,
                           x_next: torch.Tensor = None, model_out: torch.Tensor = None, stream=None):
    """Elementwise sampler step from x0; returns (x_next, model_out or None)."""
    if x0.shape != x_t.shape or x0.dtype != x_t.dtype:
        raise ValueError("x_t and x0 must have the same shape and dtype")
    if x_next is None:
        x_next = _empty_like(stream, x_t)
    if sampler.pred_out != GC_PRED_NONE and model_out is None:
        model_out = _empty_like(stream, x_t)
    smp = sampler.c()
    _check(lib().gc_sampler_reconstruct(_dev(x_t, "x_t"), _dev(x0, "x0"), _dev(x_next, "x_next"),
                                        _opt(model_out, "model_out"), x_t.numel(), dtype_code(x_t),
                                        ctypes.byref(smp), float(t), float(t_next), _stream(stream)),
           "gc_sampler_reconstruct")
    _keep(stream, [t for t in (x_next, model_out) if t is not None])
    return x_next, model_out


def gc_transport_reconstruct(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, corr: torch.Tensor,
                             weights: torch.Tensor, x_t: torch.Tensor, anchors: Sequence[int], sampler: Sampler,
                             t: float, t_next: float, x0_out: torch.Tensor = None, x_next: torch.Tensor = None,
                             model_out: torch.Tensor = None, index: VisibleIndex = None, stream=None):
    """Fused Eq. 1 + reconstruction; returns (x0_out, x_next, model_out or None).
    `index` (gc_index_correspondence of corr) selects the split launch."""
    B, N, H, W, C = _latent_shape(x0_prev)
    arr, a = _anchors(anchors)
    if tuple(x0_anchor_new.shape) != (B, a, H, W, C) or x0_anchor_new.dtype != x0_prev.dtype:
        raise ValueError(f"x0_anchor_new must be [B, a={a}, H, W, C] of the same dtype as x0_prev")
    if x_t.shape != x0_prev.shape or x_t.dtype != x0_prev.dtype:
        raise ValueError("x_t must match x0_prev in shape and dtype")
    K = weights.shape[-1]
    if x0_out is None:
        x0_out = _empty_like(stream, x0_prev)
    if x_next is None:
        x_next = _empty_like(stream, x_t)
    if sampler.pred_out != GC_PRED_NONE and model_out is None:
        model_out = _empty_like(stream, x_t)
    smp = sampler.c()
    _check(lib().gc_transport_reconstruct(_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
                                          _dev(corr, "corr") if corr.numel() else None,
                                          _dev(weights, "weights") if weights.numel() else None,
                                          *_index_args(index), _dev(x_t, "x_t"), B, N, H, W, C, arr, a, K,
                                          dtype_code(x0_prev),
                                          ctypes.byref(smp), float(t), float(t_next), _dev(x0_out, "x0_out"),
                                          _dev(x_next, "x_next"), _opt(model_out, "model_out"), _stream(stream)),
           "gc_transport_reconstruct")
    _keep(stream, [t for t in (x0_out, x_next, model_out) if t is not None])
    return x0_out, x_next, model_out


def _geom_inputs(x0_prev, x0_anchor_new, pos, cams, bbox, anchors):
    B, N, H, W, C = _latent_shape(x0_prev)
    arr, a = _anchors(anchors)
    if tuple(x0_anchor_new.shape) != (B, a, H, W, C) or x0_anchor_new.dtype != x0_prev.dtype:
        raise ValueError(f"x0_anchor_new must be [B, a={a}, H, W, C] of the same dtype as x0_prev")
    if pos.dtype != torch.float32 or tuple(pos.shape) != (B, N, H, W, 3):
        raise ValueError(f"pos must be float32 [B={B}, N={N}, H={H}, W={W}, 3]")
    if cams.dtype != torch.uint8 or tuple(cams.shape) != (B, N, 68):
        raise ValueError(f"cams must be uint8 [B={B}, N={N}, 68]")
    if bbox.dtype != torch.float32 or tuple(bbox.shape) != (B, 8):
        raise ValueError(f"bbox must be float32 [B={B}, 8]")
    return (B, N, H, W, C), arr, a


def gc_transport_step_geom(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, pos: torch.Tensor,
                           cams: torch.Tensor, bbox: torch.Tensor, anchors: Sequence[int], K: int,
                           x0_out: torch.Tensor = None, fg_index: ForegroundIndex = None, stream=None) -> torch.Tensor:
    """Eq. 1 with G_{A->v} computed on the fly from the position maps
    (pos float32 [B, N, H, W, 3], cams from camera_tensor, bbox from
    gc_posmap_bbox); equals gc_build_correspondence + gc_transport_step.
    `fg_index` (gc_index_foreground of pos) selects the foreground launch."""
    (B, N, H, W, C), arr, a = _geom_inputs(x0_prev, x0_anchor_new, pos, cams, bbox, anchors)
    if x0_out is None:
        x0_out = _empty_like(stream, x0_prev)
    fb, fr, nf = _fg_args(fg_index)
    _check(lib().gc_transport_step_geom(_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
                                        _dev(pos, "pos"), _dev(cams, "cams"), _dev(bbox, "bbox"), fb, fr, nf, B, N, H,
                                        W, C, arr, a, K, dtype_code(x0_prev), _dev(x0_out, "x0_out"),
                                        _stream(stream)),
           "gc_transport_step_geom")
    _keep(stream, (x0_out,))
    return x0_out


def gc_transport_reconstruct_geom(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, pos: torch.Tensor,
                                  cams: torch.Tensor, bbox: torch.Tensor, x_t: torch.Tensor, anchors: Sequence[int],
                                  K: int, sampler: Sampler, t: float, t_next: float, x0_out: torch.Tensor = None,
                                  x_next: torch.Tensor = None, model_out: torch.Tensor = None,
                                  fg_index: ForegroundIndex = None, stream=None):
    """gc_transport_reconstruct with G_{A->v} computed on the fly; returns
    (x0_out, x_next, model_out or None).  `fg_index` (gc_index_foreground of
    pos) selects the foreground launch."""
    (B, N, H, W, C), arr, a = _geom_inputs(x0_prev, x0_anchor_new, pos, cams, bbox, anchors)
    if x_t.shape != x0_prev.shape or x_t.dtype != x0_prev.dtype:
        raise ValueError("x_t must match x0_prev in shape and dtype")
    if x0_out is None:
        x0_out = _empty_like(stream, x0_prev)
    if x_next is None:
        x_next = _empty_like(stream, x_t)
    if sampler.pred_out != GC_PRED_NONE and model_out is None:
        model_out = _empty_like(stream, x_t)
    smp = sampler.c()
    fb, fr, nf = _fg_args(fg_index)
    _check(lib().gc_transport_reconstruct_geom(_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
                                               _dev(pos, "pos"), _dev(cams, "cams"), _dev(bbox, "bbox"), fb, fr, nf,
                                               _dev(x_t, "x_t"), B, N, H, W, C, arr, a, K, dtype_code(x0_prev),
                                               ctypes.byref(smp), float(t), float(t_next), _dev(x0_out, "x0_out"),
                                               _dev(x_next, "x_next"), _opt(model_out, "model_out"),
                                               _stream(stream)), "gc_transport_reconstruct_geom")
    _keep(stream, [t for t in (x0_out, x_next, model_out) if t is not None])
    return x0_out, x_next, model_out


class BoundCall:
    """A gc_transport_reconstruct call with every argument but (t, t_next)
    already marshalled: calling it issues exactly one ctypes call.  For
    step loops where per-call Python checks would cost more host time than
    the kernel takes on the GPU."""
    __slots__ = ("_fn", "_pre", "_post", "_smp", "keep")

    def __init__(self, fn, pre, smp, post, keep):
        self._fn, self._pre, self._smp, self._post, self.keep = fn, pre, smp, post, keep

    def __call__(self, t: float, t_next: float) -> None:
        rc = self._fn(*self._pre, ctypes.byref(self._smp), t, t_next, *self._post)
        if rc != GC_OK:
            _check(rc, "gc_transport_reconstruct")


def bind_transport_reconstruct(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, corr: torch.Tensor,
                               weights: torch.Tensor, x_t: torch.Tensor, anchors: Sequence[int], sampler: Sampler,
                               x0_out: torch.Tensor, x_next: torch.Tensor, model_out: torch.Tensor = None,
                               index: VisibleIndex = None, stream=None) -> BoundCall:
    """Marshal gc_transport_reconstruct's buffer arguments once (same checks
    as gc_transport_reconstruct); the returned object takes (t, t_next).
    The tensors must stay alive and unmoved while the object is used."""
    B, N, H, W, C = _latent_shape(x0_prev)
    arr, a = _anchors(anchors)
    if tuple(x0_anchor_new.shape) != (B, a, H, W, C) or x0_anchor_new.dtype != x0_prev.dtype:
        raise ValueError(f"x0_anchor_new must be [B, a={a}, H, W, C] of the same dtype as x0_prev")
    for name, t in (("x_t", x_t), ("x0_out", x0_out), ("x_next", x_next)):
        if t.shape != x0_prev.shape or t.dtype != x0_prev.dtype:
            raise ValueError(f"{name} must match x0_prev in shape and dtype")
    if (sampler.pred_out != GC_PRED_NONE) != (model_out is not None):
        raise ValueError("model_out must be given iff the sampler has a prediction output")
    K = weights.shape[-1]
    pre = (_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
           _dev(corr, "corr") if corr.numel() else None, _dev(weights, "weights") if weights.numel() else None,
           *_index_args(index), _dev(x_t, "x_t"), B, N, H, W, C, arr, a, K, dtype_code(x0_prev))
    post = (_dev(x0_out, "x0_out"), _dev(x_next, "x_next"), _opt(model_out, "model_out"), _stream(stream))
    return BoundCall(lib().gc_transport_reconstruct, pre, sampler.c(), post,
                     (x0_prev, x0_anchor_new, corr, weights, x_t, x0_out, x_next, model_out, arr, index))


def gc_unipc_coeffs(sampler: Sampler, S: int, k: int, order: int = 2, corrector: bool = True) -> UniPCStep:
    st = UniPCStep()
    smp = sampler.c()
    _check(lib().gc_unipc_coeffs(ctypes.byref(smp), S, k, order, int(corrector), ctypes.byref(st)),
           "gc_unipc_coeffs")
    return st


def gc_unipc_update(st: UniPCStep, m_k: torch.Tensor, x_cur: torch.Tensor = None, x_prev: torch.Tensor = None,
                    m_km2: torch.Tensor = None, m_km1: torch.Tensor = None, x_c: torch.Tensor = None,
                    x_next: torch.Tensor = None, stream=None):
    """UniPC update over all elements (a full step); returns (x_c, x_next)."""
    if x_c is None:
        x_c = _empty_like(stream, m_k)
    if x_next is None:
        x_next = _empty_like(stream, m_k)
    for name, t in (("x_cur", x_cur), ("x_prev", x_prev), ("m_km2", m_km2), ("m_km1", m_km1)):
        if t is not None and (t.shape != m_k.shape or t.dtype != m_k.dtype):
            raise ValueError(f"{name} must match m_k in shape and dtype")
    _check(lib().gc_unipc_update(_opt(x_cur, "x_cur"), _opt(x_prev, "x_prev"), _opt(m_km2, "m_km2"),
                                 _opt(m_km1, "m_km1"), _dev(m_k, "m_k"), m_k.numel(), dtype_code(m_k),
                                 ctypes.byref(st), _dev(x_c, "x_c"), _dev(x_next, "x_next"), _stream(stream)),
           "gc_unipc_update")
    _keep(stream, (x_c, x_next))
    return x_c, x_next


def gc_transport_unipc(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, corr: torch.Tensor,
                       weights: torch.Tensor, anchors: Sequence[int], st: UniPCStep, x_cur: torch.Tensor = None,
                       x_prev: torch.Tensor = None, m_km2: torch.Tensor = None, x0_out: torch.Tensor = None,
                       x_c: torch.Tensor = None, x_next: torch.Tensor = None, index: VisibleIndex = None,
                       stream=None):
    """Fused Eq. 1 + UniPC update; returns (x0_out, x_c, x_next)."""
    B, N, H, W, C = _latent_shape(x0_prev)
    arr, a = _anchors(anchors)
    if tuple(x0_anchor_new.shape) != (B, a, H, W, C) or x0_anchor_new.dtype != x0_prev.dtype:
        raise ValueError(f"x0_anchor_new must be [B, a={a}, H, W, C] of the same dtype as x0_prev")
    for name, t in (("x_cur", x_cur), ("x_prev", x_prev), ("m_km2", m_km2)):
        if t is not None and (t.shape != x0_prev.shape or t.dtype != x0_prev.dtype):
            raise ValueError(f"{name} must match x0_prev in shape and dtype")
    K = weights.shape[-1]
    x0_out = _empty_like(stream, x0_prev) if x0_out is None else x0_out
    x_c = _empty_like(stream, x0_prev) if x_c is None else x_c
    x_next = _empty_like(stream, x0_prev) if x_next is None else x_next
    _check(lib().gc_transport_unipc(_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
                                    _dev(corr, "corr") if corr.numel() else None,
                                    _dev(weights, "weights") if weights.numel() else None, *_index_args(index),
                                    _opt(x_cur, "x_cur"), _opt(x_prev, "x_prev"), _opt(m_km2, "m_km2"),
                                    B, N, H, W, C, arr, a, K, dtype_code(x0_prev), ctypes.byref(st),
                                    _dev(x0_out, "x0_out"), _dev(x_c, "x_c"), _dev(x_next, "x_next"),
                                    _stream(stream)), "gc_transport_unipc")
    _keep(stream, (x0_out, x_c, x_next))
    return x0_out, x_c, x_next


def gc_transport_unipc_geom(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, pos: torch.Tensor,
                            cams: torch.Tensor, bbox: torch.Tensor, anchors: Sequence[int], K: int, st: UniPCStep,
                            x_cur: torch.Tensor = None, x_prev: torch.Tensor = None, m_km2: torch.Tensor = None,
                            x0_out: torch.Tensor = None, x_c: torch.Tensor = None, x_next: torch.Tensor = None,
                            fg_index: ForegroundIndex = None, stream=None):
    """gc_transport_unipc with G_{A->v} computed on the fly; returns
    (x0_out, x_c, x_next).  `fg_index` (gc_index_foreground of pos) selects
    the foreground launch."""
    (B, N, H, W, C), arr, a = _geom_inputs(x0_prev, x0_anchor_new, pos, cams, bbox, anchors)
    for name, t in (("x_cur", x_cur), ("x_prev", x_prev), ("m_km2", m_km2)):
        if t is not None and (t.shape != x0_prev.shape or t.dtype != x0_prev.dtype):
            raise ValueError(f"{name} must match x0_prev in shape and dtype")
    x0_out = _empty_like(stream, x0_prev) if x0_out is None else x0_out
    x_c = _empty_like(stream, x0_prev) if x_c is None else x_c
    x_next = _empty_like(stream, x0_prev) if x_next is None else x_next
    fb, fr, nf = _fg_args(fg_index)
    _check(lib().gc_transport_unipc_geom(_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
                                         _dev(pos, "pos"), _dev(cams, "cams"), _dev(bbox, "bbox"), fb, fr, nf,
                                         _opt(x_cur, "x_cur"), _opt(x_prev, "x_prev"), _opt(m_km2, "m_km2"),
                                         B, N, H, W, C, arr, a, K, dtype_code(x0_prev), ctypes.byref(st),
                                         _dev(x0_out, "x0_out"), _dev(x_c, "x_c"), _dev(x_next, "x_next"),
                                         _stream(stream)), "gc_transport_unipc_geom")
    _keep(stream, (x0_out, x_c, x_next))
    return x0_out, x_c, x_next


class BoundUniPC:
    """A gc_transport_unipc call with its buffer arguments marshalled; the
    object takes the step's coefficients and issues exactly one ctypes call."""
    __slots__ = ("_fn", "_pre", "_post", "keep")

    def __init__(self, fn, pre, post, keep):
        self._fn, self._pre, self._post, self.keep = fn, pre, post, keep

    def __call__(self, st: UniPCStep) -> None:
        rc = self._fn(*self._pre, ctypes.byref(st), *self._post)
        if rc != GC_OK:
            _check(rc, "gc_transport_unipc")


def bind_transport_unipc(x0_prev: torch.Tensor, x0_anchor_new: torch.Tensor, corr: torch.Tensor,
                         weights: torch.Tensor, anchors: Sequence[int], x0_out: torch.Tensor, x_c: torch.Tensor,
                         x_next: torch.Tensor, x_cur: torch.Tensor = None, x_prev: torch.Tensor = None,
                         m_km2: torch.Tensor = None, index: VisibleIndex = None, stream=None) -> BoundUniPC:
    """Marshal gc_transport_unipc's buffer arguments once (same shape checks
    as gc_transport_unipc); the returned object takes a UniPCStep.  The
    tensors must stay alive and unmoved while the object is used."""
    B, N, H, W, C = _latent_shape(x0_prev)
    arr, a = _anchors(anchors)
    if tuple(x0_anchor_new.shape) != (B, a, H, W, C) or x0_anchor_new.dtype != x0_prev.dtype:
        raise ValueError(f"x0_anchor_new must be [B, a={a}, H, W, C] of the same dtype as x0_prev")
    for name, t in (("x_cur", x_cur), ("x_prev", x_prev), ("m_km2", m_km2), ("x0_out", x0_out), ("x_c", x_c),
                    ("x_next", x_next)):
        if t is not None and (t.shape != x0_prev.shape or t.dtype != x0_prev.dtype):
            raise ValueError(f"{name} must match x0_prev in shape and dtype")
    K = weights.shape[-1]
    pre = (_dev(x0_prev, "x0_prev"), _dev(x0_anchor_new, "x0_anchor_new"),
           _dev(corr, "corr") if corr.numel() else None, _dev(weights, "weights") if weights.numel() else None,
           *_index_args(index), _opt(x_cur, "x_cur"), _opt(x_prev, "x_prev"), _opt(m_km2, "m_km2"),
           B, N, H, W, C, arr, a, K, dtype_code(x0_prev))
    post = (_dev(x0_out, "x0_out"), _dev(x_c, "x_c"), _dev(x_next, "x_next"), _stream(stream))
    return BoundUniPC(lib().gc_transport_unipc, pre, post,
                      (x0_prev, x0_anchor_new, corr, weights, x_cur, x_prev, m_km2, x0_out, x_c, x_next, arr, index))


# --------------------------------------------------------------------------
# token staleness and the coverage-driven schedule
# --------------------------------------------------------------------------

def gc_coverage_pairs(pos: torch.Tensor, cams: torch.Tensor, bbox: torch.Tensor, out: torch.Tensor = None,
                      stream=None) -> torch.Tensor:
    """Single-anchor visibility bits: int32 [N, B, N, ceil(H*W/32)] (uint32
    words; bit p % 32 of word p / 32 of row (u, b, v): anchor u sees token p
    of view v)."""
    if pos.dtype != torch.float32 or pos.dim() != 5 or pos.shape[-1] != 3:
        raise ValueError("pos must be float32 [B, N, H, W, 3]")
    B, N, H, W, _ = pos.shape
    if cams.dtype != torch.uint8 or tuple(cams.shape) != (B, N, 68):
        raise ValueError(f"cams must be uint8 [B={B}, N={N}, 68]")
    wpr = (H * W + 31) // 32
    if out is None:
        out = _empty(stream, (N, B, N, wpr), torch.int32, pos.device)
    if tuple(out.shape) != (N, B, N, wpr) or out.element_size() != 4:
        raise ValueError(f"out must be a 32-bit [{N}, {B}, {N}, {wpr}] tensor")
    _check(lib().gc_coverage_pairs(_dev(pos, "pos"), _dev(cams, "cams"), _dev(bbox, "bbox"), B, N, H, W,
                                   _dev(out, "pair_bits"), _stream(stream)), "gc_coverage_pairs")
    _keep(stream, (out,))
    return out


def gc_coverage_init(pos: torch.Tensor, out: torch.Tensor = None, stream=None) -> torch.Tensor:
    """Staleness uint8 [B, N, H, W]: 0 for foreground tokens, 255 for background."""
    B, N, H, W, _ = pos.shape
    if out is None:
        out = _empty(stream, (B, N, H, W), torch.uint8, pos.device)
    _check(lib().gc_coverage_init(_dev(pos, "pos"), B, N, H, W, _dev(out, "stale"), _stream(stream)),
           "gc_coverage_init")
    _keep(stream, (out,))
    return out


def gc_coverage_update(pair_bits: torch.Tensor, stale: torch.Tensor, anchors: Sequence[int], R: int,
                       stats: torch.Tensor = None, stream=None) -> torch.Tensor:
    """One step with anchor set `anchors` (every view for a full step):
    staleness updated in place; returns stats int32 [B, N, 4] (foreground,
    staleness >= R, sum, max)."""
    if stale.dtype != torch.uint8 or stale.dim() != 4:
        raise ValueError("stale must be uint8 [B, N, H, W]")
    B, N, H, W = stale.shape
    arr = (ctypes.c_int32 * len(anchors))(*anchors)
    if stats is None:
        stats = _empty(stream, (B, N, 4), torch.int32, stale.device)
    if tuple(stats.shape) != (B, N, 4) or stats.element_size() != 4:
        raise ValueError(f"stats must be a 32-bit [{B}, {N}, 4] tensor")
    _check(lib().gc_coverage_update(_dev(pair_bits, "pair_bits"), B, N, H, W, arr, len(anchors), R,
                                    _dev(stale, "stale"), _dev(stats, "stats"), _stream(stream)),
           "gc_coverage_update")
    _keep(stream, (stats,))
    return stats


def gc_coverage_workspace_bytes() -> int:
    return int(lib().gc_coverage_workspace_bytes())


def gc_coverage_select(pair_bits: torch.Tensor, stale: torch.Tensor, a: int, forced: Sequence[int] = (),
                       out: torch.Tensor = None, workspace: torch.Tensor = None, stream=None) -> torch.Tensor:
    """Anchor set of the next cached step (greedy weighted maximum coverage):
    device int32 [a], ascending.  Enqueued only: read it after a sync."""
    B, N, H, W = stale.shape
    if out is None:
        out = _empty(stream, a, torch.int32, stale.device)
    if workspace is None:
        workspace = _empty(stream, gc_coverage_workspace_bytes(), torch.uint8, stale.device)
    farr = (ctypes.c_int32 * max(len(forced), 1))(*forced)
    _check(lib().gc_coverage_select(_dev(pair_bits, "pair_bits"), _dev(stale, "stale"), B, N, H, W, a, farr,
                                    len(forced), _dev(out, "anchors_out"), _dev(workspace, "workspace"),
                                    workspace.numel() * workspace.element_size(), _stream(stream)),
           "gc_coverage_select")
    _keep(stream, (out, workspace))
    return out


def gc_coverage_score(pair_bits: torch.Tensor, stale: torch.Tensor, sets: Sequence[Sequence[int]],
                      out: torch.Tensor = None, workspace: torch.Tensor = None, stream=None) -> torch.Tensor:
    """Weighted coverage of each candidate set: device int64 [M] (uint64 values)."""
    B, N, H, W = stale.shape
    M, a = len(sets), len(sets[0])
    if any(len(S) != a for S in sets):
        raise ValueError("candidate sets must have the same size")
    flat = (ctypes.c_int32 * (M * a))(*[int(u) for S in sets for u in S])
    if out is None:
        out = _empty(stream, M, torch.int64, stale.device)
    if workspace is None:
        workspace = _empty(stream, gc_coverage_workspace_bytes(), torch.uint8, stale.device)
    _check(lib().gc_coverage_score(_dev(pair_bits, "pair_bits"), _dev(stale, "stale"), B, N, H, W, flat, M, a,
                                   _dev(out, "scores"), _dev(workspace, "workspace"),
                                   workspace.numel() * workspace.element_size(), _stream(stream)),
           "gc_coverage_score")
    _keep(stream, (out, workspace))
    return out


def _stats_out(stale: torch.Tensor, stats: Optional[torch.Tensor], stream) -> torch.Tensor:
    B, N = stale.shape[:2]
    if stats is None:
        stats = _empty(stream, (B, N, 4), torch.int32, stale.device)
    if tuple(stats.shape) != (B, N, 4) or stats.element_size() != 4:
        raise ValueError(f"stats must be a 32-bit [{B}, {N}, 4] tensor")
    return stats


def gc_coverage_update_select(pair_bits: torch.Tensor, stale: torch.Tensor, anchors: Sequence[int], R: int,
                              a_next: int, forced: Sequence[int] = (), stats: torch.Tensor = None,
                              out: torch.Tensor = None, workspace: torch.Tensor = None, stream=None):
    """gc_coverage_update with `anchors`, then gc_coverage_select of `a_next`
    views on the updated staleness, in one pass over the tokens; returns
    (stats int32 [B, N, 4], selection device int32 [a_next])."""
    if stale.dtype != torch.uint8 or stale.dim() != 4:
        raise ValueError("stale must be uint8 [B, N, H, W]")
    B, N, H, W = stale.shape
    arr = (ctypes.c_int32 * len(anchors))(*anchors)
    stats = _stats_out(stale, stats, stream)
    if out is None:
        out = _empty(stream, a_next, torch.int32, stale.device)
    if workspace is None:
        workspace = _empty(stream, gc_coverage_workspace_bytes(), torch.uint8, stale.device)
    farr = (ctypes.c_int32 * max(len(forced), 1))(*forced)
    _check(lib().gc_coverage_update_select(_dev(pair_bits, "pair_bits"), B, N, H, W, arr, len(anchors), R,
                                           _dev(stale, "stale"), _dev(stats, "stats"), a_next, farr, len(forced),
                                           _dev(out, "anchors_out"), _dev(workspace, "workspace"),
                                           workspace.numel() * workspace.element_size(), _stream(stream)),
           "gc_coverage_update_select")
    _keep(stream, (stats, out, workspace))
    return stats, out


def gc_coverage_update_score(pair_bits: torch.Tensor, stale: torch.Tensor, anchors: Sequence[int], R: int,
                             sets: Sequence[Sequence[int]], stats: torch.Tensor = None, out: torch.Tensor = None,
                             workspace: torch.Tensor = None, stream=None):
    """gc_coverage_update with `anchors`, then gc_coverage_score of `sets` on
    the updated staleness, in one pass over the tokens; returns (stats int32
    [B, N, 4], scores device int64 [M])."""
    if stale.dtype != torch.uint8 or stale.dim() != 4:
        raise ValueError("stale must be uint8 [B, N, H, W]")
    B, N, H, W = stale.shape
    arr = (ctypes.c_int32 * len(anchors))(*anchors)
    M, a_set = len(sets), len(sets[0])
    if any(len(S) != a_set for S in sets):
        raise ValueError("candidate sets must have the same size")
    flat = (ctypes.c_int32 * (M * a_set))(*[int(u) for S in sets for u in S])
    stats = _stats_out(stale, stats, stream)
    if out is None:
        out = _empty(stream, M, torch.int64, stale.device)
    if workspace is None:
        workspace = _empty(stream, gc_coverage_workspace_bytes(), torch.uint8, stale.device)
    _check(lib().gc_coverage_update_score(_dev(pair_bits, "pair_bits"), B, N, H, W, arr, len(anchors), R,
                                          _dev(stale, "stale"), _dev(stats, "stats"), flat, M, a_set,
                                          _dev(out, "scores"), _dev(workspace, "workspace"),
                                          workspace.numel() * workspace.element_size(), _stream(stream)),
           "gc_coverage_update_score")
    _keep(stream, (stats, out, workspace))
    return stats, out


def gc_schedule_refresh_due(stats_host, tau: float) -> bool:
    """stats as returned by gc_coverage_update, on the host (numpy or CPU tensor)."""
    import numpy as np
    st = np.ascontiguousarray(stats_host.numpy() if isinstance(stats_host, torch.Tensor) else stats_host)
    if st.dtype.itemsize != 4 or st.ndim != 3 or st.shape[2] != 4:
        raise ValueError("stats must be 32-bit [B, N, 4]")
    due = ctypes.c_int()
    _check(lib().gc_schedule_refresh_due(st.ctypes.data, st.shape[0], st.shape[1], float(tau), ctypes.byref(due)),
           "gc_schedule_refresh_due")
    return bool(due.value)


def gc_schedule_forced_views(gap: Sequence[int], a: int, max_gap: int) -> List[int]:
    """Views whose anchor gap reached max_gap, longest gap first (ties: lower view), at most a."""
    N = len(gap)
    g = (ctypes.c_int32 * max(N, 1))(*[int(x) for x in gap])
    out = (ctypes.c_int32 * max(a, 1))()
    n = ctypes.c_int()
    _check(lib().gc_schedule_forced_views(g, N, a, max_gap, out, ctypes.byref(n)), "gc_schedule_forced_views")
    return list(out[:n.value])


def gc_schedule_advance_gaps(gap: Sequence[int], views: Sequence[int], full: bool) -> List[int]:
    """The anchor gaps after a step that predicted `views` (all views if full)."""
    g, N = _anchors(gap)
    arr, n = _anchors(views)
    _check(lib().gc_schedule_advance_gaps(g, N, arr, n, int(bool(full))), "gc_schedule_advance_gaps")
    return g[:N]


def gc_schedule_anchors(N: int, a: int, c: int) -> List[int]:
    out = (_I32[a] if 0 <= a <= GC_MAX_VIEWS else ctypes.c_int32 * a)()
    _check(lib().gc_schedule_anchors(N, a, c, out), "gc_schedule_anchors")
    return out[:a]


def gc_schedule_full_steps(rule: int, S: int, E: int = 0) -> List[int]:
    out = (ctypes.c_uint8 * S)()
    _check(lib().gc_schedule_full_steps(rule, S, E, out), "gc_schedule_full_steps")
    return list(out)


def gc_sampler_step_times(sampler: Sampler, S: int, k: int) -> Tuple[float, float]:
    t, tn = ctypes.c_double(), ctypes.c_double()
    smp = sampler.c()
    _check(lib().gc_sampler_step_times(ctypes.byref(smp), S, k, ctypes.byref(t), ctypes.byref(tn)),
           "gc_sampler_step_times")
    return t.value, tn.value


def gc_sampler_alpha_bar(sampler: Sampler, t: int) -> float:
    out = ctypes.c_double()
    smp = sampler.c()
    _check(lib().gc_sampler_alpha_bar(ctypes.byref(smp), int(t), ctypes.byref(out)), "gc_sampler_alpha_bar")
    return out.value


# ---------------------------------------------------------------------------
# operators of the denoiser's own blocks
# ---------------------------------------------------------------------------

_Tensor = torch.Tensor
_CONTIGUOUS = torch.contiguous_format
# GC_F32 / GC_BF16 by torch type
_HEAD_CODES = {torch.float32: GC_F32, torch.bfloat16: GC_BF16}
# (host array, columns, axes) of the position axes' columns, by their values
_SECTIONS: Dict[Tuple[int, ...], tuple] = {}


def _heads(t: torch.Tensor, name: str) -> _Heads:
    """gc_heads of a device tensor [tokens, heads, dim] whose channels are
    contiguous.  The stride of an axis of one element or none is of no
    consequence, and torch may hold any there."""
    if type(t) is not _Tensor and not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    strides = t.stride()
    if len(strides) != 3:
        raise ValueError(f"{name} must be [tokens, heads, dim] (got {tuple(t.shape)})")
    st, sh, sc = strides
    n, h, d = t.shape
    if sc != 1 and d > 1:
        raise ValueError(f"{name} must have contiguous channels")
    return _Heads(t.data_ptr(), st if n > 1 else h * d, sh if h > 1 else d)


def _head_code(t: torch.Tensor) -> int:
    code = _HEAD_CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"heads must be float32 or bfloat16 (got {t.dtype})")
    return code


def _like_heads(t: torch.Tensor, name: str, shape, like: torch.Tensor) -> torch.Tensor:
    if t.shape != shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name} must be {like.dtype} {list(shape)} on {like.device} (got {t.dtype} {list(t.shape)} "
                         f"on {t.device})")
    return t


def _sections(sections: Sequence[int]) -> tuple:
    key = tuple(map(int, sections))
    got = _SECTIONS.get(key)
    if got is None:
        if not 1 <= len(key) <= GC_MAX_AXES:
            raise ValueError(f"sections must name 1 to {GC_MAX_AXES} axes")
        if len(_SECTIONS) >= 256:
            _SECTIONS.clear()
        got = _SECTIONS[key] = (_I32[len(key)](*key), sum(key), len(key))
    return got


def _rope_args(positions: torch.Tensor, table: torch.Tensor, sections: Optional[Sequence[int]], x: torch.Tensor):
    """(positions, table, n_pos, sections, n_axes) as the C calls take them."""
    rows, cols, two = table.shape if table.dim() == 3 else (0, 0, 0)
    if two != 2 or table.dtype != torch.float32:
        raise ValueError("table must be float32 [n_pos, columns, 2]")
    sec, columns, axes = _sections((cols,) if sections is None else sections)
    if columns != cols:
        raise ValueError(f"sections {list(sec)} do not sum to the table's {cols} columns")
    T, shape = x.shape[0], positions.shape
    if positions.dtype != torch.int32 or not (shape == (T, axes) or (axes == 1 and shape == (T,))):
        raise ValueError(f"positions must be int32 [{T}, {axes}]")
    device = x.get_device()
    for t, name in ((positions, "positions"), (table, "table")):
        if t.get_device() != device:
            raise ValueError(f"{name} must be on {x.device} (got {t.device})")
    return _dev(positions, "positions"), _dev(table, "table"), rows, sec, axes


def gc_rope_table(n_pos: int, sections: Sequence[int], base: float = 10000.0, scaling: Optional[RopeScaling] = None,
                  table: torch.Tensor = None, device="cuda", stream=None) -> torch.Tensor:
    """float32 [n_pos, sum(sections), 2]: cos and sin of each position times
    each column's frequency.  sections: columns of each position axis."""
    sec, columns, axes = _sections(sections)
    if n_pos < 1:
        raise ValueError("n_pos must be at least 1")
    if table is None:
        table = _empty(stream, (n_pos, max(0, columns), 2), torch.float32, device)
    if table.dtype != torch.float32 or table.shape != (n_pos, columns, 2):
        raise ValueError(f"table must be float32 [{n_pos}, {columns}, 2]")
    _check(lib().gc_rope_table(_dev(table, "table"), n_pos, sec, axes, float(base),
                               ctypes.byref(scaling) if scaling is not None else None, _stream(stream)),
           "gc_rope_table")
    return table


def gc_rope(x: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, sections: Optional[Sequence[int]] = None,
            layout: int = GC_ROPE_HALF, out: torch.Tensor = None, stream=None) -> torch.Tensor:
    """Rotary positions on heads x [tokens, heads, dim] (float32 or bfloat16,
    any token and head strides of whole 16 bytes).  positions int32 [tokens]
    or [tokens, axes]; table from gc_rope_table; sections: its columns of each
    axis (default: one axis).  out may be x."""
    hx = _heads(x, "x")
    dt = _head_code(x)
    args = _rope_args(positions, table, sections, x)
    T, H, D = x.shape
    if out is None:
        out = _empty_like(stream, x)
        ho = _Heads(out.data_ptr(), H * D, D)
    else:
        ho = _heads(_like_heads(out, "out", x.shape, x), "out")
    _check(lib().gc_rope(hx, T, H, D, dt, *args, layout, ho, _stream(stream)), "gc_rope")
    return out


def gc_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, q_gain: torch.Tensor, k_gain: torch.Tensor,
                    positions: torch.Tensor, table: torch.Tensor, eps: float = 1e-6,
                    sections: Optional[Sequence[int]] = None, layout: int = GC_ROPE_HALF, q_out: torch.Tensor = None,
                    k_out: torch.Tensor = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """RMS norm of each head of q [tokens, heads, dim] and k [tokens,
    kv_heads, dim] with gains float32 [dim], and gc_rope, in one pass.  q_out
    and k_out may be q and k."""
    hq, hk = _heads(q, "q"), _heads(k, "k")
    dt = _head_code(q)
    T, H, D = q.shape
    Hk = k.shape[1]
    _like_heads(k, "k", (T, Hk, D), q)
    device = q.get_device()
    for g, name in ((q_gain, "q_gain"), (k_gain, "k_gain")):
        if g.dtype != torch.float32 or g.shape != (D,) or g.get_device() != device:
            raise ValueError(f"{name} must be float32 [{D}] on {q.device}")
    args = _rope_args(positions, table, sections, q)
    if q_out is None:
        q_out = _empty_like(stream, q)
        ho = _Heads(q_out.data_ptr(), H * D, D)
    else:
        ho = _heads(_like_heads(q_out, "q_out", q.shape, q), "q_out")
    if k_out is None:
        k_out = _empty_like(stream, k)
        hp = _Heads(k_out.data_ptr(), Hk * D, D)
    else:
        hp = _heads(_like_heads(k_out, "k_out", k.shape, q), "k_out")
    _check(lib().gc_qk_norm_rope(hq, H, hk, Hk, T, D, dt, _dev(q_gain, "q_gain"), _dev(k_gain, "k_gain"), eps, *args,
                                 layout, ho, hp, _stream(stream)), "gc_qk_norm_rope")
    return q_out, k_out


@dataclass
class AttentionPlan:
    """Output of gc_attention_plan: the sizes and the items on the device.
    Calls only read it, so calls in flight at the same time may share it."""
    info: AttentionInfo
    items: torch.Tensor

    def __post_init__(self):
        i = self.info
        self.sizes = (i.heads, i.kv_heads, i.dim, i.total_q, i.total_k)
        # handles of the streams after whose work torch's allocator reuses the items' memory
        self.known_streams = set()

    def used_on(self, handle: int, stream) -> None:
        """Calls on this stream read the items: their memory stays theirs
        until those are done, also where the plan is dropped before."""
        if stream is None:
            stream = torch.cuda.current_stream()
        elif not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(handle)
        self.items.record_stream(stream)
        self.known_streams.add(handle)

    def __getstate__(self):   # a copy's memory is another, known on no stream
        return {**self.__dict__, "known_streams": set()}


def gc_attention_plan(q_lens: Sequence[int], k_lens: Sequence[int], heads: int, kv_heads: int, dim: int,
                      dtype: torch.dtype, causal: bool = False, device="cuda", stream=None) -> AttentionPlan:
    """Work of attention over packed sequences of these lengths (host lists),
    for gc_attention: made once and kept while the lengths stay.  The items
    are copied on `stream` (default: torch's current stream)."""
    if len(q_lens) != len(k_lens):
        raise ValueError("q_lens and k_lens must have the same length")
    code = _HEAD_CODES.get(dtype)
    if code is None:
        raise ValueError(f"heads must be float32 or bfloat16 (got {dtype})")
    n = len(q_lens)
    ql = np.ascontiguousarray(q_lens, dtype=np.int64).reshape(n)
    kl = np.ascontiguousarray(k_lens, dtype=np.int64).reshape(n)
    if n and (ql.min() < 0 or kl.min() < 0 or ql.max() >= 1 << 31 or kl.max() >= 1 << 31):
        raise ValueError("lengths must lie in [0, 2^31)")
    ql, kl = ql.astype(np.int32), kl.astype(np.int32)
    info = AttentionInfo()
    args = (ql.ctypes.data_as(_i32p), kl.ctypes.data_as(_i32p), n, int(heads), int(kv_heads), int(dim), code,
            int(bool(causal)), ctypes.byref(info))
    host = np.empty(8192, np.int32)             # room for most plans; a longer one says how long
    rc = lib().gc_attention_plan(*args, host.ctypes.data_as(_i32p), host.size)
    words = info.n_items * GC_ATTENTION_ITEM_WORDS
    if rc == -6 and words > host.size:          # GC_ERR_CAPACITY
        host = np.empty(words, np.int32)
        rc = lib().gc_attention_plan(*args, host.ctypes.data_as(_i32p), host.size)
    _check(rc, "gc_attention_plan")
    host = host[:max(1, words)]
    s = _side_stream(stream)
    with torch.cuda.stream(s if s is not None else torch.cuda.current_stream()):
        plan = AttentionPlan(info, torch.from_numpy(host).to(device))
        if plan.items.is_cuda:
            plan.known_streams.add(torch.cuda.current_stream(plan.items.device).cuda_stream)
    return plan


def gc_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: AttentionPlan,
                 scale: Optional[float] = None, out: torch.Tensor = None, lse: torch.Tensor = None,
                 stream=None, workspace: torch.Tensor = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of q [sum of q_lens, heads, dim] over k, v [sum of k_lens,
    kv_heads, dim] with the plan of their lengths; scale defaults to
    1 / sqrt(dim).  Returns (out like q, lse float32 [heads, sum of q_lens]).
    workspace: plan.info.workspace_bytes for this call (allocated if None);
    calls in flight at the same time need one each."""
    info, need = plan.info, plan.info.workspace_bytes
    H, Hk, D, T, S = plan.sizes
    if q.shape != (T, H, D) or _head_code(q) != info.dtype:
        raise ValueError(f"q must be [{T}, {H}, {D}] of the plan's type (got {q.dtype} {list(q.shape)})")
    _like_heads(k, "k", (S, Hk, D), q)
    _like_heads(v, "v", (S, Hk, D), q)
    device = q.get_device()
    if plan.items.get_device() != device:
        raise ValueError(f"the plan is on {plan.items.device}, q on {q.device}")
    hq, hk, hv = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
    if out is None:
        out = _empty_like(stream, q)
        ho = _Heads(out.data_ptr(), H * D, D)
    else:
        ho = _heads(_like_heads(out, "out", q.shape, q), "out")
    if lse is None:
        lse = _empty(stream, (H, T), torch.float32, q.device)
    elif lse.dtype != torch.float32 or lse.shape != (H, T) or lse.get_device() != device:
        raise ValueError(f"lse must be float32 [{H}, {T}] on {q.device}")
    at, size = None, 0
    if need:
        if workspace is None:
            workspace = _empty(stream, need, torch.uint8, q.device)
        elif workspace.get_device() != device:
            raise ValueError(f"workspace must be on {q.device} (got {workspace.device})")
        at, size = _dev(workspace, "workspace"), workspace.numel() * workspace.element_size()
    handle = _stream(stream)
    if handle not in plan.known_streams:
        plan.used_on(handle, stream)
    _check(lib().gc_attention(hq, hk, hv, ho, _dev(lse, "lse"), info, plan.items.data_ptr(),
                              1.0 / math.sqrt(D) if scale is None else scale, at, size, handle), "gc_attention")
    return out, lse


# ---------------------------------------------------------------------------
# norms and matrix products of the denoiser's blocks
# ---------------------------------------------------------------------------

# codes by torch type
_ROW_CODES = {torch.float32: GC_F32, torch.bfloat16: GC_BF16, torch.float8_e4m3fn: GC_E4M3}
_INT_MAX = 2 ** 31 - 1


def _rows(t: torch.Tensor, name: str) -> _Rows:
    """gc_rows of a device tensor [rows, columns] whose columns are contiguous.
    The stride of an axis of one element or none is of no consequence."""
    if type(t) is not _Tensor and not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    strides = t.stride()
    if len(strides) != 2:
        raise ValueError(f"{name} must be [rows, columns] (got {tuple(t.shape)})")
    n, c = t.shape
    if strides[1] != 1 and c > 1:
        raise ValueError(f"{name} must have contiguous columns")
    if n > _INT_MAX or c > _INT_MAX:      # (ctypes would pass what is left of them in 32 bits)
        raise ValueError(f"{name} has a size above 2^31 - 1 (got {tuple(t.shape)})")
    return _Rows(t.data_ptr(), strides[0] if n > 1 else c)


def _device_of(x: torch.Tensor, stream) -> Tuple[int, int]:
    """(device of a call's tensors, handle of its stream), which must be on
    that device."""
    device = x.get_device()
    if stream is None and _RAW_STREAM is not None:
        at = _GET_DEVICE()
        handle = _RAW_STREAM(at)
    else:
        at = stream.device_index if isinstance(stream, torch.cuda.Stream) else torch.cuda.current_device()
        handle = _stream(stream)
    if device != at:
        raise ValueError(f"tensors are on cuda:{device}, the stream is on cuda:{at}")
    return device, handle


def _like_rows(t: torch.Tensor, name: str, shape, dtype: torch.dtype, device: int) -> _Rows:
    if t.dtype != dtype or t.shape != shape or t.get_device() != device:
        raise ValueError(f"{name} must be {dtype} {list(shape)} on cuda:{device} (got {t.dtype} {list(t.shape)} on "
                         f"{t.device})")
    return _rows(t, name)


def _floats(t: Optional[torch.Tensor], name: str, n: int, device: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (n,) or t.get_device() != device:
        raise ValueError(f"{name} must be float32 [{n}] on cuda:{device} (got {t.dtype} {list(t.shape)} on {t.device})")
    return _dev(t, name)


def gc_add_rms_norm(x: torch.Tensor, residual: torch.Tensor = None, gain: torch.Tensor = None, eps: float = 1e-6,
                    out_dtype: torch.dtype = None, total: torch.Tensor = None, out: torch.Tensor = None,
                    out_scale: torch.Tensor = None,
                    stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """RMS norm of rows x + residual (float32 or bfloat16 [rows, width], any
    strides of the rows) with a gain float32 [width], in the rows' type or as
    torch.float8_e4m3fn with a float32 scale for each row.  Returns (out, its
    scales or None, the sum; x itself without a residual).  total and out may
    be x or residual."""
    hx = _rows(x, "x")
    code = _HEAD_CODES.get(x.dtype)
    if code is None:
        raise ValueError(f"rows must be float32 or bfloat16 (got {x.dtype})")
    n, width = shape = x.shape
    device, handle = _device_of(x, stream)
    if out_dtype is None:
        out_dtype = x.dtype if out is None else out.dtype
    out_code = _ROW_CODES.get(out_dtype)
    if out_code is None:
        raise ValueError(f"out_dtype must be {x.dtype} or {torch.float8_e4m3fn} (got {out_dtype})")
    hr = ht = None
    if residual is not None:
        hr = _like_rows(residual, "residual", shape, x.dtype, device)
        if total is None:
            total = _empty_like(stream, x)
            ht = _Rows(total.data_ptr(), width)
    if total is not None and ht is None:
        ht = _like_rows(total, "total", shape, x.dtype, device)
    if out is None:
        out = _empty_like(stream, x, out_dtype)
        ho = _Rows(out.data_ptr(), width)
    else:
        ho = _like_rows(out, "out", shape, out_dtype, device)
    if out_code == GC_E4M3 and out_scale is None:
        out_scale = _empty(stream, (n,), torch.float32, x.device)
        scale_at = out_scale.data_ptr()
    else:
        scale_at = _floats(out_scale, "out_scale", n, device)
    _check(lib().gc_add_rms_norm(hx, hr, n, width, code, None if gain is None else _floats(gain, "gain", width, device), eps, ht, ho, out_code,
                                 scale_at, handle), "gc_add_rms_norm")
    return out, out_scale, x if total is None else total


def gc_quantize_rows(x: torch.Tensor, out: torch.Tensor = None, out_scale: torch.Tensor = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows x (float32 or bfloat16 [rows, width], any stride of the rows) as
    torch.float8_e4m3fn with a float32 scale for each: (out, out_scale)."""
    hx = _rows(x, "x")
    code = _HEAD_CODES.get(x.dtype)
    if code is None:
        raise ValueError(f"rows must be float32 or bfloat16 (got {x.dtype})")
    n, width = shape = x.shape
    device, handle = _device_of(x, stream)
    if out is None:
        out = _empty_like(stream, x, torch.float8_e4m3fn)
        ho = _Rows(out.data_ptr(), width)
    else:
        ho = _like_rows(out, "out", shape, torch.float8_e4m3fn, device)
    if out_scale is None:
        out_scale = _empty(stream, (n,), torch.float32, x.device)
        scale_at = out_scale.data_ptr()
    else:
        scale_at = _floats(out_scale, "out_scale", n, device)
    _check(lib().gc_quantize_rows(hx, n, width, code, ho, scale_at, handle), "gc_quantize_rows")
    return out, out_scale


def gc_linear_workspace_bytes(n_rows: int, n_out: int, n_in: int, dtype: torch.dtype, gated: bool = False) -> int:
    """Bytes of device memory that gc_linear needs beside its arguments."""
    if max(n_rows, n_out, n_in) > _INT_MAX or min(n_rows, n_out, n_in) < 0:
        raise ValueError(f"sizes must be in [0, 2^31 - 1] (got {n_rows}, {n_out}, {n_in})")
    need = lib().gc_linear_workspace_bytes(n_rows, n_out, n_in, _ROW_CODES.get(dtype, -1), int(bool(gated)))
    if need < 0:
        _check(-2, "gc_linear_workspace_bytes")
    return need


def gc_linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor = None, act: int = GC_ACT_NONE, gated: bool = False,
              residual: torch.Tensor = None, x_scale: torch.Tensor = None, w_scale: torch.Tensor = None,
              out_dtype: torch.dtype = None, out: torch.Tensor = None, stream=None,
              workspace: torch.Tensor = None) -> torch.Tensor:
    """act(x w^T + bias) + residual for x [rows, n_in] and w [n_out, n_in] of
    one type: float32, bfloat16, or torch.float8_e4m3fn with a float32 scale
    for each row of x and of w.  gated: w and bias have 2 n_out rows, and the
    result is act(p of the first n_out) * p of the others + residual.  The
    result is of out_dtype (default: out's or residual's type, else x's,
    bfloat16 for 8-bit operands): float32 with any operands, bfloat16 with
    bfloat16 and 8-bit ones.  out may be residual.
    workspace: gc_linear_workspace_bytes for this call (allocated if None)."""
    hx, hw = _rows(x, "x"), _rows(w, "w")
    code = _ROW_CODES.get(x.dtype)
    if code is None:
        raise ValueError(f"x must be float32, bfloat16 or {torch.float8_e4m3fn} (got {x.dtype})")
    n, n_in = x.shape
    w_rows = w.shape[0]
    device, handle = _device_of(x, stream)
    if w.dtype != x.dtype or w.shape[1] != n_in or w.get_device() != device:
        raise ValueError(f"w must be {x.dtype} [n_out, {n_in}] on {x.device} (got {w.dtype} {list(w.shape)} on {w.device})")
    n_out, gated = w_rows, int(bool(gated))
    if gated:
        if w_rows % 2:
            raise ValueError(f"gated products need an even number of rows of w (got {w_rows})")
        n_out = w_rows // 2
    if out_dtype is None:
        out_dtype = (out.dtype if out is not None else residual.dtype if residual is not None else
                     torch.bfloat16 if code == GC_E4M3 else x.dtype)
    out_code = _ROW_CODES.get(out_dtype)
    if out_code is None:
        raise ValueError(f"out_dtype must be float32 or bfloat16 (got {out_dtype})")
    if out is None:
        out = x.new_empty((n, n_out), dtype=out_dtype) if stream is None else _empty(stream, (n, n_out), out_dtype, x.device)
        ho = _Rows(out.data_ptr(), n_out)
    else:
        ho = _like_rows(out, "out", (n, n_out), out_dtype, device)
    hr = None if residual is None else _like_rows(residual, "residual", (n, n_out), out_dtype, device)
    at, size = None, 0
    need = lib().gc_linear_workspace_bytes(n, n_out, n_in, code, gated)
    if need > 0:
        if workspace is None:
            workspace = _empty(stream, need, torch.uint8, x.device)
        elif workspace.get_device() != device:
            raise ValueError(f"workspace must be on {x.device} (got {workspace.device})")
        at, size = _dev(workspace, "workspace"), workspace.numel() * workspace.element_size()
    _check(lib().gc_linear(hx, None if x_scale is None else _floats(x_scale, "x_scale", n, device), hw,
                           None if w_scale is None else _floats(w_scale, "w_scale", w_rows, device), n, n_out, n_in, code,
                           None if bias is None else _floats(bias, "bias", w_rows, device), act, gated, hr, ho, out_code,
                           at, size, handle), "gc_linear")
    return out


lib()
