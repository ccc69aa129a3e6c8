"""Incremental ViT encoding on GB300: Python binding of the C ABI in ``include/ivit.h``.

The functions below carry the C entry points' names and only marshal arguments
(torch tensors -> raw pointers, torch streams -> cudaStream_t); every step of the
encode runs in the CUDA library ``_build/libivit.so``.  There is no fallback: if the
library is missing, loading fails with an error that says how to build it.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

import numpy as np

from . import synth

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libivit.so")

IVIT_OK = 0
IVIT_ERR_ARG = -1
IVIT_ERR_SHAPE = -2
IVIT_ERR_OOM = -3
IVIT_ERR_CUDA = -4
IVIT_ERR_DEVICE = -5

EXPORTED = [
    "ivit_weights_size", "ivit_create", "ivit_encode_full", "ivit_encode_incremental",
    "ivit_get_changed", "ivit_get_cache", "ivit_reset", "ivit_timeline",
    "ivit_timeline_read", "ivit_device_status", "ivit_last_launch_count", "ivit_destroy",
    "ivit_last_error", "ivit_select_noalloc", "ivit_action_combine", "ivit_step_plan",
    "ivit_qk_norm_rope", "ivit_qk_norm_rope_backward_workspace", "ivit_qk_norm_rope_backward",
    "ivit_tree_attention_workspace", "ivit_tree_attention", "ivit_kv_write",
]
IVIT_NOALLOC_MAX_TOKENS = 65536
IVIT_BF16 = 0
IVIT_FP16 = 1


class IvitConfig(C.Structure):
    _fields_ = [
        ("img_h", C.c_int32), ("img_w", C.c_int32), ("patch", C.c_int32),
        ("dim", C.c_int32), ("depth", C.c_int32), ("heads", C.c_int32),
        ("mlp_dim", C.c_int32), ("n_streams", C.c_int32), ("n_views", C.c_int32),
        ("ln_eps", C.c_float), ("gelu", C.c_int32), ("select_mode", C.c_int32),
        ("threshold", C.c_float), ("topk", C.c_int32), ("ref_mode", C.c_int32),
        ("score_source", C.c_int32), ("schedule", C.c_int32), ("mlp_tokens", C.c_int32),
    ]


class IvitCacheLayout(C.Structure):
    """Layout of a paged key (or value) cache of one layer; build it with ``make_cache_layout``."""
    _fields_ = [
        ("n_pages", C.c_int32), ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("dtype", C.c_int32), ("reserved", C.c_int32), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
        ("head_stride", C.c_int64),
    ]


class IvitPlanConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_req", "max_rows", "max_pages", "page_size", "n_pages", "mask_words")]


class IvitRopeConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("heads", "kv_heads", "head_dim", "rot_dim", "n_axes", "interleaved", "dtype")]
    _fields_.append(("eps", C.c_float))


class IvitAttentionConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_req", "heads", "max_pages", "max_new", "mask_mode", "mask_words")]
    _fields_.append(("scale", C.c_float))


class IvitError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ivit error {code}: {msg}")
        self.code = code


_lib: Optional[C.CDLL] = None


def load(path: str = LIB_PATH) -> C.CDLL:
    """Loads the CUDA library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'`")
    L = C.CDLL(path)
    P, I, I64 = C.c_void_p, C.c_int, C.c_int64
    L.ivit_weights_size.restype = C.c_size_t
    L.ivit_weights_size.argtypes = [C.POINTER(IvitConfig)]
    L.ivit_create.argtypes = [C.POINTER(IvitConfig), P, C.POINTER(P)]
    L.ivit_encode_full.argtypes = [P, P, P, P]
    L.ivit_encode_incremental.argtypes = [P, P, P, P, P]
    L.ivit_get_changed.argtypes = [P, I, P, P, P]
    L.ivit_get_cache.argtypes = [P, I, I, P, P]
    L.ivit_reset.argtypes = [P, I]
    L.ivit_timeline.argtypes = [P, I]
    L.ivit_timeline_read.argtypes = [P, P, C.POINTER(C.c_double), C.POINTER(I64), C.POINTER(C.c_double),
                                     C.POINTER(C.c_double)]
    L.ivit_device_status.argtypes = [P, P]
    L.ivit_last_launch_count.restype = I64
    L.ivit_last_launch_count.argtypes = [P]
    L.ivit_destroy.argtypes = [P]
    L.ivit_destroy.restype = None
    L.ivit_last_error.restype = C.c_char_p
    L.ivit_last_error.argtypes = [P]
    L.ivit_action_combine.argtypes = [P, P, P, P, P, P, C.c_int32, C.c_int32, P, P]
    L.ivit_select_noalloc.argtypes = [P, P, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                      C.c_float, C.c_int32, P, P, P]
    I32 = C.c_int32
    L.ivit_step_plan.argtypes = [P] * 16
    L.ivit_qk_norm_rope.argtypes = [P, I32, P, I64, P, I64, P, I64, P, P, P, I64, P, P, P, I64, P, I64, P, P, P, P, P]
    L.ivit_qk_norm_rope_backward_workspace.restype = C.c_size_t
    L.ivit_qk_norm_rope_backward_workspace.argtypes = [P]
    L.ivit_qk_norm_rope_backward.argtypes = [P, I32, P, I64, P, I64, P, I64, P, I64, P, P, P, I64, P, P, P, I64, P, I64, P,
                                             P, P, C.c_size_t, P]
    L.ivit_tree_attention_workspace.restype = C.c_size_t
    L.ivit_tree_attention_workspace.argtypes = [P, P]
    L.ivit_tree_attention.argtypes = [P, P, I32, P, I64, P, I64, P, I64, P, P, P, P, P, P, P, I64, P, P, C.c_size_t, P]
    L.ivit_kv_write.argtypes = [P, I32, I32, I32, P, P, I64, I64, P, P, P, P, I64, P]
    _lib = L
    return L


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if type(t) is _dtypes.get("tensor"):
        return t.data_ptr()
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


_dtypes = {}  # torch dtypes by name, and torch.Tensor: filled on the first check (torch is imported late)
_Tensor = _Int32 = None  # torch.Tensor and torch.int32 from then on


def _tensor_type():
    global _Tensor, _Int32
    t = _dtypes.get("tensor")
    if t is None:
        import torch
        for name in ("uint8", "int32", "float32", "bfloat16", "float16"):
            _dtypes[name] = getattr(torch, name)
        _dtypes[IVIT_BF16], _dtypes[IVIT_FP16] = torch.bfloat16, torch.float16  # (by the library's codes, too)
        _Int32 = torch.int32
        t = _Tensor = _dtypes["tensor"] = torch.Tensor
    return t


def _require(t, name: str, dtype_name: str, numel: int) -> None:
    """Rejects a tensor that the kernels would misread or index out of bounds: one in host
    memory, of another dtype (``dtype_name`` is the torch dtype's name, e.g. "uint8"), a
    non-contiguous view, or one with fewer than ``numel`` elements.  ``None`` (an optional
    output) and raw integer pointers pass unchecked: the caller vouches for those."""
    if t is None or isinstance(t, int):
        return
    # the common case: the checks below without formatting names
    if (type(t) is _tensor_type() and t.is_cuda and t.dtype is _dtypes[dtype_name] and t.is_contiguous()
            and t.numel() >= numel):
        return
    if isinstance(t, np.ndarray):
        raise TypeError(f"{name}: a numpy array (host memory); a CUDA tensor is required")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: tensor on {t.device}; a CUDA tensor is required")
    if str(t.dtype) != "torch." + dtype_name:
        raise TypeError(f"{name}: dtype {t.dtype}, expected torch.{dtype_name}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: not contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, the call needs {numel}")


# handle -> (views, frame bytes per view, tokens per view, width), registered at create so
# that the entry points can check the tensors they are given against the encoder's sizes
_dims = {}


_current = []  # torch's raw stream and device lookups, once the first call has found them


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _current:  # (without building a Stream object)
            return _current[0](_current[1]())
        import torch
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        stream = torch.cuda.current_stream().cuda_stream
        if raw and device and raw(device()) == stream:
            _current.extend((raw, device))
        return stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_config(shape: "synth.EncoderShape", n_streams: int = 1, n_views: int = 1,
                select_mode: int = synth.SEL_THRESHOLD, threshold: float = 0.98, topk: int = 0,
                ref_mode: int = synth.REF_PREV_FRAME, score_source: int = synth.SCORE_EMBED,
                schedule: int = synth.SCHED_INCREMENTAL, mlp_tokens: int = 0) -> IvitConfig:
    return IvitConfig(shape.img_h, shape.img_w, shape.patch, shape.dim, shape.depth, shape.heads,
                      shape.mlp_dim, n_streams, n_views, shape.ln_eps, shape.gelu, select_mode,
                      threshold, topk, ref_mode, score_source, schedule, mlp_tokens)


# ------------------------------------------------------------- C entry points

def ivit_weights_size(cfg: IvitConfig) -> int:
    return int(load().ivit_weights_size(C.byref(cfg)))


def ivit_last_error(handle: Optional[int] = None) -> str:
    return load().ivit_last_error(handle).decode(errors="replace")


def _check(code: int, handle: Optional[int]) -> int:
    if code < 0:
        raise IvitError(code, ivit_last_error(handle))
    return code


def ivit_create(cfg: IvitConfig, weights_u16: np.ndarray) -> int:
    w = np.ascontiguousarray(weights_u16, dtype=np.uint16)
    h = C.c_void_p()
    _check(load().ivit_create(C.byref(cfg), w.ctypes.data, C.byref(h)), None)
    n_tok = (cfg.img_h // cfg.patch) * (cfg.img_w // cfg.patch)
    _dims[h.value] = (cfg.n_streams * cfg.n_views, cfg.img_h * cfg.img_w * 3, n_tok, cfg.dim)
    return h.value


def _check_call(h: int, frames, tokens_out, changed_count=None) -> None:
    if h not in _dims:
        return  # a handle created outside this module: sizes unknown here
    sv, fbytes, n_tok, dim = _dims[h]
    _require(frames, "frames", "uint8", sv * fbytes)
    _require(tokens_out, "tokens_out", "bfloat16", sv * n_tok * dim)
    _require(changed_count, "changed_count", "int32", sv)


def ivit_encode_full(h: int, frames, tokens_out=None, stream=None) -> None:
    _check_call(h, frames, tokens_out)
    _check(load().ivit_encode_full(h, _ptr(frames), _ptr(tokens_out), _stream(stream)), h)


def ivit_encode_incremental(h: int, frames, tokens_out=None, changed_count=None,
                            stream=None) -> None:
    _check_call(h, frames, tokens_out, changed_count)
    _check(load().ivit_encode_incremental(h, _ptr(frames), _ptr(tokens_out),
                                          _ptr(changed_count), _stream(stream)), h)


def ivit_get_changed(h: int, sv: int, idx_out=None, count_out=None, stream=None) -> None:
    _check(load().ivit_get_changed(h, sv, _ptr(idx_out), _ptr(count_out), _stream(stream)), h)


def ivit_get_cache(h: int, which: int, layer: int, dst, stream=None) -> None:
    _check(load().ivit_get_cache(h, which, layer, _ptr(dst), _stream(stream)), h)


def ivit_reset(h: int, stream_index: int = -1) -> None:
    _check(load().ivit_reset(h, stream_index), h)


def ivit_timeline(h: int, enable: bool) -> None:
    """Timeline mode on or off (the encoder's CUDA graphs are captured again)."""
    _check(load().ivit_timeline(h, int(bool(enable))), h)


TIMELINE_FAMILIES = ("gemm", "attention", "layernorm", "other")


def ivit_timeline_read(h: int, stream=None) -> dict:
    """Per-family kernel time (ms) and launches of the last call, the GEMM launches'
    algorithmic bytes and the call's kernel span (ms); synchronises the stream."""
    ms = (C.c_double * 4)()
    n = (C.c_int64 * 4)()
    b = C.c_double()
    span = C.c_double()
    _check(load().ivit_timeline_read(h, _stream(stream), ms, n, C.byref(b), C.byref(span)), h)
    return {"ms": dict(zip(TIMELINE_FAMILIES, list(ms))), "launches": dict(zip(TIMELINE_FAMILIES, list(n))),
            "gemm_bytes": b.value, "span_ms": span.value}


def ivit_device_status(h: int, stream=None) -> int:
    return _check(load().ivit_device_status(h, _stream(stream)), h)


def ivit_last_launch_count(h: int) -> int:
    return int(load().ivit_last_launch_count(h))


def ivit_destroy(h: int) -> None:
    _dims.pop(h, None)
    load().ivit_destroy(h)


def ivit_select_noalloc(e_cur, e_ref, n_views: int, n_tok: int, dim: int, select_mode: int,
                        threshold: float, topk: int, idx_out, counts_out, stream=None) -> None:
    """Selection without device allocation (scratch in a fixed device array); for callers
    that cannot allocate, e.g. while a stream is being captured into a CUDA graph."""
    if 0 < n_views * n_tok <= IVIT_NOALLOC_MAX_TOKENS and dim > 0:
        # (other sizes are rejected by the library before any device work)
        _require(e_cur, "e_cur", "float32", n_views * n_tok * dim)
        _require(e_ref, "e_ref", "float32", n_views * n_tok * dim)
        _require(idx_out, "idx_out", "int32", n_views * n_tok)
        _require(counts_out, "counts_out", "int32", n_views)
    _check(load().ivit_select_noalloc(_ptr(e_cur), _ptr(e_ref), n_views, n_tok, dim, select_mode,
                                      threshold, topk, _ptr(idx_out), _ptr(counts_out),
                                      _stream(stream)), None)


def ivit_action_combine(x0, v0, v7, alpha, beta, b, xT, stream=None) -> None:
    """Eq. 9 action combine on device tensors: x0, v0, v7, b (or None), xT fp32 [B, A];
    alpha, beta fp32 [B]."""
    if x0.dim() != 2:
        raise ValueError(f"x0: shape {tuple(x0.shape)}, expected [batch, action width]")
    B, A = x0.shape
    n = B * A
    _require(x0, "x0", "float32", n)
    _require(v0, "v0", "float32", n)
    _require(v7, "v7", "float32", n)
    _require(b, "b", "float32", n)
    _require(xT, "xT", "float32", n)
    _require(alpha, "alpha", "float32", B)
    _require(beta, "beta", "float32", B)
    _check(load().ivit_action_combine(_ptr(x0), _ptr(v0), _ptr(v7), _ptr(alpha), _ptr(beta), _ptr(b), B, A,
                                      _ptr(xT), _stream(stream)), None)


# ------------------------------------------------------- language backbone

IVIT_MASK_CAUSAL = 0
IVIT_MASK_ALL = 1
IVIT_MASK_TREE = 2
_DTYPES = {"bfloat16": IVIT_BF16, "float16": IVIT_FP16}
_DTYPE_NAMES = {v: k for k, v in _DTYPES.items()}
_MASKS = {"causal": IVIT_MASK_CAUSAL, "all": IVIT_MASK_ALL, "tree": IVIT_MASK_TREE}


def _dtype_code(dtype) -> int:
    name = str(dtype).replace("torch.", "")
    if name not in _DTYPES:
        raise TypeError(f"dtype {dtype}: bfloat16 or float16 is required")
    return _DTYPES[name]


def make_cache_layout(cache) -> IvitCacheLayout:
    """Layout of a paged cache given as a tensor [pages, page_size, kv_heads, head_dim] (any strides with
    contiguous heads, so a [pages, kv_heads, page_size, head_dim] array transposed will do)."""
    if len(cache.shape) != 4:
        raise ValueError(f"cache: shape {tuple(cache.shape)}, expected [pages, page_size, kv_heads, head_dim]")
    st = cache.stride()
    if st[3] != 1:
        raise ValueError("cache: the values of a head are not contiguous")
    lay = IvitCacheLayout(*cache.shape, _dtype_code(cache.dtype), 0, st[0], st[1], st[2])
    lay.shape, lay.strides = tuple(cache.shape), tuple(st)
    return lay


def make_plan_config(n_req: int, max_rows: int, max_pages: int, page_size: int, n_pages: int,
                     mask_words: int = 0) -> IvitPlanConfig:
    return IvitPlanConfig(n_req, max_rows, max_pages, page_size, n_pages, mask_words)


def make_rope_config(heads: int, kv_heads: int, head_dim: int, rot_dim: Optional[int] = None, n_axes: int = 1,
                     interleaved: bool = False, eps: float = 1e-6, dtype="bfloat16") -> IvitRopeConfig:
    return IvitRopeConfig(heads, kv_heads, head_dim, head_dim if rot_dim is None else rot_dim, n_axes,
                          int(interleaved), _dtype_code(dtype), eps)


def make_attention_config(n_req: int, heads: int, max_pages: int, max_new: int, mask="causal", mask_words: int = 0,
                          scale: float = 1.0) -> IvitAttentionConfig:
    """``mask``: "causal", "all" or "tree" (with ``mask_words`` 32-bit words a row)."""
    return IvitAttentionConfig(n_req, heads, max_pages, max_new, _MASKS.get(mask, mask), mask_words, scale)


def _arg(t, name: str, dtype_name: str, numel: int) -> Optional[int]:
    """``_require``, and the pointer."""
    if type(t) is _Tensor and t.is_cuda and t.dtype is _dtypes[dtype_name] and t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    _require(t, name, dtype_name, numel)
    return _ptr(t)


def _i32(t, name: str, numel: int) -> Optional[int]:
    """``_arg`` of an int32 array, which most are."""
    if type(t) is _Tensor and t.is_cuda and t.dtype is _Int32 and t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    if t is None:
        return None
    return _arg(t, name, "int32", numel)


def _typed(t, name: str, dtype: int) -> None:
    """Rejects what is not a device tensor of the type ``dtype`` (IVIT_BF16 or IVIT_FP16)."""
    if type(t) is _Tensor and t.is_cuda and t.dtype is _dtypes[dtype]:
        return
    if isinstance(t, (int, np.ndarray)) or t is None:
        raise TypeError(f"{name}: a CUDA tensor is required")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: tensor on {t.device}; a CUDA tensor is required")
    _tensor_type()
    if t.dtype is not _dtypes[dtype]:
        raise TypeError(f"{name}: dtype {t.dtype}, expected torch.{_DTYPE_NAMES[dtype]}")


def _rows(t, name: str, dtype: int, shape: tuple) -> tuple:
    """Pointer and row stride of a tensor [rows, heads, head_dim] of at least ``shape``'s rows whose heads are
    contiguous in a row; rejects one that the kernels would misread, as ``_require`` does."""
    if type(t) is _Tensor and t.is_cuda and t.dtype is _dtypes[dtype] and t.shape == shape:
        s0, s1, s2 = t.stride()  # the common case: the checks below without formatting names
        if s2 == 1 and s1 == shape[2] and shape[0] > 1:
            return t.data_ptr(), s0
    _typed(t, name, dtype)
    n_rows, heads, dim = shape
    sh, st = t.shape, t.stride()
    if len(sh) != 3 or sh[0] < n_rows or sh[1] != heads or sh[2] != dim:
        raise ValueError(f"{name}: shape {tuple(sh)}, expected {list(shape)}")
    if st[2] != 1 or (st[1] != dim and heads > 1):
        raise ValueError(f"{name}: the heads of a row are not contiguous")
    return t.data_ptr(), st[0] if sh[0] > 1 else heads * dim


def _workspace(t) -> tuple:
    """Pointer and bytes (the library compares them with what it needs)."""
    return _arg(t, "workspace", "uint8", 0), 0 if t is None else t.numel()


def _row_count(t, name: str) -> int:
    if type(t) is _Tensor:
        sh = t.shape
        if len(sh) == 3:
            return sh[0]
    if t is None or isinstance(t, (int, np.ndarray)) or len(t.shape) != 3:
        raise ValueError(f"{name}: a CUDA tensor [rows, heads, head_dim] is required")
    return t.shape[0]


def _cache(t, name: str, layout: IvitCacheLayout) -> int:
    """The pointer of a cache of this layout; rejects any other tensor."""
    if (type(t) is _Tensor and t.is_cuda and t.dtype is _dtypes[layout.dtype] and t.shape == layout.shape
            and t.stride() == layout.strides):
        return t.data_ptr()
    _typed(t, name, layout.dtype)
    if t.shape != layout.shape or t.stride() != layout.strides:
        raise ValueError(f"{name}: shape {tuple(t.shape)} and strides {t.stride()} are not the layout's, {layout.shape} and "
                         f"{layout.strides}")
    return t.data_ptr()


def _layers(t, name: str, dtype: int) -> tuple:
    """Shape and strides of a tensor with a leading layer dimension."""
    if t is None or isinstance(t, (int, np.ndarray)):
        raise TypeError(f"{name}: a CUDA tensor is required")
    _typed(t, name, dtype)
    return t.shape, t.stride()


def ivit_step_plan(cfg: IvitPlanConfig, held, base, new, parent, ring, ring_in, table, cu_rows, req, slots, positions,
                   mask, ring_out, status, stream=None) -> None:
    """Pages, slots, positions and tree masks of a step (int32 tensors; parent, req, positions and mask may be
    None): ``table`` [n_req, max_pages] and ``ring`` [n_pages] are updated, ``cu_rows`` [n_req + 1], the row arrays
    [max_rows], ``mask`` [max_rows, mask_words], ``ring_out`` [2] and ``status`` [1] written."""
    n, rows = cfg.n_req, cfg.max_rows
    args = (C.addressof(cfg), _i32(held, "held", n), _i32(base, "base", n), _i32(new, "new", n),
            _i32(parent, "parent", rows), _i32(ring, "ring", cfg.n_pages), _i32(ring_in, "ring_in", 2),
            _i32(table, "table", n * cfg.max_pages), _i32(cu_rows, "cu_rows", n + 1),
            _i32(req, "req", rows), _i32(slots, "slots", rows), _i32(positions, "positions", rows),
            _i32(mask, "mask", rows * cfg.mask_words), _i32(ring_out, "ring_out", 2),
            _i32(status, "status", 1), _stream(stream))
    _check(load().ivit_step_plan(*args), None)


def _rope_inputs(cfg: IvitRopeConfig, n: int, q_weight, k_weight, positions, freq, axis) -> tuple:
    """What the rotation and its gradient have in common, as the library takes it."""
    pairs, dt, dim = cfg.rot_dim // 2, _DTYPE_NAMES[cfg.dtype], cfg.head_dim
    if positions is None or isinstance(positions, (int, np.ndarray)):
        raise TypeError("positions: a CUDA tensor [rows] or [axes, rows] is required")
    sh = positions.shape
    if len(sh) == 1 or (len(sh) == 2 and sh[0] == 1):  # one position for all axes
        stride, least = 0, n
    elif len(sh) == 2 and sh[0] >= cfg.n_axes and sh[1] >= n:
        stride, least = sh[1], sh[0] * sh[1]
    else:
        raise ValueError(f"positions: shape {tuple(sh)}, expected [{cfg.n_axes}, {n}]")
    return (_arg(q_weight, "q_weight", dt, dim), _arg(k_weight, "k_weight", dt, dim),
            _i32(positions, "positions", least), stride, _arg(freq, "freq", "float32", pairs),
            _i32(axis, "axis", pairs))


def ivit_qk_norm_rope(cfg: IvitRopeConfig, q, k, v, q_weight, k_weight, positions, freq, axis, q_out, k_out=None,
                      cache: Optional[IvitCacheLayout] = None, k_cache=None, v_cache=None, slots=None,
                      stream=None) -> None:
    """Norm (where there is a weight) and rotation of q [rows, heads, head_dim] and k [rows, kv_heads, head_dim]
    into ``q_out``, ``k_out`` and, with ``cache``, of k and v into the ``slots`` of the paged caches.
    ``positions``: int32 [rows] or [axes, rows]; ``freq``, ``axis``: of each pair."""
    n, dt, dim = _row_count(q, "q"), cfg.dtype, cfg.head_dim
    q_shape, k_shape = (n, cfg.heads, dim), (n, cfg.kv_heads, dim)
    vp = lay = kc = vc = sl = ko = None
    vs = kos = 0
    if k_out is not None:
        ko, kos = _rows(k_out, "k_out", dt, k_shape)
    if cache is not None:
        vp, vs = _rows(v, "v", dt, k_shape)
        kc, vc = _cache(k_cache, "k_cache", cache), _cache(v_cache, "v_cache", cache)
        lay, sl = C.addressof(cache), _i32(slots, "slots", n)
    elif not (v is k_cache is v_cache is slots is None):
        raise ValueError("v, k_cache, v_cache and slots need the cache's layout")
    args = (C.addressof(cfg), n, *_rows(q, "q", dt, q_shape), *_rows(k, "k", dt, k_shape), vp, vs,
            *_rope_inputs(cfg, n, q_weight, k_weight, positions, freq, axis), *_rows(q_out, "q_out", dt, q_shape), ko, kos,
            lay, kc, vc, sl, _stream(stream))
    _check(load().ivit_qk_norm_rope(*args), None)


def ivit_qk_norm_rope_backward_workspace(cfg: IvitRopeConfig) -> int:
    """Bytes of the workspace of ``ivit_qk_norm_rope_backward`` (0: the configuration is invalid)."""
    return int(load().ivit_qk_norm_rope_backward_workspace(C.addressof(cfg)))


def ivit_qk_norm_rope_backward(cfg: IvitRopeConfig, grad_q, grad_k, q, k, q_weight, k_weight, positions, freq, axis, dq, dk,
                               dq_weight=None, dk_weight=None, workspace=None, stream=None) -> None:
    """Gradients of ``ivit_qk_norm_rope``: ``dq``, ``dk`` and the weights' fp32
    [head_dim] (or None)."""
    n, dt, dim = _row_count(q, "q"), cfg.dtype, cfg.head_dim
    q_shape, k_shape = (n, cfg.heads, dim), (n, cfg.kv_heads, dim)
    dqw, dkw = _arg(dq_weight, "dq_weight", "float32", dim), _arg(dk_weight, "dk_weight", "float32", dim)
    args = (C.addressof(cfg), n, *_rows(grad_q, "grad_q", dt, q_shape), *_rows(grad_k, "grad_k", dt, k_shape),
            *_rows(q, "q", dt, q_shape), *_rows(k, "k", dt, k_shape),
            *_rope_inputs(cfg, n, q_weight, k_weight, positions, freq, axis), *_rows(dq, "dq", dt, q_shape),
            *_rows(dk, "dk", dt, k_shape), dqw, dkw, *_workspace(workspace), _stream(stream))
    _check(load().ivit_qk_norm_rope_backward(*args), None)


def ivit_tree_attention_workspace(cfg: IvitAttentionConfig, cache: IvitCacheLayout) -> int:
    """Bytes of the workspace of ``ivit_tree_attention`` (0: the arguments are invalid)."""
    return int(load().ivit_tree_attention_workspace(C.addressof(cfg), C.addressof(cache)))


def ivit_tree_attention(cfg: IvitAttentionConfig, cache: IvitCacheLayout, q, k_new, v_new, k_cache, v_cache, table, lengths,
                        cu_rows, mask, out, lse=None, workspace=None, stream=None) -> None:
    """Attention of the new rows q [rows, heads, head_dim] over the cached tokens of their requests and over the new
    keys and values [rows, kv_heads, head_dim] that the mask lets them see; ``lse`` fp32 [rows, heads] or None."""
    n, dt, dim, heads, req = _row_count(q, "q"), cache.dtype, cache.head_dim, cfg.heads, cfg.n_req
    q_shape, k_shape = (n, heads, dim), (n, cache.kv_heads, dim)
    if cfg.mask_mode != IVIT_MASK_TREE:
        mask = None
    args = (C.addressof(cfg), C.addressof(cache), n, *_rows(q, "q", dt, q_shape), *_rows(k_new, "k_new", dt, k_shape),
            *_rows(v_new, "v_new", dt, k_shape), _cache(k_cache, "k_cache", cache), _cache(v_cache, "v_cache", cache),
            _i32(table, "table", req * cfg.max_pages), _i32(lengths, "lengths", req),
            _i32(cu_rows, "cu_rows", req + 1), _i32(mask, "mask", n * cfg.mask_words),
            *_rows(out, "out", dt, q_shape), _arg(lse, "lse", "float32", n * heads),
            *_workspace(workspace), _stream(stream))
    _check(load().ivit_tree_attention(*args), None)


def ivit_kv_write(cache: IvitCacheLayout, k, v, rows, slots, k_cache, v_cache, stream=None) -> None:
    """Rows ``rows`` (int32, -1: none) of k and v [layers, rows, kv_heads, head_dim] into the ``slots`` of the caches
    [layers, pages, page_size, kv_heads, head_dim] of all layers."""
    dt, kv, dim = cache.dtype, cache.kv_heads, cache.head_dim
    (sh, st), (vsh, vst) = _layers(k, "k", dt), _layers(v, "v", dt)
    if len(sh) != 4 or sh[2] != kv or sh[3] != dim or sh != vsh:
        raise ValueError(f"k, v: shapes {tuple(sh)} and {tuple(vsh)}, expected [layers, rows, {kv}, {dim}]")
    if st[3] != 1 or (st[2] != dim and kv > 1) or st != vst:
        raise ValueError("k, v: the heads of a row are not contiguous, or the strides differ")
    (csh, cst), (vcsh, vcst) = _layers(k_cache, "k_cache", dt), _layers(v_cache, "v_cache", dt)
    layers, n_src = sh[0], sh[1]
    if csh[1:] != cache.shape or cst[1:] != cache.strides or vcsh != csh or vcst != cst or csh[0] < layers:
        raise ValueError(f"k_cache, v_cache: shapes {tuple(csh)} and {tuple(vcsh)} are not {layers} caches of the layout, "
                         f"{cache.shape}, with strides {cache.strides}")
    if rows is None or isinstance(rows, (int, np.ndarray)):
        raise TypeError("rows: a CUDA tensor is required")
    n = rows.numel()
    args = (C.addressof(cache), layers, n, n_src, k.data_ptr(), v.data_ptr(), st[1] if n_src > 1 else kv * dim,
            st[0] if layers > 1 else 0, _i32(rows, "rows", n), _i32(slots, "slots", n),
            k_cache.data_ptr(), v_cache.data_ptr(), cst[0] if layers > 1 else 0, _stream(stream))
    _check(load().ivit_kv_write(*args), None)


# ------------------------------------------------------------ convenience

class IncrementalViT:
    """Owns one library handle; torch tensors in and out (device memory, torch streams)."""

    def __init__(self, shape: "synth.EncoderShape", weights_u16: np.ndarray, n_streams: int = 1,
                 n_views: int = 1, select_mode: int = synth.SEL_THRESHOLD,
                 threshold: float = 0.98, topk: int = 0, ref_mode: int = synth.REF_PREV_FRAME,
                 score_source: int = synth.SCORE_EMBED, schedule: int = synth.SCHED_INCREMENTAL,
                 mlp_tokens: int = 0):
        import torch
        self.torch = torch
        self.shape = shape
        self.sv = n_streams * n_views
        self.cfg = make_config(shape, n_streams, n_views, select_mode, threshold, topk, ref_mode,
                               score_source, schedule, mlp_tokens)
        self.h = ivit_create(self.cfg, weights_u16)
        self.device = torch.device("cuda", torch.cuda.current_device())

    @classmethod
    def for_workload(cls, wl, weights_u16):
        return cls(wl.shape, weights_u16, wl.n_streams, wl.n_views, wl.select_mode, wl.threshold,
                   wl.topk, wl.ref_mode, wl.score_source, wl.schedule, wl.mlp_tokens)

    def close(self):
        if getattr(self, "h", None):
            ivit_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def tokens_buffer(self):
        return self.torch.empty((self.sv, self.shape.n_tokens, self.shape.dim),
                                dtype=self.torch.bfloat16, device=self.device)

    def encode_full(self, frames, out=None, stream=None):
        out = self.tokens_buffer() if out is None else out
        ivit_encode_full(self.h, frames, out, stream)
        return out

    def encode_incremental(self, frames, out=None, counts=None, stream=None):
        out = self.tokens_buffer() if out is None else out
        counts = (self.torch.empty(self.sv, dtype=self.torch.int32, device=self.device)
                  if counts is None else counts)
        ivit_encode_incremental(self.h, frames, out, counts, stream)
        return out, counts

    def changed(self, sv: int, stream=None):
        idx = self.torch.empty(self.shape.n_tokens, dtype=self.torch.int32, device=self.device)
        cnt = self.torch.empty(1, dtype=self.torch.int32, device=self.device)
        ivit_get_changed(self.h, sv, idx, cnt, stream)
        return idx[: int(cnt.item())]

    def cache(self, which: str, layer: int = 0, stream=None):
        code = {"K": 0, "V": 1, "tokens": 2, "ref": 3, "A": 4}[which]
        dt = self.torch.float32 if code in (3, 4) else self.torch.bfloat16
        dst = self.torch.empty((self.sv, self.shape.n_tokens, self.shape.dim), dtype=dt,
                               device=self.device)
        ivit_get_cache(self.h, code, layer, dst, stream)
        return dst

    def reset(self, stream_index: int = -1):
        ivit_reset(self.h, stream_index)

    def device_status(self, stream=None) -> int:
        return ivit_device_status(self.h, stream)
