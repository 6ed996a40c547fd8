"""Thin ctypes binding of the C ABI in include/wq.h, include/wq_attention.h,
include/wq_fused.h, include/wq_cache.h, include/wq_window.h,
include/wq_logits.h and include/wq_probe.h.

Only argument marshalling happens here: torch tensors are turned into device
pointers and sizes, the current HIP stream is passed through, and non-OK
status codes become WQError.  Every step of the computation runs in the HIP
library; if the library is not built this module raises instead of falling
back to anything else.
"""

from __future__ import annotations

import ctypes
import os

# The in-tree build.  WQ_LIBRARY names another build of the same library to
# load instead (the host-sanitizer test loads one built with AddressSanitizer
# on its host code).
LIB_PATH = os.environ.get("WQ_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libwq.so")

WQ_OK = 0
WQ_ERR_INVALID_ARG = 1
WQ_ERR_UNSUPPORTED = 2
WQ_ERR_MISALIGNED = 3
WQ_ERR_HIP = 4

GROUP = 32

# Every function declared in the headers under include/.
EXPORTED = ("wq_status_string", "wq_last_error_message", "wq_version", "wq_pack", "wq_gemv",
            "wq_decode_linears", "wq_decode_linears_noalloc", "wq_paged_attention_workspace_size",
            "wq_paged_attention", "wq_fused_linears", "wq_fused_check", "wq_stream_read",
            "wq_cache_append", "wq_cache_copy_pages", "wq_page_workspace_size", "wq_cache_reserve", "wq_cache_free",
            "wq_cache_fork", "wq_cache_compact", "wq_process_logits_workspace_size", "wq_process_logits",
            "wq_window_attention_workspace_size", "wq_window_attention")

# Limits of wq_decode_linears_noalloc (include/wq.h).
NOALLOC_MAX_LINEARS = 1024
NOALLOC_SCRATCH_BYTES = 131072

PROLOGUE_NONE = 0
PROLOGUE_RMSNORM = 1
PROLOGUE_SILU_MUL = 2


class WqLinear(ctypes.Structure):
    _fields_ = [
        ("packed_w", ctypes.c_void_p),
        ("scales", ctypes.c_void_p),
        ("x", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("N", ctypes.c_int64),
        ("K", ctypes.c_int64),
    ]


class WqFusedLinear(ctypes.Structure):
    _fields_ = [
        ("packed_w", ctypes.c_void_p),
        ("scales", ctypes.c_void_p),
        ("x", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("norm_weight", ctypes.c_void_p),
        ("residual", ctypes.c_void_p),
        ("N", ctypes.c_int64),
        ("K", ctypes.c_int64),
        ("prologue", ctypes.c_int32),
        ("eps", ctypes.c_float),
    ]


class WqLogitsCall(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in (
        "logits", "out", "token", "mask", "history", "history_lens", "prompt_lens", "repetition", "frequency", "presence",
        "bias_ids", "bias_values", "bias_lens")] + [(name, ctypes.c_int64) for name in (
            "rows", "vocab", "logits_stride", "out_stride", "mask_stride", "history_size", "bias_size", "dtype")]


class WQError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{status_string(status)}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Load libwq.so (once) and declare the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library not built: {LIB_PATH} is missing "
                           "(run `python -m paper_2412_15803_amd.build`)")
    L = ctypes.CDLL(LIB_PATH)
    i64, vp = ctypes.c_int64, ctypes.c_void_p
    L.wq_status_string.argtypes = [ctypes.c_int]
    L.wq_status_string.restype = ctypes.c_char_p
    L.wq_last_error_message.argtypes = []
    L.wq_last_error_message.restype = ctypes.c_char_p
    L.wq_version.argtypes = []
    L.wq_version.restype = ctypes.c_int
    L.wq_pack.argtypes = [vp, vp, vp, i64, i64, i64, vp]
    L.wq_pack.restype = ctypes.c_int
    L.wq_gemv.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp]
    L.wq_gemv.restype = ctypes.c_int
    L.wq_decode_linears.argtypes = [ctypes.POINTER(WqLinear), i64, i64, i64, vp]
    L.wq_decode_linears.restype = ctypes.c_int
    L.wq_decode_linears_noalloc.argtypes = [ctypes.POINTER(WqLinear), i64, i64, i64, vp]
    L.wq_decode_linears_noalloc.restype = ctypes.c_int
    L.wq_paged_attention_workspace_size.argtypes = [i64, i64, i64, i64, i64, ctypes.POINTER(ctypes.c_size_t)]
    L.wq_paged_attention_workspace_size.restype = ctypes.c_int
    L.wq_paged_attention.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, i64,
                                     ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.wq_paged_attention.restype = ctypes.c_int
    L.wq_fused_linears.argtypes = [ctypes.POINTER(WqFusedLinear), i64, vp, i64, vp]
    L.wq_fused_linears.restype = ctypes.c_int
    L.wq_fused_check.argtypes = [vp]
    L.wq_fused_check.restype = ctypes.c_int
    L.wq_stream_read.argtypes = [vp, i64, vp, vp]
    L.wq_stream_read.restype = ctypes.c_int
    sz = ctypes.c_size_t
    for name, args in (
            ("wq_cache_append", [vp] * 7 + [i64] * 9 + [vp]),
            ("wq_cache_copy_pages", [vp, i64, i64, i64, vp, vp, i64, vp]),
            ("wq_page_workspace_size", [i64, i64, ctypes.POINTER(sz)]),
            ("wq_cache_reserve", [vp] * 4 + [i64] * 4 + [vp, vp, sz, vp]),
            ("wq_cache_free", [vp] * 4 + [i64] * 7 + [vp]),
            ("wq_cache_fork", [vp, i64] + [vp] * 5 + [i64] * 7 + [vp, vp, sz, vp]),
            ("wq_cache_compact", [vp, i64, i64] + [vp] * 5 + [i64] * 3 + [vp, sz, vp]),
            ("wq_process_logits_workspace_size", [i64, i64, i64, ctypes.POINTER(sz)]),
            ("wq_process_logits", [vp, vp, sz, vp]),
            ("wq_window_attention_workspace_size", [i64] * 9 + [ctypes.POINTER(sz)]),
            ("wq_window_attention", [vp] * 7 + [i64] * 14 + [ctypes.c_float, i64, vp, sz, vp])):
        getattr(L, name).argtypes = args
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().wq_status_string(int(status)).decode()


def last_error_message() -> str:
    return lib().wq_last_error_message().decode()


def _check(status: int) -> None:
    if status != WQ_OK:
        raise WQError(status, last_error_message())


# ------------------------------------------------------------- marshalling
#
# A small call's time is this code's (a 512 x 512 linear runs about 2 us on
# the device), so a tensor is looked at once, with plain attribute reads, and
# pointers and the stream are passed as integers (the declared argument types
# turn them into C values).

_torch = _Tensor = None
_WORDS = _HALVES = _FLOATS = _INTS = _BYTES = ()
_DTYPES = {}  # WQ_DTYPE_* of include/wq_logits.h
_raw_stream = None


def _load_torch():
    global _torch, _Tensor, _WORDS, _HALVES, _FLOATS, _INTS, _BYTES, _DTYPES, _raw_stream
    import torch

    _WORDS = (torch.int32, torch.uint32)
    _HALVES = (torch.float16, torch.int16, torch.uint16)
    _FLOATS = (torch.float32,)
    _INTS = (torch.int32,)
    _BYTES = (torch.uint8,)
    _DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
    # The current stream's handle without building a Stream object.
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _Tensor = torch.Tensor
    _torch = torch
    return torch


def _dev_tensor(t, name, dtypes, shape):
    """The device address of `t` after the checks that every argument gets."""
    if isinstance(t, _Tensor) and t.is_cuda and t.dtype in dtypes and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    # Something is wrong with it: say what.
    if not isinstance(t, _torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name} must be contiguous (row-major)")


def _stream(stream, t):
    """The handle of `stream`, or of the current stream of the device of `t`."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return _torch.cuda.current_stream(t.device).cuda_stream


def _unchecked_stream(stream, t):
    """_stream for a tensor that the call has not looked at (a marshalled
    list's, a buffer's): a host tensor has no stream."""
    if stream is None and not t.is_cuda:
        raise ValueError(f"expected a device tensor (got {t.device})")
    return _stream(stream, t)


def wq_pack(w, packed_w, scales, group: int = GROUP, stream=None) -> None:
    """Quantize fp32 w [N, K] into packed_w [N, K/8] (int32/uint32 words) and
    scales [N, K/32] (fp16), both preallocated on the same device."""
    _torch or _load_torch()
    if w.dim() != 2:
        raise ValueError("w must be 2-D [N, K]")
    n, k = w.shape
    pw = _dev_tensor(w, "w", _FLOATS, (n, k))
    pp = _dev_tensor(packed_w, "packed_w", _WORDS, (n, k // 8))
    ps = _dev_tensor(scales, "scales", _HALVES, (n, k // group if group else 0))
    _check((_lib or lib()).wq_pack(pw, pp, ps, n, k, group, _stream(stream, w)))


def wq_gemv(packed_w, scales, x, y, group: int = GROUP, stream=None) -> None:
    """y [M, N] = x [M, K] . dequant(packed_w, scales)^T (fp16 in, fp16 out)."""
    _torch or _load_torch()
    if x.dim() != 2 or packed_w.dim() != 2:
        raise ValueError("x must be [M, K] and packed_w [N, K/8]")
    m, k = x.shape
    n = packed_w.shape[0]
    pp = _dev_tensor(packed_w, "packed_w", _WORDS, (n, k // 8))
    ps = _dev_tensor(scales, "scales", _HALVES, (n, k // group if group else 0))
    px = _dev_tensor(x, "x", _HALVES, (m, k))
    py = _dev_tensor(y, "y", _HALVES, (m, n))
    _check((_lib or lib()).wq_gemv(pp, ps, px, py, n, k, m, group, _stream(stream, x)))


def make_linear_array(linears, m: int, group: int = GROUP):
    """Marshal a sequence of (packed_w, scales, x, y) tensor tuples into a
    ctypes wq_linear array."""
    _torch or _load_torch()
    arr = (WqLinear * len(linears))()
    for i, (packed_w, scales, x, y) in enumerate(linears):
        if x.dim() != 2 or x.shape[0] != m:
            raise ValueError(f"linear {i}: x must be [M={m}, K]")
        k = x.shape[1]
        n = packed_w.shape[0]
        arr[i].packed_w = _dev_tensor(packed_w, f"linears[{i}].packed_w", _WORDS, (n, k // 8))
        arr[i].scales = _dev_tensor(scales, f"linears[{i}].scales", _HALVES, (n, k // group if group else 0))
        arr[i].x = _dev_tensor(x, f"linears[{i}].x", _HALVES, (m, k))
        arr[i].y = _dev_tensor(y, f"linears[{i}].y", _HALVES, (m, n))
        arr[i].N = n
        arr[i].K = k
    return arr


def wq_decode_linears(linears, m: int = 1, group: int = GROUP, stream=None, _array=None) -> None:
    """Run a decode step's linears in order on one stream.  `linears` is a
    sequence of (packed_w, scales, x, y) tuples; a prebuilt array from
    make_linear_array may be passed as _array to skip re-marshalling."""
    arr = _array if _array is not None else make_linear_array(linears, m, group)
    _torch or _load_torch()
    _check((_lib or lib()).wq_decode_linears(arr, len(arr), m, group, _unchecked_stream(stream, linears[0][2])))


def wq_decode_linears_noalloc(linears, m: int = 1, group: int = GROUP, stream=None, _array=None) -> None:
    """wq_decode_linears through the entry point that allocates nothing (its
    plan lives in the library's fixed per-device array; see include/wq.h)."""
    arr = _array if _array is not None else make_linear_array(linears, m, group)
    _torch or _load_torch()
    _check((_lib or lib()).wq_decode_linears_noalloc(arr, len(arr), m, group, _unchecked_stream(stream, linears[0][2])))


# ------------------------------------------------------- paged attention

def paged_attention_workspace_size(num_seqs: int, num_q_heads: int, num_kv_heads: int,
                                   head_dim: int, max_seq_len: int) -> int:
    """Bytes of device workspace wq_paged_attention needs (0: none)."""
    out = ctypes.c_size_t(0)
    _check(lib().wq_paged_attention_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim,
                                                   max_seq_len, ctypes.byref(out)))
    return int(out.value)


def paged_workspace(q, max_seq_len: int, num_kv_heads: int):
    """A device workspace (uint8 tensor, or None) sized for these shapes."""
    import torch

    num_seqs, hq, d = q.shape
    n = paged_attention_workspace_size(num_seqs, hq, num_kv_heads, d, max_seq_len)
    return torch.empty(n, dtype=torch.uint8, device=q.device) if n else None


def paged_attention(q, k_cache, v_cache, block_table, seq_lens, out, scale: float, max_seq_len: int,
                    workspace=None, stream=None) -> None:
    """out [S, HQ, D] = decode attention of q [S, HQ, D] over the paged
    caches [pages, HKV, P, D] (fp16), block_table [S, max_pages] and
    seq_lens [S] (int32), all on one device.  `workspace` is a uint8 device
    tensor from paged_workspace (allocated here when omitted)."""
    _torch or _load_torch()
    if q.dim() != 3 or k_cache.dim() != 4:
        raise ValueError("q must be [S, HQ, D] and the caches [pages, HKV, P, D]")
    num_seqs, hq, d = q.shape
    num_pages, hkv, page, d2 = k_cache.shape
    max_pages = block_table.shape[1] if block_table.dim() == 2 else 0
    pq = _dev_tensor(q, "q", _HALVES, (num_seqs, hq, d))
    pk = _dev_tensor(k_cache, "k_cache", _HALVES, (num_pages, hkv, page, d2))
    pv = _dev_tensor(v_cache, "v_cache", _HALVES, (num_pages, hkv, page, d2))
    pt = _dev_tensor(block_table, "block_table", _INTS, (num_seqs, max_pages))
    pl = _dev_tensor(seq_lens, "seq_lens", _INTS, (num_seqs,))
    po = _dev_tensor(out, "out", _HALVES, (num_seqs, hq, d))
    if workspace is None:
        with _torch.cuda.stream(stream):  # memory that is `stream`'s (None: the current one's)
            workspace = paged_workspace(q, max_seq_len, hkv)
    if workspace is not None:
        if workspace.device != q.device or workspace.dtype not in _BYTES or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on the device of q")
        pw, nw = workspace.data_ptr(), workspace.numel()
    else:
        pw, nw = None, 0
    _check((_lib or lib()).wq_paged_attention(pq, pk, pv, pt, pl, po, num_seqs, hq, hkv, d, page, num_pages,
                                              max_pages, max_seq_len, float(scale), pw, nw, _stream(stream, q)))


# ------------------------------------------------------- fused decode chain

def make_fused_array(linears, group: int = GROUP):
    """Marshal dicts with keys packed_w, scales, x, y (tensors) and optional
    prologue (PROLOGUE_*), norm_weight, eps, residual into a ctypes
    wq_fused_linear array.  x is [K] ([2K] for PROLOGUE_SILU_MUL), y and
    residual [N], norm_weight [K]; 1-D or [1, n] tensors are accepted."""
    _torch or _load_torch()
    arr = (WqFusedLinear * len(linears))()
    for i, d in enumerate(linears):
        packed_w, scales, x, y = d["packed_w"], d["scales"], d["x"], d["y"]
        pro = int(d.get("prologue", PROLOGUE_NONE))
        n = packed_w.shape[0]
        k = packed_w.shape[1] * 8
        xk = 2 * k if pro == PROLOGUE_SILU_MUL else k
        arr[i].packed_w = _dev_tensor(packed_w, f"linears[{i}].packed_w", _WORDS, (n, k // 8))
        arr[i].scales = _dev_tensor(scales, f"linears[{i}].scales", _HALVES, (n, k // group))
        arr[i].x = _dev_tensor(x.reshape(-1), f"linears[{i}].x", _HALVES, (xk,))
        arr[i].y = _dev_tensor(y.reshape(-1), f"linears[{i}].y", _HALVES, (n,))
        norm = d.get("norm_weight")
        arr[i].norm_weight = _dev_tensor(norm, f"linears[{i}].norm_weight", _HALVES, (k,)) \
            if norm is not None else None
        res = d.get("residual")
        arr[i].residual = _dev_tensor(res.reshape(-1), f"linears[{i}].residual", _HALVES, (n,)) \
            if res is not None else None
        arr[i].N = n
        arr[i].K = k
        arr[i].prologue = pro
        arr[i].eps = float(d.get("eps", 0.0))
    return arr


def wq_fused_linears(linears, argmax=None, group: int = GROUP, stream=None, _array=None) -> None:
    """Run a chain of fused linears in order (see make_fused_array); when
    `argmax` (a device int32 tensor of one element) is given, the index of
    the largest element of the last linear's y is written to it."""
    _torch or _load_torch()
    arr = _array if _array is not None else make_fused_array(linears, group)
    pa = _dev_tensor(argmax.reshape(-1), "argmax", _INTS, (1,)) if argmax is not None else None
    _check((_lib or lib()).wq_fused_linears(arr, len(arr), pa, group, _unchecked_stream(stream, linears[0]["x"])))


def wq_fused_check(device=None, stream=None) -> None:
    """Synchronize the stream and raise WQError if a persistent chain on the
    device gave up since the last check (a bounded wait ran out)."""
    import torch

    stream = torch.cuda.current_stream(device) if stream is None else stream
    _check(lib().wq_fused_check(stream.cuda_stream))


# ------------------------------------------------------- window attention

def window_attention_workspace_size(num_seqs: int, num_tokens: int, max_query_len: int, num_q_heads: int, num_kv_heads: int,
                                    head_dim: int, max_seq_len: int, window: int, sinks: int) -> int:
    """Bytes of device workspace wq_window_attention needs (0: none)."""
    out = ctypes.c_size_t(0)
    _check(lib().wq_window_attention_workspace_size(num_seqs, num_tokens, max_query_len, num_q_heads, num_kv_heads, head_dim,
                                                    max_seq_len, window, sinks, ctypes.byref(out)))
    return int(out.value)


def window_workspace(q, num_kv_heads: int, num_seqs: int, max_seq_len: int, window: int, sinks: int = 0, max_query_len: int = 1):
    """A device workspace (uint8 tensor, or None) for window_attention."""
    import torch

    n = window_attention_workspace_size(num_seqs, q.shape[0], max_query_len, q.shape[1], num_kv_heads, q.shape[2], max_seq_len, window, sinks)
    return torch.empty(n, dtype=torch.uint8, device=q.device) if n else None


def window_attention(q, k_cache, v_cache, block_table, seq_lens, out, scale: float, max_seq_len: int, window: int, sinks: int = 0,
                     q_starts=None, max_query_len: int = 1, workspace=None, stream=None) -> None:
    """out [T, HQ, D] = causal attention of the new tokens' queries q [T, HQ, D]
    over the paged caches [pages, HKV, P, D] (all fp16 or all bf16): a token at
    position p sees token t <= p when t < sinks or t > p - window.  seq_lens [S]
    counts the new tokens; rows q_starts[s] to q_starts[s + 1] (int32, [S + 1],
    at most max_query_len of them) belong to the last tokens of sequence s, or
    row s to its last one when q_starts is None.  Rows of q and out may lie
    apart (slices of a wider array).  `workspace` is from window_workspace
    (allocated here when omitted)."""
    _torch or _load_torch()
    shape, cached, rows = q.shape, k_cache.shape, block_table.shape
    if len(shape) != 3 or len(rows) != 2:
        raise ValueError("q must be [T, HQ, D] and block_table [S, max_pages]")
    num_pages, hkv, page, d = cached if len(cached) == 4 else _cache_dims(k_cache, "k_cache")
    kind = k_cache.dtype
    if kind not in _DTYPES or k_cache.element_size() != 2:
        _cache_dims(k_cache, "k_cache")
        raise TypeError(f"the caches must be fp16 or bf16 (got {kind})")
    tokens, hq, dim = shape
    if dim != d:
        raise ValueError(f"q has head_dim {dim}, the caches {d}")
    num_seqs, max_pages = rows
    kinds = (kind,)
    pq, qs = _rows_tensor(q, "q", kind, shape)
    po, os_ = _rows_tensor(out, "out", kind, shape)
    pk = _dev_tensor(k_cache, "k_cache", kinds, cached)
    pv = _dev_tensor(v_cache, "v_cache", kinds, cached)
    pt = _dev_tensor(block_table, "block_table", _INTS, rows)
    pl = _dev_tensor(seq_lens, "seq_lens", _INTS, (num_seqs,))
    ps = None if q_starts is None else _dev_tensor(q_starts, "q_starts", _INTS, (num_seqs + 1,))
    if workspace is None:
        with _torch.cuda.stream(stream):  # memory that is `stream`'s (None: the current one's)
            workspace = window_workspace(q, hkv, num_seqs, max_seq_len, window, sinks, max_query_len)
    pw, nw = _workspace(workspace, q)
    _check((_lib or lib()).wq_window_attention(pq, pk, pv, pt, pl, ps, po, num_seqs, tokens, max_query_len, hq, hkv, d, qs, os_, page,
                                               num_pages, max_pages, max_seq_len, window, sinks, float(scale), _DTYPES[kind], pw, nw,
                                               _stream(stream, q)))


# ------------------------------------------------------- paged cache upkeep

def _rows_tensor(t, name, dtype, shape):
    """Address and row stride of `t` [rows, heads, dim], whose rows may lie
    apart (a slice of a wider array) but are contiguous in themselves."""
    if isinstance(t, _Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape:
        stride, head, one = t.stride()
        if (one == 1 or shape[2] == 1) and (head == shape[2] or shape[1] == 1):
            # (One row's stride says nothing.)
            return t.data_ptr(), stride if shape[0] > 1 else shape[1] * shape[2]
        raise ValueError(f"the rows of {name} must be contiguous")
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _workspace(workspace, t):
    if workspace is None:
        return None, 0
    if not workspace.is_cuda or workspace.get_device() != t.get_device() or workspace.dtype not in _BYTES or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of the other arguments")
    return workspace.data_ptr(), workspace.numel()


def _cache_dims(cache, name):
    shape = cache.shape
    if len(shape) != 4:
        raise ValueError(f"{name} must be [pages, HKV, P, D]")
    if cache.element_size() != 2:
        raise TypeError(f"{name} must hold 16-bit values (got {cache.dtype})")
    return shape


def cache_append(k, v, k_cache, v_cache, block_table, seq_lens, q_starts=None, stream=None) -> None:
    """Write the keys k and values v [T, HKV, D] of new tokens to their slots in
    the paged caches [pages, HKV, P, D] (the caches' 16-bit type).  seq_lens
    [S] counts the new tokens; rows q_starts[s] to q_starts[s + 1] (int32,
    [S + 1]) are the last tokens of sequence s, or row s its last one when
    q_starts is None.  Rows of k and v may lie apart (slices of the QKV
    projection's output)."""
    _torch or _load_torch()
    num_pages, hkv, page, d = cached = _cache_dims(k_cache, "k_cache")
    kind = k_cache.dtype
    shape, rows = k.shape, block_table.shape
    if len(rows) != 2 or len(shape) != 3:
        raise ValueError("k must be [T, HKV, D] and block_table [S, max_pages]")
    num_seqs, max_pages = rows
    if shape[1] != hkv or shape[2] != d:
        raise ValueError(f"k has shape {tuple(shape)}, the caches {hkv} heads of {d}")
    pk, ks = _rows_tensor(k, "k", kind, shape)
    pv, vs = _rows_tensor(v, "v", kind, shape)
    pkc = _dev_tensor(k_cache, "k_cache", (kind,), cached)
    pvc = _dev_tensor(v_cache, "v_cache", (kind,), cached)
    pt = _dev_tensor(block_table, "block_table", _INTS, rows)
    pl = _dev_tensor(seq_lens, "seq_lens", _INTS, (num_seqs,))
    ps = None if q_starts is None else _dev_tensor(q_starts, "q_starts", _INTS, (num_seqs + 1,))
    if shape[0] == 0:
        return
    _check((_lib or lib()).wq_cache_append(pk, pv, pkc, pvc, pt, pl, ps, num_seqs, shape[0], hkv, d, ks, vs, page, num_pages,
                                           max_pages, _stream(stream, k_cache)))


class CacheSet:
    """The caches of all layers, marshalled once: tensors [pages, HKV, P, D] of
    one shape and 16-bit type on one device.  Keeps the tensors alive."""

    def __init__(self, caches):
        _torch or _load_torch()
        caches = list(caches)
        if not caches:
            raise ValueError("a cache set needs at least one cache")
        first = caches[0]
        self.num_pages, self.kv_heads, self.page, self.head_dim = _cache_dims(first, "caches[0]")
        self.array = (ctypes.c_void_p * len(caches))(
            *[_dev_tensor(c, f"caches[{i}]", (first.dtype,), first.shape) for i, c in enumerate(caches)])
        if any(c.device != first.device for c in caches):
            raise ValueError("the caches must be on one device")
        self.caches = caches
        self.page_bytes = 2 * self.kv_heads * self.page * self.head_dim


def cache_set(caches) -> CacheSet:
    return CacheSet(caches)


def page_workspace_size(num_pages: int, num_seqs: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().wq_page_workspace_size(num_pages, num_seqs, ctypes.byref(out)))
    return int(out.value)


def page_workspace(num_pages: int, num_seqs: int, device="cuda"):
    """A device workspace for cache_reserve, cache_fork and cache_compact."""
    import torch

    return torch.empty(page_workspace_size(num_pages, num_seqs), dtype=torch.uint8, device=device)


def cache_copy_pages(caches: CacheSet, src, dst, stream=None) -> None:
    """Copy page src[i] to page dst[i] (int32 [n]) in every cache of the set."""
    n = src.shape[0] if src.dim() == 1 else -1
    ps = _dev_tensor(src, "src", _INTS, (n,))
    pd = _dev_tensor(dst, "dst", _INTS, (n,))
    _check((_lib or lib()).wq_cache_copy_pages(caches.array, len(caches.array), caches.page_bytes, caches.num_pages, ps, pd, n,
                                               _stream(stream, caches.caches[0])))


def _pool(block_table, refs):
    _torch or _load_torch()
    rows, pages = block_table.shape, refs.shape
    if len(rows) != 2 or len(pages) != 1:
        raise ValueError("block_table must be [S, max_pages] and refs [pages]")
    return (_dev_tensor(block_table, "block_table", _INTS, rows), _dev_tensor(refs, "refs", _INTS, pages), rows[0], rows[1], pages[0])


def cache_reserve(block_table, refs, old_lens, new_lens, page_size: int, shortfall, workspace=None, stream=None) -> None:
    """Give sequences that grow from old_lens to new_lens (int32 [S]) the pages
    they lack, lowest free page first.  shortfall (int32 [1]) becomes 0, or the
    number of pages too few, and then nothing else changes."""
    pt, pr, num_seqs, max_pages, num_pages = _pool(block_table, refs)
    po = _dev_tensor(old_lens, "old_lens", _INTS, (num_seqs,))
    pn = _dev_tensor(new_lens, "new_lens", _INTS, (num_seqs,))
    pf = _dev_tensor(shortfall, "shortfall", _INTS, (1,))
    if workspace is None:
        with _torch.cuda.stream(stream):  # memory that is `stream`'s (None: the current one's)
            workspace = page_workspace(num_pages, num_seqs, refs.device)
    pw, nw = _workspace(workspace, refs)
    _check((_lib or lib()).wq_cache_reserve(pt, pr, po, pn, num_seqs, page_size, num_pages, max_pages, pf, pw, nw, _stream(stream, refs)))


def cache_free(block_table, refs, seq_lens, seqs, page_size: int, window: int = 0, sinks: int = 0, stream=None) -> None:
    """Take from the sequences listed in seqs (int32 [n]) the pages that hold
    neither one of the first `sinks` tokens nor one that the next token sees
    through a window of `window` tokens; all pages when both are 0."""
    pt, pr, num_seqs, max_pages, num_pages = _pool(block_table, refs)
    pl = _dev_tensor(seq_lens, "seq_lens", _INTS, (num_seqs,))
    n = seqs.shape[0] if seqs.dim() == 1 else -1
    ps = _dev_tensor(seqs, "seqs", _INTS, (n,))
    _check((_lib or lib()).wq_cache_free(pt, pr, pl, ps, n, window, sinks, num_seqs, page_size, num_pages, max_pages, _stream(stream, refs)))


def cache_fork(caches: CacheSet, block_table, refs, seq_lens, src, dst, shortfall, workspace=None, stream=None) -> None:
    """Make sequence dst[i] a copy of sequence src[i] (int32 [n]): full pages are
    shared, a partly filled last page is copied in every cache."""
    pt, pr, num_seqs, max_pages, num_pages = _pool(block_table, refs)
    if num_pages != caches.num_pages:
        raise ValueError(f"refs has {num_pages} pages, the caches {caches.num_pages}")
    pl = _dev_tensor(seq_lens, "seq_lens", _INTS, (num_seqs,))
    n = src.shape[0] if src.dim() == 1 else -1
    ps = _dev_tensor(src, "src", _INTS, (n,))
    pd = _dev_tensor(dst, "dst", _INTS, (n,))
    pf = _dev_tensor(shortfall, "shortfall", _INTS, (1,))
    if workspace is None:
        with _torch.cuda.stream(stream):  # memory that is `stream`'s (None: the current one's)
            workspace = page_workspace(num_pages, num_seqs, refs.device)
    pw, nw = _workspace(workspace, refs)
    _check((_lib or lib()).wq_cache_fork(caches.array, len(caches.array), pt, pr, pl, ps, pd, n, num_seqs, caches.kv_heads, caches.head_dim,
                                         caches.page, num_pages, max_pages, pf, pw, nw, _stream(stream, refs)))


def cache_compact(caches: CacheSet, block_table, refs, new_table, new_refs, live, workspace=None, stream=None) -> None:
    """Move the pages in use to the numbers below their count, which live (int32
    [1]) receives; new_table and new_refs (which may be block_table and refs)
    receive the table and the counts with the new numbers."""
    pt, pr, num_seqs, max_pages, num_pages = _pool(block_table, refs)
    if num_pages != caches.num_pages:
        raise ValueError(f"refs has {num_pages} pages, the caches {caches.num_pages}")
    pnt = _dev_tensor(new_table, "new_table", _INTS, block_table.shape)
    pnr = _dev_tensor(new_refs, "new_refs", _INTS, refs.shape)
    pl = _dev_tensor(live, "live", _INTS, (1,))
    if workspace is None:
        with _torch.cuda.stream(stream):  # memory that is `stream`'s (None: the current one's)
            workspace = page_workspace(num_pages, num_seqs, refs.device)
    pw, nw = _workspace(workspace, refs)
    _check((_lib or lib()).wq_cache_compact(caches.array, len(caches.array), caches.page_bytes, pt, pr, pnt, pnr, pl, num_seqs, num_pages,
                                            max_pages, pw, nw, _stream(stream, refs)))


# ------------------------------------------------------- logits to token

def logits_workspace(logits):
    """A device workspace (uint8 tensor, or None) for process_logits."""
    _torch or _load_torch()
    n = ctypes.c_size_t(0)
    _check(lib().wq_process_logits_workspace_size(logits.shape[0], logits.shape[1], _DTYPES[logits.dtype], ctypes.byref(n)))
    return _torch.empty(n.value, dtype=_torch.uint8, device=logits.device) if n.value else None


def _row_stride(t, name, shape):
    """Address and row stride of a device tensor whose rows may lie apart."""
    if isinstance(t, _Tensor) and t.is_cuda and t.shape == shape:
        stride, one = t.stride()
        if one == 1 or shape[1] == 1:
            return t.data_ptr(), stride if shape[0] > 1 else shape[1]
        raise ValueError(f"the rows of {name} must be contiguous")
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def process_logits(logits, out, token=None, mask=None, history=None, history_lens=None, prompt_lens=None, repetition=None,
                   frequency=None, presence=None, bias_ids=None, bias_values=None, bias_lens=None, workspace=None, stream=None) -> None:
    """Penalties, biases and a grammar's mask on logits [R, V] (fp16, bf16 or
    fp32; rows may lie apart), into out (which may be logits), and the best
    word of each row into token (int32 [R], -1 where none is allowed).

    mask [R, ceil(V / 32)] int32/uint32: bit w % 32 of word w / 32 allows word
    w.  history [R, H] int32: the prompt's words (prompt_lens of them), then the
    generated ones (history_lens in all).  repetition, frequency, presence
    fp32 [R].  bias_ids int32 and bias_values fp32 [R, B], bias_lens of them used.
    What is None is left out (include/wq_logits.h has the formulas)."""
    _torch or _load_torch()
    if logits.dim() != 2:
        raise ValueError("logits must be [R, V]")
    shape = logits.shape
    rows, vocab = shape
    kind = _DTYPES.get(logits.dtype)
    if kind is None or out.dtype != logits.dtype:
        raise TypeError(f"logits and out must share one of {tuple(_DTYPES)} (got {logits.dtype}, {out.dtype})")
    px, xs = _row_stride(logits, "logits", shape)
    py, ys = _row_stride(out, "out", shape)
    one = (rows,)
    pt = _dev_tensor(token, "token", _INTS, one) if token is not None else None
    pm = ms = 0
    if mask is not None:
        if mask.dtype not in _WORDS:
            raise TypeError(f"mask has dtype {mask.dtype}, expected one of {_WORDS}")
        pm, ms = _row_stride(mask, "mask", (rows, (vocab + 31) // 32))
    hs = bs = 0
    ph = phl = ppl = pr = pf = pp = pbi = pbv = pbl = None
    if history is not None:
        hs = history.shape[-1]
        ph = _dev_tensor(history, "history", _INTS, (rows, hs))
    if history_lens is not None:
        phl = _dev_tensor(history_lens, "history_lens", _INTS, one)
    if prompt_lens is not None:
        ppl = _dev_tensor(prompt_lens, "prompt_lens", _INTS, one)
    if repetition is not None:
        pr = _dev_tensor(repetition, "repetition", _FLOATS, one)
    if frequency is not None:
        pf = _dev_tensor(frequency, "frequency", _FLOATS, one)
    if presence is not None:
        pp = _dev_tensor(presence, "presence", _FLOATS, one)
    if bias_ids is not None:
        bs = bias_ids.shape[-1]
        pbi = _dev_tensor(bias_ids, "bias_ids", _INTS, (rows, bs))
    if bias_values is not None:
        pbv = _dev_tensor(bias_values, "bias_values", _FLOATS, (rows, bs))
    if bias_lens is not None:
        pbl = _dev_tensor(bias_lens, "bias_lens", _INTS, one)
    if workspace is None and token is not None:
        with _torch.cuda.stream(stream):  # memory that is `stream`'s (None: the current one's)
            workspace = logits_workspace(logits)
    pw, nw = _workspace(workspace, logits)
    call = WqLogitsCall(px, py, pt, pm or None, ph, phl, ppl, pr, pf, pp, pbi, pbv, pbl, rows, vocab, xs, ys, ms, hs, bs, kind)
    _check((_lib or lib()).wq_process_logits(ctypes.addressof(call), pw, nw, _stream(stream, logits)))


# ------------------------------------------------------- measurement probe

def stream_read(buf, sink, stream=None) -> None:
    """Read the whole device tensor `buf` once (wq_stream_read); `sink` is a
    device int32/uint32 tensor of at least 1024 elements."""
    import torch

    if buf.device.type != "cuda" or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous device tensor")
    nbytes = buf.numel() * buf.element_size()
    if sink.device != buf.device or sink.dtype not in (torch.int32, torch.uint32) or sink.numel() < 1024:
        raise ValueError("sink must be a device int32 tensor of at least 1024 elements")
    _torch or _load_torch()
    _check(lib().wq_stream_read(buf.data_ptr(), nbytes, sink.data_ptr(), _unchecked_stream(stream, buf)))
