"""GB300 (sm_103a) MemDecay decode-time eviction loop.

Python binding of ``include/memdecay.h``: the same calls, argument
marshalling only.  Every step of the path runs in the CUDA kernels of
``libmemdecay.so``; there is no CPU or PyTorch fallback, and importing the
binding fails loudly when the library has not been built.  PyTorch provides
device memory (the workspace, input and output tensors) and streams.  The
calls of a decode loop go through a small C module (csrc/md_binding.c); the
others, and arguments it does not take in place, through ctypes.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmemdecay.so")

MD_OK = 0
MD_WARN_OVER_BUDGET = 1
MD_ERR_INVALID_ARG = -1
MD_ERR_CAPACITY = -2
MD_ERR_WORKSPACE = -3
MD_ERR_CUDA = -4
MD_ERR_DEVICE_TIMEOUT = -5
MD_ERR_STATE = -6
STATUS_NAMES = {0: "MD_OK", 1: "MD_WARN_OVER_BUDGET", -1: "MD_ERR_INVALID_ARG", -2: "MD_ERR_CAPACITY",
                -3: "MD_ERR_WORKSPACE", -4: "MD_ERR_CUDA", -5: "MD_ERR_DEVICE_TIMEOUT",
                -6: "MD_ERR_STATE"}

(MD_REGION_SYSTEM, MD_REGION_PLAN, MD_REGION_USER, MD_REGION_TOOL_IN, MD_REGION_TOOL_OUT,
 MD_REGION_RETRIEVAL, MD_REGION_SCRATCHPAD) = range(7)
MD_NUM_REGIONS = 7
MD_MAX_BATCH = 256
MD_HEAD_DIM = 128
MD_MAX_GROUP = 8
MD_MAX_CHUNKS = 64
MD_MAX_CHUNK_TOKENS = 4096

(MD_STATE_BLOCK_TABLE, MD_STATE_PAGE_SCORE, MD_STATE_TOKEN_PRIO, MD_STATE_A, MD_STATE_T_REF,
 MD_STATE_AHAT, MD_STATE_FREE, MD_STATE_REGION, MD_STATE_WINDOW, MD_STATE_MASS, MD_STATE_POOL,
 MD_STATE_T_INS, MD_STATE_PAGE_FILL, MD_STATE_SEQ_TOKENS, MD_STATE_CALIB) = range(15)
MD_CALIB_BUCKETS = 256
MD_CALIB_BUCKET_WIDTH = 4
MD_TYPE_BF16, MD_TYPE_F16, MD_TYPE_F32 = range(3)
MD_MAX_AXES = 4
MD_MAX_TOP_TOKENS = 65536
(MD_QUERY_TOKENS, MD_QUERY_PAGES, MD_QUERY_FREE_TOP, MD_QUERY_STEP, MD_QUERY_WINDOW,
 MD_QUERY_PINNED_PAGES) = range(6)
(MD_DEBUG_SPIN_LIMIT_NS, MD_DEBUG_EXTRA_ARRIVALS, MD_DEBUG_GRID_LIMIT, MD_DEBUG_UNIT_OVERHEAD,
 MD_DEBUG_FORCE_CHUNKS, MD_DEBUG_COMBINE_OVERHEAD, MD_DEBUG_ZERO_COPY, MD_DEBUG_CLUSTER_FORM,
 MD_DEBUG_LOST_TILE) = range(9)
STAGES = ("append", "attention", "fold", "score", "select")


class md_config(ctypes.Structure):
    _fields_ = [
        ("num_layers", ctypes.c_int), ("num_q_heads", ctypes.c_int), ("num_kv_heads", ctypes.c_int),
        ("head_dim", ctypes.c_int), ("page_size", ctypes.c_int),
        ("max_batch", ctypes.c_int), ("max_pages_per_seq", ctypes.c_int), ("num_phys_pages", ctypes.c_int),
        ("rho", ctypes.c_float), ("gamma", ctypes.c_float), ("tau_scale", ctypes.c_float),
        ("attn_weight", ctypes.c_float),
        ("score_mode", ctypes.c_int), ("page_reduce", ctypes.c_int), ("keep_token_prio", ctypes.c_int),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p),
        ("random_seed", ctypes.c_uint64),
        ("region_aligned_pages", ctypes.c_int),
    ]


class md_norm_rope_args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("n_tokens", "num_q_heads", "num_kv_heads", "type", "rotary_dim",
                                             "interleaved", "num_axes", "table_len")] +
                [("eps", ctypes.c_float)] +
                [(n, ctypes.c_void_p) for n in ("q", "k", "v", "q_out", "k_out", "v_out")] +
                [(n, ctypes.c_int64) for n in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head",
                                               "q_out_token", "q_out_head", "k_out_token", "k_out_head",
                                               "v_out_token", "v_out_head")] +
                [(n, ctypes.c_void_p) for n in ("q_weight", "k_weight", "table", "positions", "axis_host", "stream")])


# name -> (restype, argtypes); the names and order of include/memdecay.h
_c = ctypes
_P = _c.c_void_p
SIGNATURES = {
    "md_workspace_size": (_c.c_size_t, [_c.POINTER(md_config)]),
    "md_create": (_c.c_int, [_c.POINTER(md_config), _c.POINTER(_P)]),
    "md_set_region_params": (_c.c_int, [_P, _c.c_int, _c.c_float, _c.c_float, _c.c_int]),
    "md_append_tokens": (_c.c_int, [_P, _c.c_int, _c.c_int, _P, _P, _P, _P]),
    "md_decode_step": (_c.c_int, [_P, _c.c_int, _P, _P, _P, _P, _P]),
    "md_decode_step_host": (_c.c_int, [_P, _c.c_int, _P, _P, _P, _P, _P]),
    "md_decode_layer": (_c.c_int, [_P, _c.c_int, _c.c_int, _P, _P, _P, _P, _P]),
    "md_evict": (_c.c_int, [_P, _c.c_int, _P, _P, _P]),
    "md_sync": (_c.c_int, [_P]),
    "md_destroy": (_c.c_int, [_P]),
    "md_get_state": (_c.c_int, [_P, _c.c_int, _P, _c.c_size_t]),
    "md_set_state": (_c.c_int, [_P, _c.c_int, _P, _c.c_size_t]),
    "md_query": (_c.c_int, [_P, _c.c_int, _c.c_int, _c.POINTER(_c.c_int64)]),
    "md_state_bytes": (_c.c_int, [_P, _c.POINTER(_c.c_size_t), _c.POINTER(_c.c_size_t)]),
    "md_save_state": (_c.c_int, [_P, _P, _P]),
    "md_load_state": (_c.c_int, [_P, _P, _P]),
    "md_profile_enable": (_c.c_int, [_P, _c.c_int]),
    "md_profile_read": (_c.c_int, [_P, _P, _P, _c.c_int]),
    "md_debug_set": (_c.c_int, [_P, _c.c_int, _c.c_int64]),
    "md_calib_enable": (_c.c_int, [_P, _c.c_int]),
    "md_calib_read": (_c.c_int, [_P, _P, _P]),
    "md_calib_fit": (_c.c_int, [_P, _P, _c.c_int, _c.c_int, _c.c_int64, _P, _P]),
    "md_last_error": (_c.c_char_p, [_P]),
    "md_attend_mass_noalloc": (_c.c_int, [_P, _P, _P, _P, _P, _P, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                          _c.c_int, _c.c_int, _c.c_int, _P]),
    "md_rope_table": (_c.c_int, [_P, _c.c_int, _c.c_int, _c.c_double, _P, _P]),
    "md_norm_rope": (_c.c_int, [_c.POINTER(md_norm_rope_args)]),
    "md_page_bounds": (_c.c_int, [_P] * 5 + [_c.c_int] * 6 + [_P]),
    "md_page_scores": (_c.c_int, [_P] * 5 + [_c.c_int] * 7 + [_P]),
    "md_page_top": (_c.c_int, [_P] * 3 + [_c.c_int] * 8 + [_P]),
    "md_attend_pages": (_c.c_int, [_P] * 7 + [_c.c_int] * 8 + [_P]),
    "md_sparse_bytes": (_c.c_size_t, [_c.POINTER(md_config), _c.c_int]),
    "md_sparse_enable": (_c.c_int, [_P, _c.c_int, _c.c_int, _c.c_int, _P, _c.c_size_t]),
}

_lib = None


def lib():
    """The loaded libmemdecay.so.  Raises if it has not been built: there is
    no fallback implementation."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               f"`python -m paper_2607_10582_gb300.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


_fast = None


class _NoCalls:
    """In place of the C module where Python's headers are missing: every call
    is left to ctypes."""

    @staticmethod
    def _leave(*args):
        return None

    decode_step = decode_step_host = decode_layer = evict = get_state = _leave
    load_torch = norm_rope = page_bounds = page_scores = page_top = attend_pages = _leave


def _binding():
    """The C module of the per-step calls, bound to the library.  Raises if it
    could have been built and has not been."""
    global _fast
    if _fast is None:
        lib()
        try:
            from . import _calls as m
            m.load(LIB_PATH)
        except ImportError as e:
            from . import build
            if build.python_include():
                raise RuntimeError("the module _calls is missing: build it with "
                                   "`python -m paper_2607_10582_gb300.build`") from e
            m = _NoCalls
        _fast = m
    return _fast


class MemDecayError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _ptr(x) -> Optional[int]:
    """Device pointer of a torch tensor (or an int / None)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _hptr(x) -> int:
    """Address of a contiguous host buffer: a CPU torch tensor (pinned for
    full copy speed) or a numpy array."""
    if isinstance(x, np.ndarray):
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("host buffer must be contiguous")
        return x.ctypes.data
    if x.is_cuda or not x.is_contiguous():
        raise ValueError("host buffer must be a contiguous CPU tensor")
    return x.data_ptr()


def _host(arr, dtype):
    a = np.ascontiguousarray(np.asarray(arr, dtype=dtype))
    return a, a.ctypes.data


def md_workspace_size(cfg: md_config) -> int:
    return int(lib().md_workspace_size(ctypes.byref(cfg)))


def md_calib_fit(mass_sum: np.ndarray, count: np.ndarray, bucket_width: int = MD_CALIB_BUCKET_WIDTH,
                 min_count: int = 1):
    """Eq. 6-7 fit of a calibration histogram: (rate[7], half_life[7])."""
    s = np.ascontiguousarray(mass_sum, np.float64)
    n = np.ascontiguousarray(count, np.int64)
    rate = np.zeros(MD_NUM_REGIONS)
    half = np.zeros(MD_NUM_REGIONS)
    st = lib().md_calib_fit(s.ctypes.data, n.ctypes.data, s.shape[1], bucket_width, min_count,
                            rate.ctypes.data, half.ctypes.data)
    if st != MD_OK:
        raise MemDecayError(st, "md_calib_fit")
    return rate, half


# ---- rows for the cache, attention over selected pages: calls without a handle ----
# The C module takes a call whose arguments are as its description says; what it leaves
# goes through the checks below, which say what is wrong.
_torch_calls = None


def _ops():
    """The C module with what it needs of torch."""
    global _torch_calls
    if _torch_calls is None:
        import torch
        b = _binding()
        d = os.path.join(os.path.dirname(torch.__file__), "lib")
        b.load_torch(torch.Tensor, torch.nn.Parameter, os.path.join(d, "libtorch_cpu.so"),
                     os.path.join(d, "libtorch_cuda.so"))
        _torch_calls = b
    return _torch_calls


def _bad(what: str):
    raise MemDecayError(MD_ERR_INVALID_ARG, what)


def _here(name, t):
    """Every tensor of a call lies on the current device."""
    import torch
    if t is None:
        _bad(f"{name} is missing")
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        _bad(f"{name} on {t.device}: a tensor on the current device expected")


def _on(t, stream):
    """The stream a call on tensor t goes to (default: the current one of its device)."""
    import torch
    _here("rows or pages", t)
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


_KINDS = {"bf16": ("bfloat16", "int16"), "f32": ("float32",), "i32": ("int32",)}    # int16: raw bf16 bits


def _dense(name, t, shape, kind):
    """Address of a contiguous tensor of this shape and kind on the current device."""
    _here(name, t)
    if tuple(t.shape) != tuple(shape) or str(t.dtype).split(".")[-1] not in _KINDS[kind] or not t.is_contiguous():
        _bad(f"{name}: a contiguous tensor {tuple(shape)} of {kind} expected, not {tuple(t.shape)} of {t.dtype}")
    return t.data_ptr()


def _whole(name, arr, dtype):
    """A host array of this type, each value as it was given."""
    a = np.asarray(arr)
    try:
        with np.errstate(invalid="ignore"):
            b = np.ascontiguousarray(a.astype(dtype))
    except (OverflowError, TypeError, ValueError):
        b = None
    if b is None or not np.array_equal(a, b):
        _bad(f"{name}: whole numbers of {np.dtype(dtype).name} expected")
    return b, b.ctypes.data


def _dims(name, t, n):
    if t is None:
        _bad(f"{name} is missing")
    if t.dim() != n:
        _bad(f"{name}: {n} dimensions expected, not {t.dim()}")
    return t.shape


def _status(st: int, what: str):
    if st != MD_OK:
        raise MemDecayError(st, what)


def md_rope_table(inv_freq, table_len: int, *, scale: float = 1.0, stream=None):
    """Table of a rotation, fp32 [table_len][rotary_dim / 2][2] on the current device:
    scale * (cos, sin) of pos * inv_freq[i], from 64-bit angles.  inv_freq: float64
    [rotary_dim / 2] on the host.  Written on `stream`, which waits for the current stream
    (whose memory the table is); the current stream does not wait for it."""
    import torch
    f, p = _host(inv_freq, np.float64)
    if f.ndim != 1 or table_len < 1:
        _bad("inv_freq must have one dimension, table_len must be positive")
    out = torch.empty((table_len, f.size, 2), dtype=torch.float32, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
        out.record_stream(stream)
    _status(lib().md_rope_table(p, 2 * f.size, table_len, scale, out.data_ptr(), _on(out, stream)), "md_rope_table")
    return out


def _row_types():
    import torch
    return {torch.bfloat16: MD_TYPE_BF16, torch.float16: MD_TYPE_F16, torch.float32: MD_TYPE_F32}


def md_norm_rope(q, k, v, q_out, k_out, v_out, *, positions, table, q_weight=None, k_weight=None, eps: float = 1e-6,
                 axes=None, interleaved: bool = False, stream=None):
    """One layer's rows from a projection's output to what the cache takes: head norms
    (where a weight is given), rotation by position, layout; see md_norm_rope in the header.
      q, k, v      [tokens][heads][128] bf16, f16 or f32, any strides over tokens and heads
                   (parts of one fused tensor); q, or k and v, or v alone may be None
      *_out        the same shapes in bf16 (or its raw bits), any such strides; written
      positions    int32 [tokens] or [num_axes][tokens]
      table        md_rope_table's, or None: no rotation
      axes         uint8 [rotary_dim / 2] on the host: the axis of each pair (None: the first)
      weights      fp32 [128]"""
    st = (_torch_calls or _ops()).norm_rope(q, k, v, q_out, k_out, v_out, positions, table, q_weight, k_weight, eps,
                                             axes, interleaved, None if stream is None else stream.cuda_stream)
    if st is not None:
        return _status(st, "md_norm_rope: head counts, alignment or strides")
    a = md_norm_rope_args()
    types = _row_types()
    first = q if q is not None else k
    if first is None:
        _bad("neither q nor k")
    T = first.shape[0]
    for name, x, y in (("q", q, q_out), ("k", k, k_out), ("v", v, v_out)):
        if x is None:
            continue
        if x.dim() != 3 or x.shape[0] != T or x.shape[2] != MD_HEAD_DIM or x.dtype != first.dtype:
            _bad(f"{name}: {T} tokens of heads of 128 elements, of {first.dtype}, expected")
        if y is None or y.shape != x.shape or str(y.dtype).split(".")[-1] not in ("bfloat16", "int16", "uint16"):
            _bad(f"{name}_out: bf16 (or its raw bits) of the shape of {name} expected")
        _here(name, x)
        _here(name + "_out", y)
        if x.numel() and (x.stride(2) != 1 or y.stride(2) != 1):
            _bad(f"{name}: the elements of a row must be adjacent")
        setattr(a, name, x.data_ptr())
        setattr(a, name + "_out", y.data_ptr())
        for n, s, dim in (("_token", x, 0), ("_head", x, 1), ("_out_token", y, 0), ("_out_head", y, 1)):
            setattr(a, name + n, s.stride(dim) if s.shape[dim] > 1 else 0)
    if first.dtype not in types:
        _bad(f"rows of {first.dtype}")
    if v is not None and (k is None or v.shape != k.shape):
        _bad("v must have k's shape")
    a.n_tokens, a.type, a.eps, a.interleaved = T, types[first.dtype], eps, int(bool(interleaved))
    a.num_q_heads = q.shape[1] if q is not None else 0
    a.num_kv_heads = k.shape[1] if k is not None else 0
    if q is not None and q_weight is not None:
        a.q_weight = _dense("q_weight", q_weight, (MD_HEAD_DIM,), "f32")
    if k is not None and k_weight is not None:
        a.k_weight = _dense("k_weight", k_weight, (MD_HEAD_DIM,), "f32")
    host = None
    if table is not None:
        _dims("table", table, 3)
        a.table = _dense("table", table, (table.shape[0], table.shape[1], 2), "f32")
        a.table_len, a.rotary_dim = table.shape[0], 2 * table.shape[1]
        _here("positions", positions)
        a.num_axes = positions.shape[0] if positions.dim() == 2 else 1
        a.positions = _dense("positions", positions, (a.num_axes, T) if positions.dim() == 2 else (T,), "i32")
        if axes is not None:
            host, a.axis_host = _whole("axes", axes, np.uint8)
            if host.size < table.shape[1]:
                _bad(f"{host.size} axes for {table.shape[1]} pairs")
    a.stream = _on(first, stream)
    _status(lib().md_norm_rope(ctypes.byref(a)), "md_norm_rope: head counts, alignment or strides")


def _counts(n_tokens, batch: int):
    n, p = _whole("token counts or first pages", n_tokens, np.int32)
    if n.size < batch:
        _bad(f"{n.size} token counts for a batch of {batch}")
    return n, p


def md_page_bounds(pool, block_table, n_tokens, bounds, *, first_pages=None, stream=None):
    """Channelwise least and largest key of the pages from first_pages[b] on (None: all).
      pool         bf16 [L][pages][Hkv][2][page_size][128]
      block_table  int32 [batch][max_pages_per_seq]
      n_tokens     int32 [batch] on the host
      bounds       bf16 [L][pages][Hkv][2][128]; written for those pages"""
    st = (_torch_calls or _ops()).page_bounds(pool, block_table, n_tokens, first_pages, bounds,
                                              None if stream is None else stream.cuda_stream)
    if st is not None:
        return _status(st, "md_page_bounds")
    B, P_max = _dims("block_table", block_table, 2)
    L, P, Hkv, _, ps, _ = _dims("pool", pool, 6)
    n, np_ = _counts(n_tokens, B)
    f, fp = (None, None) if first_pages is None else _counts(first_pages, B)
    _status(lib().md_page_bounds(_dense("pool", pool, (L, P, Hkv, 2, ps, MD_HEAD_DIM), "bf16"),
                                 _dense("block_table", block_table, (B, P_max), "i32"), np_, fp,
                                 _dense("bounds", bounds, (L, P, Hkv, 2, MD_HEAD_DIM), "bf16"), B, L, Hkv, ps, P_max, P,
                                 _on(pool, stream)), "md_page_bounds")


def md_page_scores(q, bounds, block_table, n_tokens, scores, *, page_size: int, stream=None):
    """Per page, the largest logit that any query head of a KV head could have on one of its tokens.
      q       bf16 [batch][L][Hq][128]
      bounds  as md_page_bounds writes them
      scores  fp32 [batch][L][Hkv][max_pages_per_seq]; written for each sequence's pages"""
    st = (_torch_calls or _ops()).page_scores(q, bounds, block_table, n_tokens, scores, page_size,
                                              None if stream is None else stream.cuda_stream)
    if st is not None:
        return _status(st, "md_page_scores")
    B, P_max = _dims("block_table", block_table, 2)
    L, P, Hkv = _dims("bounds", bounds, 5)[:3]
    Hq = _dims("q", q, 4)[2]
    n, np_ = _counts(n_tokens, B)
    _status(lib().md_page_scores(_dense("q", q, (B, L, Hq, MD_HEAD_DIM), "bf16"),
                                 _dense("bounds", bounds, (L, P, Hkv, 2, MD_HEAD_DIM), "bf16"),
                                 _dense("block_table", block_table, (B, P_max), "i32"), np_,
                                 _dense("scores", scores, (B, L, Hkv, P_max), "f32"), B, L, Hq, Hkv, page_size, P_max, P,
                                 _on(q, stream)), "md_page_scores")


def md_page_top(scores, n_tokens, page_ids, *, page_size: int, first: int = 1, last: int = 1, stream=None):
    """The pages to attend: the first, the last, and the highest scored of the others.
      scores    fp32 [batch][L][Hkv][max_pages_per_seq]
      page_ids  int32 [batch][L][Hkv][top_pages]; written, in rising order, -1 behind them"""
    st = (_torch_calls or _ops()).page_top(scores, n_tokens, page_ids, page_size, first, last,
                                           None if stream is None else stream.cuda_stream)
    if st is not None:
        return _status(st, "md_page_top")
    B, L, Hkv, P_max = _dims("scores", scores, 4)
    top = _dims("page_ids", page_ids, 4)[3]
    n, np_ = _counts(n_tokens, B)
    _status(lib().md_page_top(_dense("scores", scores, (B, L, Hkv, P_max), "f32"), np_,
                              _dense("page_ids", page_ids, (B, L, Hkv, top), "i32"), B, L, Hkv, page_size, P_max, top,
                              first, last, _on(scores, stream)), "md_page_top")


def md_attend_pages(q, pool, block_table, n_tokens, page_ids, out, *, mass=None, stream=None):
    """Attention of one new token per sequence over the listed pages.
      q, out    bf16 [batch][L][Hq][128]
      page_ids  int32 [batch][L][Hkv][top_pages]
      mass      fp32 [batch][L][Hkv][top_pages * page_size] or None; written"""
    st = (_torch_calls or _ops()).attend_pages(q, pool, block_table, n_tokens, page_ids, out, mass,
                                               None if stream is None else stream.cuda_stream)
    if st is not None:
        return _status(st, "md_attend_pages")
    B, P_max = _dims("block_table", block_table, 2)
    L, P, Hkv, _, ps, _ = _dims("pool", pool, 6)
    Hq, top = _dims("q", q, 4)[2], _dims("page_ids", page_ids, 4)[3]
    n, np_ = _counts(n_tokens, B)
    _status(lib().md_attend_pages(
        _dense("q", q, (B, L, Hq, MD_HEAD_DIM), "bf16"), _dense("pool", pool, (L, P, Hkv, 2, ps, MD_HEAD_DIM), "bf16"),
        _dense("block_table", block_table, (B, P_max), "i32"), np_, _dense("page_ids", page_ids, (B, L, Hkv, top), "i32"),
        _dense("out", out, (B, L, Hq, MD_HEAD_DIM), "bf16"),
        None if mass is None else _dense("mass", mass, (B, L, Hkv, top * ps), "f32"), B, L, Hq, Hkv, ps, P_max, P, top,
        _on(q, stream)), "md_attend_pages")


class Cache:
    """One md_ctx with the workspace it lives in (a torch uint8 tensor on the
    current CUDA device).  Methods map one to one onto the C calls."""

    def __init__(self, num_layers: int, num_q_heads: int, num_kv_heads: int, page_size: int,
                 max_batch: int, max_pages_per_seq: int, num_phys_pages: int, *,
                 rho: float = 0.9, gamma: float = 0.1, tau_scale: float = 2.0,
                 attn_weight: float = 1.0, score_mode: int = 0, page_reduce: int = 0,
                 keep_token_prio: int = 1, random_seed: int = 0, region_aligned_pages: int = 0,
                 stream=None, device=None):
        import torch
        self.torch = torch
        self.device = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        c = md_config(num_layers, num_q_heads, num_kv_heads, MD_HEAD_DIM, page_size,
                      max_batch, max_pages_per_seq, num_phys_pages,
                      rho, gamma, tau_scale, attn_weight, score_mode, page_reduce, keep_token_prio,
                      None, 0, ctypes.c_void_p(self.stream.cuda_stream), random_seed,
                      int(region_aligned_pages))
        need = md_workspace_size(c)
        if need == 0:
            raise MemDecayError(MD_ERR_INVALID_ARG, "invalid configuration")
        # on the handle's stream, the only one that uses it: taken and given up in its order
        with torch.cuda.stream(self.stream):
            self.workspace = torch.empty(need + 1024, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        aligned = (base + 1023) // 1024 * 1024
        c.workspace = aligned
        c.workspace_bytes = need
        self.cfg = c
        self.L, self.Hq, self.Hkv, self.ps = num_layers, num_q_heads, num_kv_heads, page_size
        self.max_batch, self.P_max, self.P_phys = max_batch, max_pages_per_seq, num_phys_pages
        h = ctypes.c_void_p()
        self._check(lib().md_create(ctypes.byref(c), ctypes.byref(h)), None)
        self.h = h
        self._b, self._hv, self._specs = _binding(), h.value, self._state_specs()

    # -- plumbing --
    def _check(self, st: int, h=0, ok=(MD_OK,)):
        if st == MD_OK or st in ok:
            return st
        msg = ""
        if h is not None:
            hh = self.h if h == 0 else h
            msg = lib().md_last_error(hh).decode()
        raise MemDecayError(st, msg)

    def close(self):
        if getattr(self, "h", None):
            lib().md_destroy(self.h)
            self.h = None
            self._hv = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _labels(self, regions, batch: int):
        """The labels as an array the library may read `batch` entries of."""
        regs, p = _host(regions, np.uint8)
        if regs.size < batch <= self.max_batch:
            raise MemDecayError(MD_ERR_INVALID_ARG, f"{regs.size} labels for a batch of {batch}")
        return regs, p

    # -- calls --
    def set_region_params(self, region: int, base: float, half_life: float, pinned: bool):
        return self._check(lib().md_set_region_params(self.h, region, base, half_life, int(pinned)))

    def append_tokens(self, seq: int, regions, k, v, insert_steps=None):
        regs, rp = _host(regions, np.uint8)
        sp = None
        if insert_steps is not None:
            steps, sp = _host(insert_steps, np.int32)
            if steps.size < regs.size:
                raise MemDecayError(MD_ERR_INVALID_ARG, f"{steps.size} insertion steps for {regs.size} labels")
        return self._check(lib().md_append_tokens(self.h, seq, len(regs), rp, sp, _ptr(k), _ptr(v)))

    def decode_step(self, batch: int, q, k_new, v_new, new_regions, out):
        st = self._b.decode_step(self._hv, batch, q, k_new, v_new, new_regions, out)
        if st is not None:
            return self._check(st)
        regs, rp = self._labels(new_regions, batch)
        return self._check(lib().md_decode_step(self.h, batch, _ptr(q), _ptr(k_new), _ptr(v_new), rp, _ptr(out)))

    def decode_step_host(self, batch: int, q, k_new, v_new, new_regions, out):
        """md_decode_step_host: q, k_new, v_new and out are host buffers (CPU
        tensors or numpy arrays, bf16 bits); out is written once the stream
        gets there (sync() or a stream synchronisation)."""
        st = self._b.decode_step_host(self._hv, batch, q, k_new, v_new, new_regions, out)
        if st is not None:
            return self._check(st)
        regs, rp = self._labels(new_regions, batch)
        return self._check(lib().md_decode_step_host(self.h, batch, _hptr(q), _hptr(k_new), _hptr(v_new), rp,
                                                     _hptr(out)))

    def decode_layer(self, layer: int, batch: int, q, k_new, v_new, new_regions, out):
        st = self._b.decode_layer(self._hv, layer, batch, q, k_new, v_new, new_regions, out)
        if st is not None:
            return self._check(st)
        regs, rp = self._labels(new_regions, batch if layer == 0 else 0)
        return self._check(lib().md_decode_layer(self.h, layer, batch, _ptr(q), _ptr(k_new), _ptr(v_new), rp,
                                                 _ptr(out)))

    def evict(self, budgets: Sequence[int], evicted_ids=None):
        st = None
        if type(budgets) is np.ndarray and budgets.ndim == 1:
            n_ev = np.zeros(len(budgets), np.int32)
            st = self._b.evict(self._hv, budgets, n_ev, evicted_ids)
        if st is None:
            bud, bp = _host(budgets, np.int32)
            n_ev = np.zeros(len(bud), np.int32)
            st = lib().md_evict(self.h, len(bud), bp, n_ev.ctypes.data, _ptr(evicted_ids))
        self._check(st, 0, ok=(MD_OK, MD_WARN_OVER_BUDGET))
        return st, n_ev

    def sync(self):
        return lib().md_sync(self.h)

    def query(self, what: int, seq: int = 0) -> int:
        v = ctypes.c_int64()
        self._check(lib().md_query(self.h, what, seq, ctypes.byref(v)))
        return int(v.value)

    def _state_specs(self):
        slots = self.P_phys * self.ps
        t = self.torch
        return {
            MD_STATE_BLOCK_TABLE: ((self.max_batch, self.P_max), t.int32),
            MD_STATE_PAGE_SCORE: ((self.max_batch, self.P_max), t.float32),
            MD_STATE_TOKEN_PRIO: ((slots,), t.float32),
            MD_STATE_A: ((slots,), t.float32),
            MD_STATE_T_REF: ((slots,), t.int32),
            MD_STATE_AHAT: ((slots,), t.float32),
            MD_STATE_FREE: ((self.P_phys,), t.int32),
            MD_STATE_REGION: ((slots,), t.uint8),
            MD_STATE_WINDOW: ((slots,), t.float32),
            MD_STATE_MASS: ((slots,), t.int64),
            MD_STATE_POOL: ((self.L, self.P_phys, self.Hkv, 2, self.ps, MD_HEAD_DIM), t.int16),
            MD_STATE_T_INS: ((slots,), t.int32),
            MD_STATE_PAGE_FILL: ((self.max_batch, self.P_max), t.uint8),
            MD_STATE_SEQ_TOKENS: ((self.max_batch,), t.int32),
            MD_STATE_CALIB: ((8 * MD_CALIB_BUCKETS * 12,), t.uint8),
        }

    def state_spec(self, what: int):
        """(shape, dtype) of a state array."""
        return self._specs[what]

    def get_state(self, what: int):
        shape, dt = self._specs[what]
        out = self.torch.empty(shape, dtype=dt, device=self.device)
        st = self._b.get_state(self._hv, what, out, out.nbytes)
        self._check(lib().md_get_state(self.h, what, out.data_ptr(), out.nbytes) if st is None else st)
        return out

    def set_state(self, what: int, src):
        self._check(lib().md_set_state(self.h, what, src.data_ptr(), src.numel() * src.element_size()))

    def state_bytes(self):
        d, h = ctypes.c_size_t(), ctypes.c_size_t()
        self._check(lib().md_state_bytes(self.h, ctypes.byref(d), ctypes.byref(h)))
        return d.value, h.value

    def save_state(self):
        d, h = self.state_bytes()
        dev = self.torch.empty(d, dtype=self.torch.uint8, device=self.device)
        host = np.zeros(h, np.uint8)
        self._check(lib().md_save_state(self.h, dev.data_ptr(), host.ctypes.data))
        return dev, host

    def load_state(self, saved):
        dev, host = saved
        self._check(lib().md_load_state(self.h, dev.data_ptr(), host.ctypes.data))

    def profile_enable(self, on: bool = True):
        self._check(lib().md_profile_enable(self.h, int(on)))

    def profile_read(self):
        ms = np.zeros(5, np.float64)
        n = np.zeros(5, np.int64)
        self._check(lib().md_profile_read(self.h, ms.ctypes.data, n.ctypes.data, 5))
        return {STAGES[i]: (float(ms[i]), int(n[i])) for i in range(5)}

    def calib_enable(self, on: bool = True):
        self._check(lib().md_calib_enable(self.h, int(on)))

    def calib_read(self):
        """(mass_sum [7][256], count [7][256]) of the calibration histogram."""
        s = np.zeros((MD_NUM_REGIONS, MD_CALIB_BUCKETS), np.float64)
        n = np.zeros((MD_NUM_REGIONS, MD_CALIB_BUCKETS), np.int64)
        self._check(lib().md_calib_read(self.h, s.ctypes.data, n.ctypes.data))
        return s, n

    def sparse_enable(self, top_pages: int, first_pages: int = 1, last_pages: int = 1):
        """md_sparse_enable with a buffer from torch's allocator: decode steps of sequences of
        more than top_pages pages attend that many of them.  0: off."""
        buf, p, n = None, None, 0
        if top_pages:
            n = int(lib().md_sparse_bytes(ctypes.byref(self.cfg), top_pages))
            if n:
                # on the handle's stream, the only one that uses it: taken and given up in its order
                with self.torch.cuda.stream(self.stream):
                    buf = self.torch.empty(n + 256, dtype=self.torch.uint8, device=self.device)
                p = (buf.data_ptr() + 255) // 256 * 256
        self._check(lib().md_sparse_enable(self.h, top_pages, first_pages, last_pages, p, n))
        self.sparse_buffer = buf

    def debug_set(self, key: int, value: int):
        self._check(lib().md_debug_set(self.h, key, value))
