"""ctypes binding of libampd.so: argument marshalling only.

Every step of the hot path (append, attention, combine) runs in the library's HIP kernels;
PyTorch is used for device memory and streams.  Function names mirror the C entry points.
"""
from __future__ import annotations

import ctypes
import os
import struct
import types
import warnings
from dataclasses import dataclass

import numpy as np

LIB_PATH = os.environ.get("AMPD_LIB_PATH") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libampd.so")

EXPORTED_SYMBOLS = [
    "ampd_workspace_bytes", "ampd_workspace_bytes_opts", "ampd_kv_append",
    "ampd_incr_prefill_attn", "ampd_mixed_batch_attn", "ampd_incr_prefill_attn_opts",
    "ampd_mixed_batch_attn_opts", "ampd_paged_attn", "ampd_plan_describe", "ampd_plan_items",
    "ampd_set_timing", "ampd_last_timing", "ampd_status_string", "ampd_version", "ampd_kv_pack", "ampd_kv_unpack",
    "ampd_init", "ampd_mixed_batch_attn_static", "ampd_static_workspace_limit",
    "ampd_rope_kv_append", "ampd_page_bounds_update", "ampd_select_pages_workspace_bytes", "ampd_select_pages",
    "ampd_sparse_attn_workspace_bytes", "ampd_sparse_attn",
]

AMPD_KV_BF16, AMPD_KV_FP8_E4M3 = 0, 1


class AmpdError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _Cache(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("num_pages", ctypes.c_int64),
                ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("softmax_scale", ctypes.c_float), ("reserved2", ctypes.c_int32)]


class _Batch(ctypes.Structure):
    _fields_ = [("num_reqs", ctypes.c_int32), ("max_pages_per_req", ctypes.c_int32),
                ("h_ctx_len", ctypes.c_void_p), ("h_incr_len", ctypes.c_void_p),
                ("d_block_table", ctypes.c_void_p), ("h_block_table", ctypes.c_void_p)]


class _Opts(ctypes.Structure):
    _fields_ = [("force_kv_splits", ctypes.c_int32), ("reserved", ctypes.c_int32 * 7)]


class _PlanInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("num_items", "num_wide_items", "num_narrow_items",
                                              "num_combine_items", "num_append_launches",
                                              "partial_bytes", "plan_bytes", "num_append_items", "num_workgroups")]


class _Rope(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("inv_freq", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class _Rows(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v")] + [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride")]


class _Bounds(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class _Selection(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("budget", "first_pages", "last_pages", "group_tokens")] + [("reserved", ctypes.c_int32 * 4)]


HOST_ONLY_SYMBOLS = ["ampd_workspace_bytes", "ampd_workspace_bytes_opts", "ampd_plan_describe", "ampd_plan_items",
                     "ampd_status_string", "ampd_version", "ampd_select_pages_workspace_bytes", "ampd_sparse_attn_workspace_bytes"]


class _HostOnly:
    """Stands in for an entry point that a host-only build of the library (the sanitizer build of the planner and
    of argument validation: AMPD_HOST_ONLY=1 next to AMPD_LIB_PATH) does not hold: attributes can be set, a call raises."""

    def __init__(self, name):
        self._name = name

    def __call__(self, *a):
        raise RuntimeError(f"{self._name} is not part of a host-only build of libampd")


def _declare(f, cp, bp):
    """Result and argument types of the entry points that f holds; cp, bp: of an ampd_kv_cache / ampd_batch argument."""
    vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
    op = ctypes.POINTER(_Opts)
    attn = [cp, bp, vp, vp, vp, vp, vp, sz, vp]
    for name, res, args in (
            ("ampd_workspace_bytes", sz, [cp, bp]),
            ("ampd_workspace_bytes_opts", sz, [cp, bp, op]),
            ("ampd_kv_append", i32, [cp, bp, vp, vp, vp]),
            ("ampd_kv_pack", i32, [cp, bp, i32, i32, vp, vp, vp]),
            ("ampd_kv_unpack", i32, [cp, bp, i32, i32, vp, vp, vp]),
            ("ampd_incr_prefill_attn", i32, attn),
            ("ampd_mixed_batch_attn", i32, attn),
            ("ampd_incr_prefill_attn_opts", i32, attn + [op]),
            ("ampd_mixed_batch_attn_opts", i32, attn + [op]),
            ("ampd_paged_attn", i32, [cp, bp, vp, vp, vp, sz, vp, op]),
            ("ampd_init", i32, []),
            ("ampd_static_workspace_limit", sz, []),
            ("ampd_mixed_batch_attn_static", i32, [cp, bp, vp, vp, vp, vp, vp]),
            ("ampd_plan_describe", i32, [cp, bp, op, ctypes.POINTER(_PlanInfo)]),
            ("ampd_plan_items", i64, [cp, bp, op, vp, i64]),
            ("ampd_set_timing", None, [ctypes.c_int]),
            ("ampd_last_timing", i32, [ctypes.POINTER(ctypes.c_float)] * 3),
            ("ampd_rope_kv_append", i32, [cp, bp, vp, vp, vp, vp, vp]),
            ("ampd_page_bounds_update", i32, [cp, bp, vp, vp]),
            ("ampd_select_pages_workspace_bytes", sz, [cp, bp, vp]),
            ("ampd_select_pages", i32, [cp, bp, vp, vp, vp, vp, vp, sz, vp]),
            ("ampd_sparse_attn_workspace_bytes", sz, [cp, bp, i32, i32]),
            ("ampd_sparse_attn", i32, [cp, bp, vp, i32, i32, vp, vp, vp, sz, vp]),
            ("ampd_status_string", ctypes.c_char_p, [i32]),
            ("ampd_version", ctypes.c_char_p, [])):
        fn = getattr(f, name)
        fn.restype = res
        fn.argtypes = args


def _load():
    """The library, and its entry points once more as functions that take the two structures by address."""
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2602_14516_amd/build.py` "
                          "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    packed = types.SimpleNamespace()
    host_only = os.environ.get("AMPD_HOST_ONLY") == "1"
    for name in EXPORTED_SYMBOLS:
        if host_only and name not in HOST_ONLY_SYMBOLS:
            setattr(L, name, _HostOnly(name))
            setattr(packed, name, _HostOnly(name))
        else:
            setattr(packed, name, L[name])          # a function object of its own
    _declare(L, ctypes.POINTER(_Cache), ctypes.POINTER(_Batch))
    _declare(packed, ctypes.c_void_p, ctypes.c_void_p)
    return L, packed


lib, _packed = _load()


def status_string(s: int) -> str:
    return lib.ampd_status_string(int(s)).decode()


def version() -> str:
    return lib.ampd_version().decode()


def _ptr(t):
    """Device/host address of a torch tensor or numpy array (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


@dataclass
class KVCache:
    """Shape of a paged pool plus the (torch, device) tensors that back it.

    k_pool / v_pool: [num_pages, Hkv, P, d]; dtype bfloat16 (or int16/uint16 bit patterns)
    for a bf16 cache, uint8 for an E4M3 cache (then k_scale / v_scale: float32 [num_pages, Hkv]).
    """
    num_q_heads: int
    num_kv_heads: int
    head_dim: int
    page_size: int
    k_pool: object
    v_pool: object
    softmax_scale: float
    k_scale: object = None
    v_scale: object = None
    kv_dtype: int = AMPD_KV_BF16

    def c_struct(self, with_pools=True) -> _Cache:
        num_pages = int(self.k_pool.shape[0]) if self.k_pool is not None else int(getattr(self, "num_pages_hint", 1))
        return _Cache(self.num_q_heads, self.num_kv_heads, self.head_dim, self.page_size, self.kv_dtype, 0,
                      num_pages, _ptr(self.k_pool), _ptr(self.v_pool), _ptr(self.k_scale), _ptr(self.v_scale),
                      float(self.softmax_scale), 0)


def _batch(ctx_len, incr_len, block_table_dev, block_table_host=None, max_pages=None):
    ctx = np.ascontiguousarray(ctx_len, dtype=np.int32)
    inc = np.ascontiguousarray(incr_len, dtype=np.int32)
    assert ctx.shape == inc.shape and ctx.ndim == 1
    if block_table_dev is not None:
        max_pages = int(block_table_dev.shape[1]) if block_table_dev.ndim == 2 else int(max_pages)
    bth = None
    if block_table_host is not None:
        bth = np.ascontiguousarray(block_table_host, dtype=np.int32)
    b = _Batch(ctx.shape[0], int(max_pages or 0), ctx.ctypes.data, inc.ctypes.data,
               _ptr(block_table_dev), None if bth is None else bth.ctypes.data)
    return b, (ctx, inc, bth)          # keep the host arrays alive for the duration of the call


# The two structures of a call as packed bytes, which the functions in _packed take by address (lib's own take the structures and
# check their types).  A decode step of one row takes 9 us on the
# GPU, and building the ctypes structures (numpy's .ctypes, one conversion per field) took a third of the 14.5 us that calls of it
# were apart; packed, they are 10.5 us apart (one short prefill 13.2 -> 10.4, a pack and an unpack of 8 700 tokens 20.8 -> 18.3).
_pack_cache = struct.Struct("@6iq4Pfi").pack
_pack_batch = struct.Struct("@2i4P").pack
_char_at = ctypes.c_char.from_buffer
_addressof = ctypes.addressof
_INT32 = np.dtype(np.int32)


def _cache_arg(c: KVCache):
    """The ampd_kv_cache argument of a call."""
    try:
        return _pack_cache(c.num_q_heads, c.num_kv_heads, c.head_dim, c.page_size, c.kv_dtype, 0, c.k_pool.shape[0],
                           _ptr(c.k_pool) or 0, _ptr(c.v_pool) or 0, _ptr(c.k_scale) or 0, _ptr(c.v_scale) or 0,
                           c.softmax_scale, 0)
    except (struct.error, OverflowError, TypeError, AttributeError):      # a value that only the field's own conversion takes
        return ctypes.byref(c.c_struct())


def _host_addr(a: np.ndarray) -> int:
    try:
        return _addressof(_char_at(a))
    except (TypeError, ValueError, BufferError):                          # read-only or empty
        return a.ctypes.data


def _batch_arg(ctx_len, incr_len, block_table_dev, block_table_host=None):
    """The ampd_batch argument of a call, and the host arrays it points into (to be kept until the call has returned)."""
    ctx, inc = np.ascontiguousarray(ctx_len, _INT32), np.ascontiguousarray(incr_len, _INT32)
    if block_table_host is not None or block_table_dev is None or block_table_dev.ndim != 2:
        b, keep = _batch(ctx, inc, block_table_dev, block_table_host)
        return ctypes.byref(b), keep
    assert ctx.shape == inc.shape and ctx.ndim == 1
    return _pack_batch(len(ctx), block_table_dev.shape[1], _host_addr(ctx), _host_addr(inc), _ptr(block_table_dev) or 0, 0), (ctx, inc)


# Calls with arguments of the usual kind go through an extension module (csrc/fastcall.cpp), which fills the two structures itself and
# answers None, before anything is called, for the others; those take the functions below.  Once the smallest launches take 6.5 us on the
# GPU, 3 us of interpreted marshalling in front of 4 us of library and launch kept them 7.9 us apart.
_fastcall = None                 # (call, addresses of the entry points, module) after the first use; False: there is no such module


def _load_fastcall():
    if os.environ.get("AMPD_HOST_ONLY") == "1":
        return False
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None or not hasattr(torch._C, "_cuda_getDevice") or not hasattr(torch._C, "_cuda_isInBadFork"):
        return False
    try:
        from . import _fastcall as module
        built_for = getattr(module, "torch_version", "an older one")
        if built_for != torch.__version__:
            raise ImportError(f"built for torch {built_for}, not {torch.__version__}")
    except ImportError as e:                                              # not built, or for another Python or torch
        warnings.warn(f"paper_2602_14516_amd: calls are marshalled without the extension module, 3 us slower each ({e}); "
                      "python paper_2602_14516_amd/build.py builds it", RuntimeWarning)
        return False
    module.streams(torch._C._cuda_getDevice, raw, torch._C._cuda_isInBadFork)
    return module.call, {n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in EXPORTED_SYMBOLS}, module


def _fast(name, *args):
    """The status of an entry point called that way, or None."""
    global _fastcall
    if _fastcall is None:
        _fastcall = _load_fastcall()
    if not _fastcall:
        return None
    call, address, _ = _fastcall
    return call(address[name], *args)


def _fast_sparse(function, name, *args):
    """The same through the module's function for an operator of sparse attention, which checks the tensors too."""
    global _fastcall
    if _fastcall is None:
        _fastcall = _load_fastcall()
    if not _fastcall:
        return None
    return getattr(_fastcall[2], function)(_fastcall[1][name], *args)


def _opts(force_kv_splits=0):
    if not force_kv_splits:
        return None
    o = _Opts()
    o.force_kv_splits = int(force_kv_splits)
    return ctypes.byref(o)


def _stream_ptr(stream):
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)        # without a Stream object around it: 1.5 us less
        return raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(st, where):
    if st != 0:
        raise AmpdError(int(st), where)


def workspace_bytes(cache: KVCache, ctx_len, incr_len, max_pages, force_kv_splits=0) -> int:
    b, keep = _batch(ctx_len, incr_len, None, max_pages=max_pages)
    c = cache.c_struct()
    return int(lib.ampd_workspace_bytes_opts(ctypes.byref(c), ctypes.byref(b), _opts(force_kv_splits)))


def plan_describe(cache: KVCache, ctx_len, incr_len, max_pages, force_kv_splits=0) -> dict:
    b, keep = _batch(ctx_len, incr_len, None, max_pages=max_pages)
    c = cache.c_struct()
    info = _PlanInfo()
    _check(lib.ampd_plan_describe(ctypes.byref(c), ctypes.byref(b), _opts(force_kv_splits), ctypes.byref(info)),
           "ampd_plan_describe")
    return {n: int(getattr(info, n)) for n, _ in _PlanInfo._fields_}


def plan_items(cache: KVCache, ctx_len, incr_len, max_pages, force_kv_splits=0) -> np.ndarray:
    """int32 [n, 10]: request, kind, kv_head, first_head_in_group, heads, first_token, tokens, key_begin,
    key_end, partial_offset."""
    b, keep = _batch(ctx_len, incr_len, None, max_pages=max_pages)
    c = cache.c_struct()
    o = _opts(force_kv_splits)
    n = int(lib.ampd_plan_items(ctypes.byref(c), ctypes.byref(b), o, None, 0))
    if n < 0:
        raise AmpdError(n, "ampd_plan_items")
    items = np.zeros((n, 10), dtype=np.int32)
    if n:
        lib.ampd_plan_items(ctypes.byref(c), ctypes.byref(b), o, items.ctypes.data, n)
    return items


def kv_append(cache: KVCache, ctx_len, incr_len, block_table, k_new, v_new, *, stream=None,
              block_table_host=None) -> None:
    if stream is None and block_table_host is None:
        st = _fast("ampd_kv_append", cache, ctx_len, incr_len, block_table, k_new, v_new)
        if st is not None:
            return _check(st, "ampd_kv_append")
    b, keep = _batch_arg(ctx_len, incr_len, block_table, block_table_host)
    c = _cache_arg(cache)
    _check(_packed.ampd_kv_append(c, b, _ptr(k_new), _ptr(v_new), _stream_ptr(stream)),
           "ampd_kv_append")


def kv_pack(cache: KVCache, first_token, num_tokens, block_table, head_begin, head_count, k_out, v_out, *, stream=None,
            block_table_host=None) -> None:
    """Pages -> packed rows [sum tokens, head_count, d] for KV heads [head_begin, head_begin + head_count)."""
    if stream is None and block_table_host is None:
        st = _fast("ampd_kv_pack", cache, first_token, num_tokens, block_table, head_begin, head_count, k_out, v_out)
        if st is not None:
            return _check(st, "ampd_kv_pack")
    b, keep = _batch_arg(first_token, num_tokens, block_table, block_table_host)
    c = _cache_arg(cache)
    _check(_packed.ampd_kv_pack(c, b, int(head_begin), int(head_count), _ptr(k_out), _ptr(v_out),
                            _stream_ptr(stream)), "ampd_kv_pack")


def kv_unpack(cache: KVCache, first_token, num_tokens, block_table, head_begin, head_count, k_in, v_in, *, stream=None,
              block_table_host=None) -> None:
    """Packed rows -> pages, the inverse of kv_pack."""
    if stream is None and block_table_host is None:
        st = _fast("ampd_kv_unpack", cache, first_token, num_tokens, block_table, head_begin, head_count, k_in, v_in)
        if st is not None:
            return _check(st, "ampd_kv_unpack")
    b, keep = _batch_arg(first_token, num_tokens, block_table, block_table_host)
    c = _cache_arg(cache)
    _check(_packed.ampd_kv_unpack(c, b, int(head_begin), int(head_count), _ptr(k_in), _ptr(v_in),
                              _stream_ptr(stream)), "ampd_kv_unpack")


def _temp_workspace(need, q, stream):
    """A workspace for one call: allocated, and later returned to torch's caching allocator, on the stream the call
    runs on, so that the block cannot be handed out again while that stream still uses it."""
    import torch
    if stream is None or isinstance(stream, int):
        # a raw hipStream_t cannot be named to the allocator: the caller passes workspace= in that case
        if isinstance(stream, int) and stream != torch.cuda.current_stream().cuda_stream:
            raise ValueError("pass workspace= when stream= is a raw stream handle other than torch's current stream")
        return torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    with torch.cuda.stream(stream):
        return torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)


def _attn_call(fn_name, cache, ctx_len, incr_len, block_table, q, k_new, v_new, out, workspace, stream,
               block_table_host, force_kv_splits):
    if workspace is not None and out is not None and stream is None and block_table_host is None and not force_kv_splits:
        st = _fast(fn_name + "_opts", cache, ctx_len, incr_len, block_table, q, k_new, v_new, out, workspace)
        if st is not None:
            _check(st, fn_name)
            return out
    import torch
    b, keep = _batch_arg(ctx_len, incr_len, block_table, block_table_host)
    c = _cache_arg(cache)
    o = _opts(force_kv_splits)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        need = int(_packed.ampd_workspace_bytes_opts(c, b, o))
        workspace = _temp_workspace(need, q, stream)
    fn = getattr(_packed, fn_name + "_opts")
    _check(fn(c, b, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(workspace),
              workspace.numel() * workspace.element_size(), _stream_ptr(stream), o), fn_name)
    return out


def incr_prefill_attn(cache: KVCache, ctx_len, incr_len, block_table, q, k_new, v_new, *, out=None,
                      workspace=None, stream=None, block_table_host=None, force_kv_splits=0):
    """Append k_new/v_new, then causal GQA attention of the new queries; returns out (bf16 [sum L, Hq, d])."""
    return _attn_call("ampd_incr_prefill_attn", cache, ctx_len, incr_len, block_table, q, k_new, v_new, out,
                      workspace, stream, block_table_host, force_kv_splits)


def mixed_batch_attn(cache: KVCache, ctx_len, incr_len, block_table, q, k_new, v_new, *, out=None,
                     workspace=None, stream=None, block_table_host=None, force_kv_splits=0):
    """The same for a batch mixing decode rows (L=1) and prefill rows (L>1): one fused attention launch."""
    return _attn_call("ampd_mixed_batch_attn", cache, ctx_len, incr_len, block_table, q, k_new, v_new, out,
                      workspace, stream, block_table_host, force_kv_splits)


def init() -> None:
    """One-time set-up of the current device (pins the staging ring, resolves the static workspace)."""
    _check(lib.ampd_init(), "ampd_init")


def static_workspace_limit() -> int:
    return int(lib.ampd_static_workspace_limit())


def mixed_batch_attn_static(cache: KVCache, ctx_len, incr_len, block_table, q, k_new, v_new, out, *, stream=None,
                            block_table_host=None):
    """mixed_batch_attn on the library's static workspace: the call allocates nothing (out is required)."""
    b, keep = _batch_arg(ctx_len, incr_len, block_table, block_table_host)
    c = _cache_arg(cache)
    _check(_packed.ampd_mixed_batch_attn_static(c, b, _ptr(q), _ptr(k_new), _ptr(v_new),
                                            _ptr(out), _stream_ptr(stream)), "ampd_mixed_batch_attn_static")
    return out


def paged_attn(cache: KVCache, ctx_len, incr_len, block_table, q, *, out=None, workspace=None, stream=None,
               block_table_host=None, force_kv_splits=0):
    """Attention only; the pools must already hold all C + L tokens of every row."""
    import torch
    b, keep = _batch_arg(ctx_len, incr_len, block_table, block_table_host)
    c = _cache_arg(cache)
    o = _opts(force_kv_splits)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        need = int(_packed.ampd_workspace_bytes_opts(c, b, o))
        workspace = _temp_workspace(need, q, stream)
    _check(_packed.ampd_paged_attn(c, b, _ptr(q), _ptr(out), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream_ptr(stream), o),
           "ampd_paged_attn")
    return out


# ---- sparse attention over a long cache ----------------------------------------------------------------------------------


@dataclass
class Rope:
    """Position rotation: the inverse frequencies (torch, device, float32 [rotary_dim / 2]) and how elements are paired:
    (j, j + rotary_dim / 2), or (2j, 2j + 1) when interleaved.  scale multiplies cosine and sine."""
    inv_freq: object
    interleaved: bool = False
    scale: float = 1.0


@dataclass
class PageBounds:
    """Per (page, KV head) the largest and smallest stored key of every channel in 8 bits: codes int8 [num_pages, Hkv, 2, d],
    scale float32 [num_pages, Hkv] (torch, device)."""
    codes: object
    scale: object


def _want(name, t, dtype, shape=None):
    """Refuse a tensor that the library would read as something else: type, shape, order."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != getattr(torch, dtype):
        raise ValueError(f"{name}: a torch tensor of {dtype} is wanted, not {getattr(t, 'dtype', type(t).__name__)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor is wanted (strides {tuple(t.stride())} for {tuple(t.shape)})")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: {tuple(shape)} is wanted, not {tuple(t.shape)}")


def _same_device(named):
    """The library enqueues on the current GPU: everything has to live there."""
    import torch
    dev = None
    for name, t in named:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name}: device memory is wanted, not a tensor on {t.device}")
        if dev is None:
            dev = torch.cuda.current_device()
        if t.device.index != dev:
            raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")


def _want_table(block_table, rows):
    _want("block_table", block_table, "int32")
    if block_table.ndim != 2 or block_table.shape[0] != rows:
        raise ValueError(f"block_table: one row for each of {rows} requests is wanted, not {tuple(block_table.shape)}")


def _want_pools(cache: KVCache):
    fp8 = cache.kv_dtype == AMPD_KV_FP8_E4M3
    n = cache.k_pool.shape[0]
    shape = (n, cache.num_kv_heads, cache.page_size, cache.head_dim)
    for name, t in (("k_pool", cache.k_pool), ("v_pool", cache.v_pool)):
        if t.element_size() != (1 if fp8 else 2) or not t.is_contiguous() or tuple(t.shape) != shape:
            raise ValueError(f"{name}: {shape}, contiguous, {1 if fp8 else 2} bytes an element is wanted, not {tuple(t.shape)} of {t.dtype}")
    if fp8:
        _want("k_scale", cache.k_scale, "float32", (n, cache.num_kv_heads))
        _want("v_scale", cache.v_scale, "float32", (n, cache.num_kv_heads))


def _want_bounds(cache: KVCache, bounds: PageBounds):
    n = cache.k_pool.shape[0] if cache.k_pool is not None else bounds.codes.shape[0]
    _want("bounds.codes", bounds.codes, "int8", (n, cache.num_kv_heads, 2, cache.head_dim))
    _want("bounds.scale", bounds.scale, "float32", (n, cache.num_kv_heads))


def _want_workspace(workspace):
    if not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor is wanted (strides {tuple(workspace.stride())} for {tuple(workspace.shape)})")


def _rows(name, t, tokens, heads, d):
    """[tokens, heads, d] with the heads of a token next to each other: elements from token to token."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16 or tuple(t.shape) != (tokens, heads, d):
        raise ValueError(f"{name}: bfloat16 {(tokens, heads, d)} is wanted, not {getattr(t, 'dtype', type(t).__name__)} {tuple(getattr(t, 'shape', ()))}")
    s = t.stride()
    if tokens and (s[2] != 1 or heads > 1 and s[1] != d):
        raise ValueError(f"{name}: the heads of a token have to lie next to each other (strides {tuple(s)})")
    return int(s[0]) if tokens > 1 else heads * d


def _lengths(ctx_len, incr_len):
    ctx, inc = np.ascontiguousarray(ctx_len, _INT32), np.ascontiguousarray(incr_len, _INT32)
    if ctx.shape != inc.shape or ctx.ndim != 1:
        raise ValueError(f"ctx_len and incr_len: two vectors of one length are wanted, not {ctx.shape} and {inc.shape}")
    return ctx, inc


def _output(name, shape, dtype, q, stream):
    """A result of a call on `stream`, from that stream's memory."""
    import torch
    if isinstance(stream, int) and stream != torch.cuda.current_stream().cuda_stream:
        raise ValueError(f"pass {name}= when stream= is a raw stream handle other than torch's current stream")
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else None):
        return torch.empty(shape, dtype=getattr(torch, dtype), device=q.device)


def _int32(name, x):
    """A number that the library takes in 32 bits (ctypes would cut it)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name}: {x} does not fit 32 bits")
    return x


def num_groups(incr_len, group_tokens=1) -> int:
    """Groups of group_tokens consecutive new tokens that a batch has: rows of a selection."""
    if _int32("group_tokens", group_tokens) < 1:
        raise ValueError(f"group_tokens: at least 1 is wanted, not {group_tokens}")
    L = np.asarray(incr_len, dtype=np.int64)
    return int((-(-L // int(group_tokens))).sum())


def rope_kv_append(cache: KVCache, ctx_len, incr_len, block_table, rope: Rope, q, k_new, v_new, *, q_out=None, positions=None, bounds=None,
                   stream=None, block_table_host=None):
    """Rotate q and k_new by their positions and append k_new, v_new; returns the rotated queries (bf16 [sum L, Hq, d]).

    q [sum L, Hq, d], k_new and v_new [sum L, Hkv, d] may be views of one projection's rows (a token's heads next to each other);
    q None: keys and values alone.  q_out may be q where that is contiguous.  positions: int32 [sum L], device (None: token i of a
    row is at ctx_len + i).  bounds: PageBounds, set for the pages that receive tokens."""
    if q_out is not None and stream is None and block_table_host is None:
        st = _fast_sparse("rope", "ampd_rope_kv_append", cache, ctx_len, incr_len, block_table, rope, q, k_new, v_new, q_out, positions, bounds)
        if st is not None:
            _check(st, "ampd_rope_kv_append")
            return q_out
    ctx, inc = _lengths(ctx_len, incr_len)
    n = int(inc.sum())
    _want_table(block_table, len(ctx))
    _want_pools(cache)
    d = cache.head_dim
    _want("inv_freq", rope.inv_freq, "float32")
    if rope.inv_freq.ndim != 1:
        raise ValueError(f"inv_freq: a vector is wanted, not {tuple(rope.inv_freq.shape)}")
    strides = [0 if q is None else _rows("q", q, n, cache.num_q_heads, d), _rows("k_new", k_new, n, cache.num_kv_heads, d),
               _rows("v_new", v_new, n, cache.num_kv_heads, d)]
    if positions is not None:
        _want("positions", positions, "int32", (n,))
    if bounds is not None:
        _want_bounds(cache, bounds)
    if q is not None and q_out is None:
        q_out = _output("q_out", (n, cache.num_q_heads, d), "bfloat16", q, stream)
    if q is not None:
        _want("q_out", q_out, "bfloat16", (n, cache.num_q_heads, d))
    _same_device((("k_pool", cache.k_pool), ("v_pool", cache.v_pool), ("k_scale", cache.k_scale), ("v_scale", cache.v_scale),
                  ("block_table", block_table), ("inv_freq", rope.inv_freq), ("q", q), ("k_new", k_new), ("v_new", v_new), ("q_out", q_out if q is not None else None),
                  ("positions", positions), ("bounds", None if bounds is None else bounds.codes), ("bounds", None if bounds is None else bounds.scale)))
    b, keep = _batch_arg(ctx, inc, block_table, block_table_host)
    ro = _Rope(2 * rope.inv_freq.shape[0], int(bool(rope.interleaved)), _ptr(rope.inv_freq), _ptr(positions), float(rope.scale), 0)
    rows = _Rows(_ptr(q), _ptr(k_new), _ptr(v_new), *strides)
    bo = None if bounds is None else ctypes.byref(_Bounds(_ptr(bounds.codes), _ptr(bounds.scale)))
    _check(_packed.ampd_rope_kv_append(_cache_arg(cache), b, ctypes.byref(ro), ctypes.byref(rows), None if q is None else _ptr(q_out), bo, _stream_ptr(stream)),
           "ampd_rope_kv_append")
    return q_out if q is not None else None


def page_bounds_update(cache: KVCache, ctx_len, incr_len, block_table, bounds: PageBounds, *, stream=None, block_table_host=None) -> None:
    """Set the bounds of every page that holds some of a row's tokens ctx_len .. ctx_len + incr_len, from the keys it stores."""
    if stream is None and block_table_host is None:
        st = _fast_sparse("page_bounds", "ampd_page_bounds_update", cache, ctx_len, incr_len, block_table, bounds)
        if st is not None:
            return _check(st, "ampd_page_bounds_update")
    ctx, inc = _lengths(ctx_len, incr_len)
    _want_table(block_table, len(ctx))
    _want_pools(cache)
    _want_bounds(cache, bounds)
    _same_device((("k_pool", cache.k_pool), ("k_scale", cache.k_scale), ("block_table", block_table), ("bounds", bounds.codes), ("bounds", bounds.scale)))
    b, keep = _batch_arg(ctx, inc, block_table, block_table_host)
    _check(_packed.ampd_page_bounds_update(_cache_arg(cache), b, ctypes.byref(_Bounds(_ptr(bounds.codes), _ptr(bounds.scale))), _stream_ptr(stream)),
           "ampd_page_bounds_update")


def _selection(budget, first_pages, last_pages, group_tokens):
    return _Selection(_int32("budget", budget), _int32("first_pages", first_pages), _int32("last_pages", last_pages), _int32("group_tokens", group_tokens),
                      (ctypes.c_int32 * 4)())


def select_pages_workspace_bytes(cache: KVCache, ctx_len, incr_len, max_pages, budget, *, first_pages=1, last_pages=1, group_tokens=1) -> int:
    b, keep = _batch(ctx_len, incr_len, None, max_pages=max_pages)
    c = cache.c_struct()
    s = _selection(budget, first_pages, last_pages, group_tokens)
    return int(lib.ampd_select_pages_workspace_bytes(ctypes.byref(c), ctypes.byref(b), ctypes.byref(s)))


def select_pages(cache: KVCache, ctx_len, incr_len, block_table, bounds: PageBounds, q, budget, *, first_pages=1, last_pages=1, group_tokens=1,
                 out=None, workspace=None, stream=None, block_table_host=None):
    """The `budget` pages of a row that every group of group_tokens new tokens attends, per KV head, chosen by their bounds: int32
    [num_groups, Hkv, budget], logical page indices in ascending order, -1 behind.  The first first_pages, and the last last_pages up to
    the group's own, are always among them.  q: the rotated queries, bf16 [sum L, Hq, d]."""
    if out is not None and workspace is not None and stream is None and block_table_host is None:
        st = _fast_sparse("select_pages", "ampd_select_pages", cache, ctx_len, incr_len, block_table, bounds, q, budget, first_pages, last_pages,
                          group_tokens, out, workspace)
        if st is not None:
            _check(st, "ampd_select_pages")
            return out
    ctx, inc = _lengths(ctx_len, incr_len)
    _want_table(block_table, len(ctx))
    _want_bounds(cache, bounds)
    _want("q", q, "bfloat16", (int(inc.sum()), cache.num_q_heads, cache.head_dim))
    s = _selection(budget, first_pages, last_pages, group_tokens)
    shape = (num_groups(inc, group_tokens), cache.num_kv_heads, int(budget))
    if out is None:
        out = _output("out", shape, "int32", q, stream)
    _want("out", out, "int32", shape)
    b, keep = _batch_arg(ctx, inc, block_table, block_table_host)
    c = _selecting_cache(cache, bounds)
    if workspace is None:
        workspace = _temp_workspace(int(_packed.ampd_select_pages_workspace_bytes(c, b, ctypes.byref(s))), q, stream)
    _want_workspace(workspace)
    _same_device((("block_table", block_table), ("bounds", bounds.codes), ("bounds", bounds.scale), ("q", q), ("out", out), ("workspace", workspace)))
    _check(_packed.ampd_select_pages(c, b, ctypes.byref(_Bounds(_ptr(bounds.codes), _ptr(bounds.scale))), ctypes.byref(s), _ptr(q), _ptr(out), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "ampd_select_pages")
    return out


def _selecting_cache(cache: KVCache, bounds: PageBounds):
    """The cache argument of a call that reads no pool: it may have none."""
    if cache.k_pool is not None:
        return _cache_arg(cache)
    c = cache.c_struct()
    c.num_pages = bounds.codes.shape[0]
    return ctypes.byref(c)


def sparse_attn_workspace_bytes(cache: KVCache, ctx_len, incr_len, max_pages, budget, *, group_tokens=1) -> int:
    b, keep = _batch(ctx_len, incr_len, None, max_pages=max_pages)
    c = cache.c_struct()
    return int(lib.ampd_sparse_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(b), _int32("budget", budget), _int32("group_tokens", group_tokens)))


def sparse_attn(cache: KVCache, ctx_len, incr_len, block_table, selected, q, *, group_tokens=1, out=None, workspace=None, stream=None,
                block_table_host=None):
    """Attention of every new token over the keys up to its own position on the pages that its group's row of `selected` (int32 [num_groups,
    Hkv, budget], as select_pages returns it) names; the pools must already hold all tokens.  Returns out (bf16 [sum L, Hq, d])."""
    if out is not None and workspace is not None and stream is None and block_table_host is None:
        st = _fast_sparse("sparse_attn", "ampd_sparse_attn", cache, ctx_len, incr_len, block_table, selected, q, group_tokens, out, workspace)
        if st is not None:
            _check(st, "ampd_sparse_attn")
            return out
    ctx, inc = _lengths(ctx_len, incr_len)
    _want_table(block_table, len(ctx))
    _want_pools(cache)
    shape = (int(inc.sum()), cache.num_q_heads, cache.head_dim)
    _want("q", q, "bfloat16", shape)
    _want("selected", selected, "int32")
    if selected.ndim != 3 or tuple(selected.shape[:2]) != (num_groups(inc, group_tokens), cache.num_kv_heads):
        raise ValueError(f"selected: [{num_groups(inc, group_tokens)}, {cache.num_kv_heads}, budget] is wanted, not {tuple(selected.shape)}")
    budget = _int32("budget", selected.shape[2])
    if out is None:
        out = _output("out", shape, "bfloat16", q, stream)
    _want("out", out, "bfloat16", shape)
    b, keep = _batch_arg(ctx, inc, block_table, block_table_host)
    c = _cache_arg(cache)
    if workspace is None:
        workspace = _temp_workspace(int(_packed.ampd_sparse_attn_workspace_bytes(c, b, budget, int(group_tokens))), q, stream)
    _want_workspace(workspace)
    _same_device((("k_pool", cache.k_pool), ("v_pool", cache.v_pool), ("k_scale", cache.k_scale), ("v_scale", cache.v_scale), ("block_table", block_table),
                  ("selected", selected), ("q", q), ("out", out), ("workspace", workspace)))
    _check(_packed.ampd_sparse_attn(c, b, _ptr(selected), budget, int(group_tokens), _ptr(q), _ptr(out), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "ampd_sparse_attn")
    return out


def set_timing(enabled: bool) -> None:
    lib.ampd_set_timing(1 if enabled else 0)


def last_timing():
    """(attention ms, combine ms, append+plan-copy ms) of the last call on this thread; sync the stream first."""
    a, c, p = ctypes.c_float(), ctypes.c_float(), ctypes.c_float()
    _check(lib.ampd_last_timing(ctypes.byref(a), ctypes.byref(c), ctypes.byref(p)), "ampd_last_timing")
    return a.value, c.value, p.value
