"""Python binding of libmone.so (MoNe test-time learning on one GB300 GPU).

Argument marshalling only: every function below forwards to the C entry point
of the same name declared in ``include/mone.h``; all arithmetic runs in the
library's CUDA kernels.  PyTorch tensors are accepted for device buffers (their
``data_ptr()`` is passed) and the current torch CUDA stream is used when no
stream is given.  There is no fallback: if ``libmone.so`` is missing or cannot
be loaded, ``lib()`` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
# MONE_LIB selects another build of the library, e.g. the MONE_DEBUG build (libmone_debug.so)
LIB_PATH = os.environ.get("MONE_LIB") or os.path.join(_PKG, "libmone.so")
DEBUG_LIB_PATH = os.path.join(_PKG, "libmone_debug.so")

MONE_FP32, MONE_BF16 = 0, 1
MONE_PLAIN, MONE_PAPER = 0, 1
MONE_LOSS_DOT, MONE_LOSS_MSE = 0, 1
MONE_MEM_MLP, MONE_MEM_SWIGLU = 0, 1
MONE_RENORM_ROWS, MONE_RENORM_OUT = 0, 1
MONE_GATE_LINEAR, MONE_GATE_SILU = 0, 1
MONE_ROTATE_HALVES, MONE_ROTATE_NEIGHBOURS = 0, 1
MONE_ALL_LAYERS = -1

STATUS = {0: "MONE_OK", 1: "MONE_ERR_INVALID_ARG", 2: "MONE_ERR_UNSUPPORTED_SHAPE", 3: "MONE_ERR_OOM",
          4: "MONE_ERR_CUDA", 5: "MONE_ERR_TIMEOUT", 6: "MONE_ERR_NONFINITE", 7: "MONE_ERR_UNSUPPORTED",
          8: "MONE_ERR_CHECK"}

# Every symbol include/mone.h declares.
EXPORTS = ("mone_mem_init", "mone_ttl_segment", "mone_ttl_context", "mone_mem_generate_kv", "mone_mem_free",
           "mone_mem_read_state", "mone_mem_write_state", "mone_mem_sync", "mone_mem_launch_count",
           "mone_status_string", "mone_abi_version", "mone_mem_set_timing", "mone_mem_kernel_time",
           "mone_last_error", "mone_mem_generate_kv_noalloc", "mone_attention", "mone_mem_kernel_busy",
           "mone_ttl_context_metrics", "mone_ttl_context_host", "mone_window_attention", "mone_cache_append",
           "mone_cache_attention", "mone_cache_evict", "mone_cache4_append", "mone_cache4_read", "mone_cache4_attention",
           "mone_cache4_evict", "mone_cache_reserve", "mone_cache_release", "mone_rotary_make", "mone_norm_rotate")

KERNEL_KINDS = ("prepass", "phase_a", "phase_b", "finalize", "read", "mse", "attention", "resident", "stage",
                 "cache")


class MoneError(RuntimeError):
    def __init__(self, fn: str, code: int, detail: str = ""):
        self.code = code
        super().__init__(f"{fn} failed: {STATUS.get(code, code)}" + (f" ({detail})" if detail else ""))


class mone_config(ctypes.Structure):
    _fields_ = [("n_ctx", ctypes.c_int), ("n_layers", ctypes.c_int), ("d_in", ctypes.c_int),
                ("d_hid", ctypes.c_int), ("d_out", ctypes.c_int), ("n_kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("seg_T", ctypes.c_int), ("dtype", ctypes.c_int),
                ("mode", ctypes.c_int), ("lr", ctypes.c_float), ("rms_eps", ctypes.c_float), ("loss", ctypes.c_int),
                ("memory", ctypes.c_int), ("mem_heads", ctypes.c_int), ("renorm_axis", ctypes.c_int),
                ("gate_act", ctypes.c_int)]


class mone_meta(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("alpha", "gamma", "w_eta", "b_eta", "w_beta", "b_beta", "gate")]


_LL4 = ctypes.c_longlong * 4


class mone_cache(ctypes.Structure):
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("strides", _LL4),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("table", ctypes.c_void_p),
                ("table_width", ctypes.c_int), ("lens", ctypes.c_void_p), ("score", ctypes.c_void_p)]
    _of = None  # make_cache's: its tensors' layers, contexts, KV heads, head_dim, dtype; layers and KV heads of its score
    _fits = None  # the handle's that they were found to do for


class mone_cache4(ctypes.Structure):
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("K_scale", ctypes.c_void_p), ("V_scale", ctypes.c_void_p),
                ("strides", _LL4), ("scale_strides", _LL4), ("k_exp", ctypes.c_int), ("v_exp", ctypes.c_int),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("table", ctypes.c_void_p),
                ("table_width", ctypes.c_int), ("lens", ctypes.c_void_p), ("score", ctypes.c_void_p)]
    _of = None  # make_cache4's, as mone_cache's (no dtype)
    _fits = None


class mone_pages(ctypes.Structure):
    _fields_ = [("free", ctypes.c_void_p), ("n_free", ctypes.c_void_p), ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int),
                ("table", ctypes.c_void_p), ("table_width", ctypes.c_int), ("lens", ctypes.c_void_p)]
    _of = None  # make_pages': its contexts


class mone_rotary(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int), ("pairing", ctypes.c_int), ("period", ctypes.c_int), ("eps", ctypes.c_float),
                ("turns", ctypes.c_ulonglong * 64)]


class mone_heads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("strides", _LL4),
                ("out_strides", _LL4), ("n_heads", ctypes.c_int)]
    _of = None  # make_heads': contexts, layers, tokens, head_dim, dtype, layers of its weight
    _fits = None  # the handle's, whether all layers, and the tokens that they were found to do for


_lib = None
_types = {}  # torch's, by name
_handles = {}  # a live handle's layers, contexts, KV heads, head_dim and dtype


def lib(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libmone.so (once).  Raises OSError when it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise OSError(f"libmone.so not found at {p}; build it with paper_2608_17616_gb300.build.build()")
    L = ctypes.CDLL(p)
    vp, i, ll, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float
    sig = {
        "mone_mem_init": ([ctypes.POINTER(mone_config), vp, vp, ctypes.POINTER(mone_meta), vp,
                           ctypes.POINTER(vp)], i),
        "mone_ttl_segment": ([vp, i, i, vp, vp, vp, i, vp, vp, vp], i),
        "mone_ttl_context": ([vp, vp, vp, vp, ll, vp], i),
        "mone_ttl_context_metrics": ([vp, vp, vp, vp, ll, vp, vp, vp], i),
        "mone_ttl_context_host": ([vp, vp, vp, vp, ll, ll, vp], i),
        "mone_mem_generate_kv": ([vp, vp, i, vp, vp, ctypes.POINTER(ll), vp], i),
        "mone_mem_generate_kv_noalloc": ([vp, vp, i, vp, vp, ctypes.POINTER(ll), vp], i),
        "mone_attention": ([vp, vp, i, i, vp, vp, ctypes.POINTER(ll), i, vp, vp], i),
        "mone_window_attention": ([vp, i, vp, i, i, vp, vp, ctypes.POINTER(ll), i, i, i, vp, vp], i),
        "mone_cache_append": ([vp, i, ctypes.POINTER(mone_cache), vp, vp, ctypes.POINTER(ll), i, vp, vp, vp], i),
        "mone_cache_attention": ([vp, i, ctypes.POINTER(mone_cache), vp, i, i, i, i, vp, vp], i),
        "mone_cache_evict": ([vp, i, ctypes.POINTER(mone_cache), i, i, i, vp, i, vp, vp, vp, vp], i),
        # (structs by address: 0.1 us less a call for each than by a typed pointer)
        "mone_cache4_append": ([vp, i, vp, vp, vp, vp, i, vp, vp, vp], i),
        "mone_cache4_read": ([vp, i, vp, vp, i, vp, vp, vp, vp], i),
        "mone_cache4_attention": ([vp, i, vp, vp, i, i, i, i, vp, vp], i),
        "mone_cache4_evict": ([vp, i, vp, i, i, i, vp, i, vp, vp, vp, vp], i),
        "mone_cache_reserve": ([vp, vp, i, vp, vp, vp, vp, vp, vp], i),
        "mone_cache_release": ([vp, vp, vp, vp, vp, vp], i),
        "mone_rotary_make": ([ctypes.POINTER(mone_rotary), i, i, ctypes.POINTER(ctypes.c_double), ctypes.c_double, i, f], i),
        "mone_norm_rotate": ([vp, i, vp, vp, i, vp, vp, vp], i),
        "mone_mem_free": ([vp], i),
        "mone_mem_read_state": ([vp, vp, vp, vp, vp, vp], i),
        "mone_mem_write_state": ([vp, vp, vp, vp, vp, vp], i),
        "mone_mem_sync": ([vp, vp], i),
        "mone_mem_launch_count": ([vp], ll),
        "mone_status_string": ([i], ctypes.c_char_p),
        "mone_abi_version": ([], i),
        "mone_last_error": ([], ctypes.c_char_p),
        "mone_mem_set_timing": ([vp, i], i),
        "mone_mem_kernel_time": ([vp, i, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ll)], i),
        "mone_mem_kernel_busy": ([vp, i, ctypes.POINTER(ctypes.c_double)], i),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    if path is None:
        _lib = L
    return L


def _ptr(x) -> Optional[int]:
    if x is None or isinstance(x, int):
        return x
    return x.data_ptr()


_address = ctypes.addressof
_strides4 = {}


def _strides(strides: Sequence[int]):
    """Four strides as the library takes them, made once for each value (0.1 us for 0.5 us, where a small operator's call takes 5)."""
    key = strides if type(strides) is tuple else tuple(strides)
    arr = _strides4.get(key)
    if arr is None:
        if len(_strides4) >= 1024:
            _strides4.clear()
        if len(key) != 4:
            raise ValueError("four strides")
        arr = _strides4[key] = _LL4(*key)
    return arr


def _current_stream() -> int:
    """The current torch stream of the current device, without the objects that torch.cuda.current_stream() makes around it
    (0.2 us for 3.0 us a call, where a small operator's whole call takes 8)."""
    global _current_stream
    import torch
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    get, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

    def current() -> int:
        return get(device())

    _current_stream = current
    return current()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(fn: str, rc: int):
    if rc != 0:
        detail = lib().mone_last_error().decode() if rc in (3, 4, 8) else ""
        raise MoneError(fn, rc, detail)


def make_config(n_ctx, n_layers, d_in, d_hid, d_out, n_kv_heads, head_dim, seg_T, dtype, mode, lr,
                rms_eps=1e-6, loss=0, memory=0, mem_heads=1, renorm_axis=0, gate_act=0) -> mone_config:
    return mone_config(n_ctx, n_layers, d_in, d_hid, d_out, n_kv_heads, head_dim, seg_T, dtype, mode, lr, rms_eps,
                       loss, memory, mem_heads, renorm_axis, gate_act)


def make_meta(meta: Optional[dict]) -> Optional[mone_meta]:
    """mone_meta from a dict of device fp32 tensors (keys as in the header)."""
    if meta is None:
        return None
    return mone_meta(*[_ptr(meta.get(k)) for k in ("alpha", "gamma", "w_eta", "b_eta", "w_beta", "b_beta", "gate")])


def mone_mem_init(cfg: mone_config, W1_0, W2_0, meta=None, stream=None) -> int:
    h = ctypes.c_void_p()
    m = make_meta(meta) if isinstance(meta, dict) else meta
    rc = lib().mone_mem_init(ctypes.byref(cfg), _ptr(W1_0), _ptr(W2_0), ctypes.byref(m) if m is not None else None,
                             _stream(stream), ctypes.byref(h))
    _check("mone_mem_init", rc)
    _handles[h.value] = (cfg.n_layers, cfg.n_ctx, cfg.n_kv_heads, cfg.head_dim, cfg.dtype)
    return h.value


def mone_ttl_segment(h: int, ctx: int, layer: int, X, K, V, n_tok: int, eta=None, loss_out=None, stream=None):
    _check("mone_ttl_segment", lib().mone_ttl_segment(h, ctx, layer, _ptr(X), _ptr(K), _ptr(V), n_tok, _ptr(eta),
                                                      _ptr(loss_out), _stream(stream)))


def mone_ttl_context(h: int, X, K, V, N: int, stream=None):
    _check("mone_ttl_context", lib().mone_ttl_context(h, _ptr(X), _ptr(K), _ptr(V), N, _stream(stream)))


def mone_ttl_context_metrics(h: int, X, K, V, N: int, seg_loss=None, seg_step=None, stream=None):
    """mone_ttl_context with per-segment loss and squared step norm ([S][C] fp32 device buffers)."""
    _check("mone_ttl_context_metrics", lib().mone_ttl_context_metrics(h, _ptr(X), _ptr(K), _ptr(V), N, _ptr(seg_loss),
                                                                      _ptr(seg_step), _stream(stream)))


def mone_ttl_context_host(h: int, X, K, V, N: int, chunk_tokens: int = 0, stream=None):
    """mone_ttl_context over host tensors (pinned CPU tensors, or host memory the device reads through
    the host's page tables): the library stages chunks of whole segments into its device windows."""
    _check("mone_ttl_context_host", lib().mone_ttl_context_host(h, _ptr(X), _ptr(K), _ptr(V), N, chunk_tokens,
                                                                _stream(stream)))


def mone_mem_generate_kv(h: int, Xq, Q: int, K_out, V_out, strides: Sequence[int], stream=None):
    arr = (ctypes.c_longlong * 4)(*[int(s) for s in strides])
    _check("mone_mem_generate_kv", lib().mone_mem_generate_kv(h, _ptr(Xq), Q, _ptr(K_out), _ptr(V_out), arr,
                                                              _stream(stream)))


def mone_mem_generate_kv_noalloc(h: int, Xq, Q: int, K_out, V_out, strides: Sequence[int], stream=None):
    """The memory read without any device allocation (fixed 16 MiB library scratch)."""
    arr = (ctypes.c_longlong * 4)(*[int(s) for s in strides])
    _check("mone_mem_generate_kv_noalloc", lib().mone_mem_generate_kv_noalloc(h, _ptr(Xq), Q, _ptr(K_out),
                                                                              _ptr(V_out), arr, _stream(stream)))


def mone_attention(h: int, Q, n_q_heads: int, Lq: int, K, V, kv_strides: Sequence[int], n_mem: int, out,
                   stream=None):
    """Consumer attention of the read (Eq. 5): query tokens over [memory tokens || their own keys]."""
    arr = (ctypes.c_longlong * 4)(*[int(s) for s in kv_strides])
    _check("mone_attention", lib().mone_attention(h, _ptr(Q), n_q_heads, Lq, _ptr(K), _ptr(V), arr, n_mem, _ptr(out),
                                                  _stream(stream)))


def mone_window_attention(h: int, layer: int, Q, n_q_heads: int, Lq: int, K, V, kv_strides: Sequence[int], n_past: int,
                          n_sink: int, window: int, out, stream=None):
    """Attention of a prompt's tokens over the first n_sink positions and the last `window` up to their own."""
    arr = _strides(kv_strides)
    _check("mone_window_attention", lib().mone_window_attention(h, layer, _ptr(Q), n_q_heads, Lq, _ptr(K), _ptr(V), arr, n_past,
                                                                n_sink, window, _ptr(out), _stream(stream)))


def _buffer(name: str, t, dtype: str, at_least: int, shape: str):
    """Refuses a tensor of another type, with gaps or too small (an address is taken as it is)."""
    if not hasattr(t, "is_contiguous"):
        return
    want = _types.get(dtype)
    if want is None:
        import torch
        want = _types[dtype] = getattr(torch, dtype)
    if t.dtype is not want or not t.is_contiguous() or t.numel() < at_least:
        raise ValueError(f"{name}: a contiguous {dtype} tensor {shape}, not {tuple(t.shape)}, {t.dtype}")


def _vector(name: str, t, dtype: str, at_least: int, shape: str) -> Optional[int]:
    """The address of a tensor that _buffer takes; None and addresses as they are."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not _types.get(dtype) or t.numel() < at_least or not t.is_contiguous():
        _buffer(name, t, dtype, at_least, shape)
    return t.data_ptr()


def _tables(table, lens, score, page: int):
    """Checks a cache's table, lengths and scores; contexts and entries of the table."""
    for name, t, dims in (("table", table, 2), ("lens", lens, 1), ("score", score, 4)):
        if t is not None and t.dim() != dims:
            raise ValueError(f"{name}: a tensor of {dims} dimensions")
    n_ctx, width = table.shape
    _buffer("table", table, "int32", 1, "[contexts, width]")
    _buffer("lens", lens, "int32", n_ctx, "[contexts]")
    if score is not None:
        _buffer("score", score, "float32", 1, "[contexts, layers, KV heads, width * page_size]")
        if score.shape[0] < n_ctx or score.shape[3] != width * page:
            raise ValueError(f"score: [{n_ctx} contexts, layers, KV heads, {width} * {page}], not {tuple(score.shape)}")
    return n_ctx, width


def make_cache(K, V, table, lens, score=None) -> mone_cache:
    """A paged cache over torch tensors: K, V [layers, pages, KV heads, page_size, head_dim] of any strides with head_dim
    contiguous (K.stride() == V.stride()), table [contexts, width] and lens [contexts] int32, score
    [contexts, layers, KV heads, width * page_size] fp32.  It holds their addresses, not the tensors: keep them alive."""
    if K.stride() != V.stride() or K.shape != V.shape or K.dtype != V.dtype or K.dim() != 5 or K.stride(4) != 1:
        raise ValueError("K and V: [layers, pages, KV heads, page_size, head_dim], the same strides, head_dim contiguous")
    dtype = {"torch.float32": MONE_FP32, "torch.bfloat16": MONE_BF16}.get(str(K.dtype))
    if dtype is None:
        raise ValueError("K and V: float32 or bfloat16")
    n_layers, n_pages, n_kv, page, hd = K.shape
    n_ctx, width = _tables(table, lens, score, page)
    c = mone_cache(_ptr(K), _ptr(V), _LL4(*K.stride()[:4]), n_pages, page, _ptr(table), width, _ptr(lens), _ptr(score))
    c._of = (n_layers, n_ctx, n_kv, hd, dtype, None if score is None else tuple(score.shape[1:3]))
    return c


def _struct(x, cls) -> int:
    """The address of a struct of this class: it goes to the library untyped."""
    if x.__class__ is not cls and not isinstance(x, cls):
        raise ctypes.ArgumentError(f"expected a {cls.__name__}, not a {type(x).__name__}")
    return _address(x)


def _cache4(h: int, cache) -> int:
    if cache.__class__ is not mone_cache4:
        _struct(cache, mone_cache4)
    return _address(_fitting(h, cache))


def _fitting(h: int, cache):
    need = _handles.get(h)
    if cache._fits is not need:
        of = cache._of
        if None not in (of, need) and (of[4] not in (None, need[4]) or any(a < b for a, b in zip(of[:4], need)) or of[5] not in (None, need[0:3:2])):
            raise ValueError(f"the cache's layers, contexts, KV heads, head_dim, dtype (and its score's layers and KV heads) are {of}, "
                             f"the handle's {need}")
        cache._fits = need
    return cache


def _cache(h: int, cache):
    return ctypes.byref(_fitting(h, cache))


def mone_cache_append(h: int, layer: int, cache: mone_cache, K, V, strides: Sequence[int], n_tok: int, lens_out=None, counts=None,
                      stream=None):
    """New tokens' keys and values after each context's positions."""
    arr = _strides(strides)
    _check("mone_cache_append", lib().mone_cache_append(h, layer, _cache(h, cache), _ptr(K), _ptr(V), arr, n_tok, _ptr(counts),
                                                        _ptr(lens_out), _stream(stream)))


def mone_cache_attention(h: int, layer: int, cache: mone_cache, Q, n_q_heads: int, n_tok: int, n_sink: int, window: int, out,
                         stream=None):
    """Attention of each context's newest n_tok tokens over its pages; with cache.score, the weights are added up there."""
    _check("mone_cache_attention", lib().mone_cache_attention(h, layer, _cache(h, cache), _ptr(Q), n_q_heads, n_tok, n_sink,
                                                              window, _ptr(out), _stream(stream)))


def _targets(h: int, layer: int, page: int, keep: int, to_table, to_score, kept) -> int:
    """Checks an eviction's targets; entries of their table."""
    width, need = to_table.shape[1], _handles.get(h)
    if need is not None:
        n_layers, n_ctx, n_kv = need[:3]
        per, rows = width * page, n_ctx * n_kv
        _buffer("to_table", to_table, "int32", n_ctx * width, "[contexts, width]")
        _buffer("to_score", to_score, "float32", rows * n_layers * per, "[contexts, layers, KV heads, width * page_size]")
        _buffer("kept", kept, "int32", rows * (n_layers if layer == MONE_ALL_LAYERS else 1) * keep, "[contexts, layers, KV heads, keep]")
        if getattr(to_score, "ndim", 0) == 4 and to_score.shape[1:] != (n_layers, n_kv, per):
            raise ValueError(f"to_score: [contexts, {n_layers}, {n_kv}, {per}], not {tuple(to_score.shape)}")
    return width


def mone_cache_evict(h: int, layer: int, cache: mone_cache, keep: int, n_sink: int, n_recent: int, to_table, to_score, kept,
                     lens_out=None, stream=None):
    """The first n_sink positions, the last n_recent and the best scored others, `keep` in all, into the pages of to_table
    [contexts, width]; to_score and kept as in the header."""
    width = _targets(h, layer, cache.page_size, keep, to_table, to_score, kept)
    _check("mone_cache_evict", lib().mone_cache_evict(h, layer, _cache(h, cache), keep, n_sink, n_recent, _ptr(to_table), width,
                                                      _ptr(to_score), _ptr(kept), _ptr(lens_out), _stream(stream)))


def make_cache4(K, V, K_scale, V_scale, table, lens, score=None, k_exp=0, v_exp=0) -> mone_cache4:
    """A paged cache in 4 bits over torch tensors: K, V [layers, pages, KV heads, page_size, head_dim / 2] uint8 of any strides
    with the last dimension contiguous (K.stride() == V.stride()), K_scale, V_scale [.., head_dim / 16] likewise, uint8 or
    float8_e4m3fn; the rest as for make_cache.  It holds their addresses, not the tensors: keep them alive."""
    for x, y in ((K, V), (K_scale, V_scale)):
        if x.stride() != y.stride() or x.shape != y.shape or x.dtype != y.dtype or x.dim() != 5 or x.stride(4) != 1:
            raise ValueError("K and V, and their scales: [layers, pages, KV heads, page_size, head_dim / 2 (/ 16)], the same strides, the "
                             "last dimension contiguous")
    if str(K.dtype) != "torch.uint8" or str(K_scale.dtype) not in ("torch.uint8", "torch.float8_e4m3fn"):
        raise ValueError("codes: uint8; scales: uint8 or float8_e4m3fn")
    n_layers, n_pages, n_kv, page, half = K.shape
    if K_scale.shape[:4] != K.shape[:4] or 8 * K_scale.shape[4] != half:
        raise ValueError(f"scales: {(*K.shape[:4], half // 8)}, not {tuple(K_scale.shape)}")
    n_ctx, width = _tables(table, lens, score, page)
    c = mone_cache4(_ptr(K), _ptr(V), _ptr(K_scale), _ptr(V_scale), _LL4(*K.stride()[:4]), _LL4(*K_scale.stride()[:4]), k_exp, v_exp,
                    n_pages, page, _ptr(table), width, _ptr(lens), _ptr(score))
    c._of = (n_layers, n_ctx, n_kv, 2 * half, None, None if score is None else tuple(score.shape[1:3]))
    return c


def mone_cache4_append(h: int, layer: int, cache: mone_cache4, K, V, strides: Sequence[int], n_tok: int, lens_out=None, counts=None,
                       stream=None):
    """New tokens' keys and values, rounded to 4 bits, after each context's positions."""
    rc = (_lib or lib()).mone_cache4_append(h, layer, _cache4(h, cache), _ptr(K), _ptr(V), _strides(strides), n_tok, _ptr(counts),
                                            _ptr(lens_out), _stream(stream))
    if rc:
        _check("mone_cache4_append", rc)


def mone_cache4_read(h: int, layer: int, cache: mone_cache4, first, n_pos: int, K, V, strides: Sequence[int], stream=None):
    """Positions first[c] .. first[c] + n_pos - 1 (None: from 0) of each context as dense keys and values."""
    rc = (_lib or lib()).mone_cache4_read(h, layer, _cache4(h, cache), _ptr(first), n_pos, _ptr(K), _ptr(V), _strides(strides),
                                          _stream(stream))
    if rc:
        _check("mone_cache4_read", rc)


def mone_cache4_attention(h: int, layer: int, cache: mone_cache4, Q, n_q_heads: int, n_tok: int, n_sink: int, window: int, out,
                          stream=None):
    """mone_cache_attention over a 4-bit cache."""
    rc = (_lib or lib()).mone_cache4_attention(h, layer, _cache4(h, cache), _ptr(Q), n_q_heads, n_tok, n_sink, window, _ptr(out),
                                               _stream(stream))
    if rc:
        _check("mone_cache4_attention", rc)


def mone_cache4_evict(h: int, layer: int, cache: mone_cache4, keep: int, n_sink: int, n_recent: int, to_table, to_score, kept,
                      lens_out=None, stream=None):
    """mone_cache_evict of a 4-bit cache."""
    width = _targets(h, layer, cache.page_size, keep, to_table, to_score, kept)
    rc = (_lib or lib()).mone_cache4_evict(h, layer, _cache4(h, cache), keep, n_sink, n_recent, _ptr(to_table), width, _ptr(to_score),
                                           _ptr(kept), _ptr(lens_out), _stream(stream))
    if rc:
        _check("mone_cache4_evict", rc)


def make_pages(free, n_free, table, lens, page_size: int) -> mone_pages:
    """The free pages of a pool of free.numel() pages and the contexts' tables, int32: free [pages], n_free [1], table
    [contexts, width], lens [contexts].  It holds their addresses, not the tensors: keep them alive."""
    for name, t, dims in (("free", free, 1), ("n_free", n_free, 1), ("table", table, 2), ("lens", lens, 1)):
        if t.dim() != dims:
            raise ValueError(f"{name}: a tensor of {dims} dimensions")
        _buffer(name, t, "int32", 1, f"of {dims} dimensions")
    n_ctx, width = table.shape
    _buffer("lens", lens, "int32", n_ctx, "[contexts]")
    p = mone_pages(_ptr(free), _ptr(n_free), free.numel(), page_size, _ptr(table), width, _ptr(lens))
    p._of = n_ctx
    return p


def _pages(h: int, pages: mone_pages):
    """Checks the pages' contexts; their address and the handle's contexts."""
    at, need = _struct(pages, mone_pages), _handles.get(h)
    if need is None:
        return at, 1
    if pages._of is not None and pages._of < need[1]:
        raise ValueError(f"pages of {pages._of} contexts, the handle has {need[1]}")
    return at, need[1]


def mone_cache_reserve(h: int, pages: mone_pages, n_tok: int, n_free_out, lens_out=None, granted=None, slots=None, counts=None,
                       stream=None):
    """Pages for each context's next n_tok (or counts) tokens from the free list, and the tokens' slots [contexts, n_tok] int64."""
    at, n = _pages(h, pages)
    rc = (_lib or lib()).mone_cache_reserve(h, at, n_tok, _vector("counts", counts, "int32", n, "[contexts]"),
                                  _vector("granted", granted, "int32", n, "[contexts]"),
                                  _vector("slots", slots, "int64", n * n_tok, "[contexts, n_tok]"),
                                  _vector("lens_out", lens_out, "int32", n, "[contexts]"), _vector("n_free_out", n_free_out, "int32", 1, "[1]"),
                                  _stream(stream))
    if rc:
        _check("mone_cache_reserve", rc)


def mone_cache_release(h: int, pages: mone_pages, n_free_out, keep=None, lens_out=None, stream=None):
    """The pages that hold no position below keep (None: 0) back to the free list."""
    at, n = _pages(h, pages)
    rc = (_lib or lib()).mone_cache_release(h, at, _vector("keep", keep, "int32", n, "[contexts]"),
                                  _vector("lens_out", lens_out, "int32", n, "[contexts]"), _vector("n_free_out", n_free_out, "int32", 1, "[1]"),
                                  _stream(stream))
    if rc:
        _check("mone_cache_release", rc)


def make_rotary(rot_dim: int, pairing: int = MONE_ROTATE_HALVES, base: float = 10000.0, freq: Optional[Sequence[float]] = None,
                period: int = 0, eps: float = 1e-6) -> mone_rotary:
    """The rotation of mone_norm_rotate: frequencies freq [rot_dim / 2] in radians per position, or base^(-2 i / rot_dim)."""
    r = mone_rotary()
    if freq is not None and len(freq) != rot_dim // 2:
        raise ValueError(f"freq: {rot_dim // 2} frequencies, not {len(freq)}")
    arr = None if freq is None else (ctypes.c_double * max(len(freq), 1))(*[float(x) for x in freq])
    _check("mone_rotary_make", lib().mone_rotary_make(ctypes.byref(r), rot_dim, pairing, arr, base, period, eps))
    return r


def make_heads(x, out, weight=None) -> mone_heads:
    """One side of mone_norm_rotate: x, out [contexts, the call's layers, heads, tokens, head_dim] of any strides with head_dim contiguous,
    weight [the handle's layers, head_dim] fp32 or None.  It holds their addresses, not the tensors: keep them alive."""
    if x.shape != out.shape or x.dtype != out.dtype or x.dim() != 5 or x.stride(4) != 1 or out.stride(4) != 1:
        raise ValueError("x and out: [contexts, layers, heads, tokens, head_dim], the same type, head_dim contiguous")
    dtype = {"torch.float32": MONE_FP32, "torch.bfloat16": MONE_BF16}.get(str(x.dtype))
    if dtype is None:
        raise ValueError("x and out: float32 or bfloat16")
    if weight is not None:
        _buffer("weight", weight, "float32", 1, "[layers, head_dim]")
        if weight.dim() != 2 or weight.shape[1] != x.shape[4]:
            raise ValueError(f"weight: [layers, {x.shape[4]}], not {tuple(weight.shape)}")
    s = mone_heads(_ptr(x), _ptr(out), _ptr(weight), _LL4(*x.stride()[:4]), _LL4(*out.stride()[:4]), x.shape[2])
    s._of = (x.shape[0], x.shape[1], x.shape[3], x.shape[4], dtype, None if weight is None else weight.shape[0])
    return s


def mone_norm_rotate(h: int, layer: int, rotary: mone_rotary, first, n_tok: int, q: Optional[mone_heads], k: Optional[mone_heads],
                     stream=None):
    """Queries and keys normalised by head and rotated by position; first [contexts] int32: the first token's (None: 0)."""
    rc = (_lib or lib()).mone_norm_rotate(h, layer, _struct(rotary, mone_rotary), _heads(h, layer, n_tok, q, k, first), n_tok,
                                          None if q is None else _address(q), None if k is None else _address(k), _stream(stream))
    if rc:
        _check("mone_norm_rotate", rc)


def _heads(h: int, layer: int, n_tok: int, q: Optional[mone_heads], k: Optional[mone_heads], first) -> Optional[int]:
    """Checks the sides against the handle; the address of first."""
    for side in (q, k):
        if side is not None and side.__class__ is not mone_heads:
            _struct(side, mone_heads)
    need = _handles.get(h)
    if need is None:
        return _ptr(first)
    call = need, layer < 0, n_tok
    for side in (q, k):
        if side is None or side._of is None or side._fits == call:
            continue
        of = side._of
        if (of[0] < need[1] or of[1] < (need[0] if layer == MONE_ALL_LAYERS else 1) or of[2] < n_tok or of[3:5] != need[3:5] or
                (of[5] is not None and of[5] < need[0])):
            raise ValueError(f"contexts, layers, tokens, head_dim, dtype (and the weight's layers) are {of}, the handle's layers, contexts, "
                             f"KV heads, head_dim, dtype {need}")
        side._fits = call
    return _vector("first", first, "int32", need[1], "[contexts]")


def mone_mem_free(h: int):
    _check("mone_mem_free", lib().mone_mem_free(h))
    _handles.pop(h, None)


def mone_mem_read_state(h: int, W1=None, W2=None, mu1=None, mu2=None, stream=None):
    _check("mone_mem_read_state", lib().mone_mem_read_state(h, _ptr(W1), _ptr(W2), _ptr(mu1), _ptr(mu2),
                                                            _stream(stream)))


def mone_mem_write_state(h: int, W1=None, W2=None, mu1=None, mu2=None, stream=None):
    _check("mone_mem_write_state", lib().mone_mem_write_state(h, _ptr(W1), _ptr(W2), _ptr(mu1), _ptr(mu2),
                                                              _stream(stream)))


def mone_mem_sync(h: int, stream=None):
    _check("mone_mem_sync", lib().mone_mem_sync(h, _stream(stream)))


def mone_mem_launch_count(h: int) -> int:
    return lib().mone_mem_launch_count(h)


def mone_status_string(code: int) -> str:
    return lib().mone_status_string(code).decode()


def mone_abi_version() -> int:
    return lib().mone_abi_version()


def mone_last_error() -> str:
    return lib().mone_last_error().decode()


def mone_mem_set_timing(h: int, enable: bool):
    _check("mone_mem_set_timing", lib().mone_mem_set_timing(h, 1 if enable else 0))


def mone_mem_kernel_time(h: int, kind: int):
    """(total device ms, launches) of one kernel kind since timing was enabled."""
    ms = ctypes.c_double()
    n = ctypes.c_longlong()
    _check("mone_mem_kernel_time", lib().mone_mem_kernel_time(h, kind, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def mone_mem_kernel_busy(h: int, kind: int) -> float:
    """Busy time (ms) of one kernel kind since timing was enabled: the union of its launches'
    event intervals, overlapping launches counted once."""
    ms = ctypes.c_double()
    _check("mone_mem_kernel_busy", lib().mone_mem_kernel_busy(h, kind, ctypes.byref(ms)))
    return ms.value


def kv_strides(n_layers: int, n_kv: int, Q: int, head_dim: int):
    """Element strides (ctx, layer, kv_head, q) of a dense [n_ctx][n_layers][n_kv][Q][head_dim] output."""
    return (n_layers * n_kv * Q * head_dim, n_kv * Q * head_dim, Q * head_dim, head_dim)
