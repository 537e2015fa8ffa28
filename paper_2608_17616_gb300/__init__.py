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
           "mone_cache_attention", "mone_cache_evict")

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
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


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


def make_cache(K, V, table, lens, score=None) -> mone_cache:
    """A paged cache over torch tensors: K, V [layers, pages, KV heads, page_size, head_dim] of any strides with head_dim
    contiguous (K.stride() == V.stride()), table [contexts, width] and lens [contexts] int32, score
    [contexts, layers, KV heads, width * page_size] fp32.  It holds their addresses, not the tensors: keep them alive."""
    if K.stride() != V.stride() or K.shape != V.shape or K.dtype != V.dtype or K.dim() != 5 or K.stride(4) != 1:
        raise ValueError("K and V: [layers, pages, KV heads, page_size, head_dim], the same strides, head_dim contiguous")
    dtype = {"torch.float32": MONE_FP32, "torch.bfloat16": MONE_BF16}.get(str(K.dtype))
    if dtype is None:
        raise ValueError("K and V: float32 or bfloat16")
    for name, t, dims in (("table", table, 2), ("lens", lens, 1), ("score", score, 4)):
        if t is not None and t.dim() != dims:
            raise ValueError(f"{name}: a tensor of {dims} dimensions")
    n_layers, n_pages, n_kv, page, hd = K.shape
    n_ctx, width = table.shape
    _buffer("table", table, "int32", 1, "[contexts, width]")
    _buffer("lens", lens, "int32", n_ctx, "[contexts]")
    if score is not None:
        _buffer("score", score, "float32", 1, "[contexts, layers, KV heads, width * page_size]")
        if score.shape[0] < n_ctx or score.shape[3] != width * page:
            raise ValueError(f"score: [{n_ctx} contexts, layers, KV heads, {width} * {page}], not {tuple(score.shape)}")
    c = mone_cache(_ptr(K), _ptr(V), _LL4(*K.stride()[:4]), n_pages, page, _ptr(table), width, _ptr(lens), _ptr(score))
    c._of = (n_layers, n_ctx, n_kv, hd, dtype, None if score is None else tuple(score.shape[1:3]))
    return c


def _cache(h: int, cache: mone_cache):
    need = _handles.get(h)
    if cache._fits is not need:
        of = cache._of
        if None not in (of, need) and (of[4] != need[4] or any(a < b for a, b in zip(of[:4], need)) or of[5] not in (None, need[0:3:2])):
            raise ValueError(f"the cache's layers, contexts, KV heads, head_dim, dtype (and its score's layers and KV heads) are {of}, "
                             f"the handle's {need}")
        cache._fits = need
    return ctypes.byref(cache)


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


def mone_cache_evict(h: int, layer: int, cache: mone_cache, keep: int, n_sink: int, n_recent: int, to_table, to_score, kept,
                     lens_out=None, stream=None):
    """The first n_sink positions, the last n_recent and the best scored others, `keep` in all, into the pages of to_table
    [contexts, width]; to_score and kept as in the header."""
    width, need = to_table.shape[1], _handles.get(h)
    if need is not None:
        n_layers, n_ctx, n_kv = need[:3]
        per, rows = width * cache.page_size, n_ctx * n_kv
        _buffer("to_table", to_table, "int32", n_ctx * width, "[contexts, width]")
        _buffer("to_score", to_score, "float32", rows * n_layers * per, "[contexts, layers, KV heads, width * page_size]")
        _buffer("kept", kept, "int32", rows * (n_layers if layer == MONE_ALL_LAYERS else 1) * keep, "[contexts, layers, KV heads, keep]")
        if getattr(to_score, "ndim", 0) == 4 and to_score.shape[1:] != (n_layers, n_kv, per):
            raise ValueError(f"to_score: [contexts, {n_layers}, {n_kv}, {per}], not {tuple(to_score.shape)}")
    _check("mone_cache_evict", lib().mone_cache_evict(h, layer, _cache(h, cache), keep, n_sink, n_recent, _ptr(to_table), width,
                                                      _ptr(to_score), _ptr(kept), _ptr(lens_out), _stream(stream)))


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
