"""Thin Python binding of include/cacheback.h (argument marshalling only).

Every step of the path runs in libcacheback.so's CUDA kernels; this module only
turns torch tensors into pointers, sizes and strides.  If the library is missing
the import of `CacheBack` fails loudly: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from array import array
from typing import Optional, Sequence

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libcacheback.so")

CB_OK, CB_EINVAL, CB_ESHAPE, CB_EBUDGET, CB_ENOMEM, CB_ECUDA, CB_ETIMEOUT, CB_EDEVICE = range(8)
STATUS_NAMES = ["CB_OK", "CB_EINVAL", "CB_ESHAPE", "CB_EBUDGET", "CB_ENOMEM", "CB_ECUDA", "CB_ETIMEOUT",
                "CB_EDEVICE"]

# Every entry point include/cacheback.h declares (checked by the tests).
EXPORTED = ["cb_config_init", "cb_create", "cb_score", "cb_budget", "cb_select", "cb_compact",
            "cb_sync_status", "cb_destroy", "cb_last_error", "cb_scratch_bytes", "cb_score_path", "cb_select_noalloc",
            "cb_select_noalloc_status", "cb_gather", "cb_chain_budget", "cb_compact_rope",
            "cb_enable_stage_timing", "cb_stage_times", "cb_set_wait_limit", "cb_set_score_sms",
            "cb_create_receiver", "cb_rotary", "cb_pack", "cb_unpack", "cb_attend"]


class CBError(RuntimeError):
    def __init__(self, status: int, message: str):
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__("%s: %s" % (name, message))
        self.status = status


class cb_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("max_query_tokens", ctypes.c_int32),
                ("max_positions", ctypes.c_int64), ("max_senders", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("p", ctypes.c_float), ("alpha", ctypes.c_float),
                ("pool_width", ctypes.c_int32), ("span_width", ctypes.c_int32),
                ("n_sink", ctypes.c_int32), ("n_latent", ctypes.c_int32), ("score_kernel", ctypes.c_int32)]


class cb_kv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("T", ctypes.c_int64),
                ("s_layer", ctypes.c_int64), ("s_head", ctypes.c_int64), ("s_pos", ctypes.c_int64),
                ("pages", ctypes.c_void_p), ("page_size", ctypes.c_int32), ("s_page", ctypes.c_int64),
                ("n_pages", ctypes.c_int64)]


class cb_query(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("m", ctypes.c_int32), ("s_layer", ctypes.c_int64),
                ("s_tok", ctypes.c_int64), ("s_head", ctypes.c_int64), ("k_self", ctypes.c_void_p),
                ("ks_layer", ctypes.c_int64), ("ks_tok", ctypes.c_int64), ("ks_head", ctypes.c_int64)]


class cb_rope(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("style", ctypes.c_int32), ("dims", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("factor", ctypes.c_double), ("original", ctypes.c_int64),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double), ("attention", ctypes.c_double),
                ("inverse", ctypes.c_int32)]


class cb_packed(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("T", ctypes.c_int64), ("s_layer", ctypes.c_int64),
                ("s_head", ctypes.c_int64), ("s_pos", ctypes.c_int64), ("pages", ctypes.c_void_p),
                ("page_size", ctypes.c_int32), ("s_page", ctypes.c_int64), ("n_pages", ctypes.c_int64),
                ("length", ctypes.c_void_p)]


_LIB = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libcacheback.so (built by paper_2609_32046_gb300.build); raises if absent."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ImportError("libcacheback.so is not built (%s); run `python -m paper_2609_32046_gb300.build` "
                          "or __graft_entry__.build()" % p)
    lib = ctypes.CDLL(p)
    P = ctypes.c_void_p
    lib.cb_config_init.argtypes = [ctypes.POINTER(cb_config)]
    lib.cb_config_init.restype = None
    lib.cb_create.argtypes = [ctypes.POINTER(cb_config), ctypes.POINTER(P)]
    lib.cb_create.restype = ctypes.c_int
    lib.cb_score.argtypes = [P, ctypes.c_int32, ctypes.POINTER(cb_kv), ctypes.POINTER(cb_query), P, P]
    lib.cb_score.restype = ctypes.c_int
    lib.cb_budget.argtypes = [ctypes.c_int64, ctypes.c_double]
    lib.cb_budget.restype = ctypes.c_int64
    lib.cb_chain_budget.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_double, ctypes.c_int32, ctypes.c_int64]
    lib.cb_chain_budget.restype = ctypes.c_int64
    lib.cb_select.argtypes = [P, ctypes.c_int32, P, P, P, P, P]
    lib.cb_select.restype = ctypes.c_int
    lib.cb_compact.argtypes = [P, ctypes.c_int32, ctypes.POINTER(cb_kv), P, P, P, P, ctypes.c_int64, P,
                               ctypes.c_int64, ctypes.c_int64, P]
    lib.cb_compact.restype = ctypes.c_int
    lib.cb_compact_rope.argtypes = [P, ctypes.c_int32, ctypes.POINTER(cb_kv), P, P, P, P, ctypes.c_int64, P,
                                    ctypes.c_int64, ctypes.c_int64, ctypes.c_double, ctypes.c_int32,
                                    ctypes.c_int64, P]
    lib.cb_compact_rope.restype = ctypes.c_int
    lib.cb_gather.argtypes = [P, ctypes.c_int32, P, P, ctypes.c_int64, ctypes.c_int64, P, P, P, ctypes.c_int64, P,
                              ctypes.c_int64, P]
    lib.cb_gather.restype = ctypes.c_int
    lib.cb_sync_status.argtypes = [P, P]
    lib.cb_sync_status.restype = ctypes.c_int
    lib.cb_destroy.argtypes = [P]
    lib.cb_destroy.restype = None
    lib.cb_last_error.argtypes = [P]
    lib.cb_last_error.restype = ctypes.c_char_p
    lib.cb_scratch_bytes.argtypes = [P]
    lib.cb_scratch_bytes.restype = ctypes.c_int64
    lib.cb_score_path.argtypes = [P]
    lib.cb_score_path.restype = ctypes.c_int32
    lib.cb_select_noalloc.argtypes = [ctypes.c_int32, P, P, P, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P]
    lib.cb_select_noalloc.restype = ctypes.c_int
    lib.cb_set_wait_limit.argtypes = [P, ctypes.c_int64, ctypes.c_int32]
    lib.cb_set_wait_limit.restype = ctypes.c_int
    lib.cb_set_score_sms.argtypes = [P, ctypes.c_int32]
    lib.cb_set_score_sms.restype = ctypes.c_int
    lib.cb_select_noalloc_status.argtypes = [P]
    lib.cb_select_noalloc_status.restype = ctypes.c_int
    lib.cb_enable_stage_timing.argtypes = [P, ctypes.c_int32]
    lib.cb_enable_stage_timing.restype = ctypes.c_int
    lib.cb_stage_times.argtypes = [P, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]
    lib.cb_stage_times.restype = ctypes.c_int
    lib.cb_create_receiver.argtypes = lib.cb_create.argtypes
    lib.cb_create_receiver.restype = ctypes.c_int
    lib.cb_rotary.argtypes = [P, ctypes.c_int32, P, ctypes.POINTER(cb_rope), P]
    lib.cb_rotary.restype = ctypes.c_int
    lib.cb_pack.argtypes = [P, ctypes.c_int32, P, P, P, P, P, P,
                            ctypes.c_int32, ctypes.c_int32, P]
    lib.cb_pack.restype = ctypes.c_int
    lib.cb_unpack.argtypes = [P, ctypes.c_int32, P, P, P, P, P, ctypes.c_int64, P,
                              ctypes.c_int64, ctypes.c_int64, P]
    lib.cb_unpack.restype = ctypes.c_int
    lib.cb_attend.argtypes = [P, ctypes.c_int32, ctypes.c_int32, P, P, ctypes.c_int32, ctypes.c_int64, P]
    lib.cb_attend.restype = ctypes.c_int
    if path is None:
        _LIB = lib
    return lib


def budget(T: int, keep: float) -> int:
    """ceil(keep * T) in double, clamped to [0, T] (App. C.2), computed by the library."""
    return int(load_library().cb_budget(int(T), float(keep)))


def chain_budget(T_old: int, T_new: int, keep: float = 0.0, mode: str = "relative", B_max: int = 0) -> int:
    """Budget of one hop of a sequential chain (App. C.2): relative T_old + ceil(keep T_new) or
    fixed min(B_max, T_old + T_new), computed by the library."""
    m = {"relative": 0, "fixed": 1}[mode]
    b = int(load_library().cb_chain_budget(int(T_old), int(T_new), float(keep), m, int(B_max)))
    if b < 0:
        raise ValueError("invalid chain budget arguments")
    return b


def select_noalloc(scores: Sequence, Ts: Sequence[int], budgets: Sequence[int], idx: Sequence, n_sink: int = 1,
                   n_latent: int = 40, span_width: int = 16, stream=None):
    """cb_select_noalloc: selection without a context and without device allocation."""
    lib = load_library()
    n = len(scores)
    st = lib.cb_select_noalloc(n, _ptr_array([s.data_ptr() for s in scores]),
                               _ptr_array(list(map(int, Ts)), ctypes.c_int64),
                               _ptr_array(list(map(int, budgets)), ctypes.c_int64),
                               _ptr_array([x.data_ptr() for x in idx]), n_sink, n_latent, span_width,
                               _stream_handle(stream))
    if st != CB_OK:
        raise CBError(st, lib.cb_last_error(None).decode())


def select_noalloc_status(stream=None):
    """cb_select_noalloc_status: wait for the stream and raise if the allocation-free selection's
    kernel check failed since the last read."""
    lib = load_library()
    st = lib.cb_select_noalloc_status(_stream_handle(stream))
    if st != CB_OK:
        raise CBError(st, lib.cb_last_error(None).decode())


def _ptr_array(values, ctype=ctypes.c_void_p):
    return (ctype * len(values))(*values)


_torch_cuda = None
_raw_stream = None


def _stream_handle(stream) -> int:
    if stream is None:
        global _torch_cuda
        if _torch_cuda is None:
            import torch
            _torch_cuda = torch.cuda
        return _torch_cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _stream_on(stream, tensor) -> int:
    """The stream's handle; None: torch's current stream of the tensor's device."""
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    if not tensor.is_cuda:
        return _stream_handle(None)       # (the call refuses the tensor)
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = torch._C._cuda_getCurrentRawStream
    return _raw_stream(tensor.device.index)


class PagedKV:
    """A sender cache in the paged (block-table) layout of a vLLM-style server (App. F).

    k_pool, v_pool: bf16 tensors indexed [l][page][row][g][k] (vLLM's per-layer
                    [n_pages][page_size][Hkv][d] caches stacked over layers, or any view with
                    that index order and a unit head-dim stride; both with the same strides)
    pages:          int32 device tensor, pages[b] = the page holding positions
                    b * page_size .. b * page_size + page_size - 1 (the sequence's block table)
    T:              positions cached
    Quacks like the [nL][Hkv][T][d] tensor it stands for (shape, dtype, device), so it can be
    passed wherever a sender's K is expected; kv_desc(p) describes both pools.
    """

    def __init__(self, k_pool, v_pool, pages, T: int):
        assert k_pool.dim() == 5 and k_pool.dtype.itemsize == 2 and k_pool.stride(4) == 1
        assert v_pool.shape == k_pool.shape and v_pool.stride() == k_pool.stride()
        nL, n_pages, P, Hkv, d = k_pool.shape
        assert P & (P - 1) == 0, "page_size must be a power of two"
        assert pages.dtype.itemsize == 4 and pages.is_contiguous() and pages.numel() >= (T + P - 1) // P
        self.k_pool, self.v_pool, self.pages, self.T = k_pool, v_pool, pages, int(T)
        self.page_size, self.n_pages = P, n_pages
        self.shape = (nL, Hkv, int(T), d)
        self.dtype = k_pool.dtype
        self.device = k_pool.device

    def desc(self) -> cb_kv:
        k = self.k_pool
        return cb_kv(k.data_ptr(), self.v_pool.data_ptr(), self.T, k.stride(0), k.stride(3), k.stride(2),
                     self.pages.data_ptr(), self.page_size, k.stride(1), self.n_pages)


def kv_desc(K, V=None) -> cb_kv:
    """K, V: bf16 [nL][Hkv][T][d] (any strides with unit head-dim stride), or K a PagedKV
    (V ignored: the PagedKV holds both pools)."""
    if isinstance(K, PagedKV):
        return K.desc()
    st = K.stride()
    assert K.element_size() == 2 and st[3] == 1
    if V is None:
        return cb_kv(K.data_ptr(), None, K.size(2), st[0], st[1], st[2])
    assert V.stride() == st and V.size() == K.size()
    return cb_kv(K.data_ptr(), V.data_ptr(), K.size(2), st[0], st[1], st[2])


def query_desc(Q, Kself=None) -> cb_query:
    """Q: bf16 [nL][m][Hq][d]; Kself (optional): the query tokens' own keys, bf16 [nL][m][Hkv][d]."""
    st = Q.stride()
    assert Q.element_size() == 2 and st[3] == 1
    if Kself is None:
        return cb_query(Q.data_ptr(), Q.size(1), st[0], st[1], st[2])   # (the rest: no own keys)
    ks = Kself.stride()
    assert Kself.element_size() == 2 and ks[3] == 1 and Kself.size(1) == Q.size(1)
    return cb_query(Q.data_ptr(), Q.size(1), st[0], st[1], st[2], Kself.data_ptr(), ks[0], ks[1], ks[2])


class PackedKV:
    """A cache or message held in 4 bits (cb_packed): codes c in -7..7 and one scale s for every 32
    neighbouring elements of a row; an element's value is c * s.

    k, v:                uint8 codes, [nL][Hkv][T][d / 2]; paged: [nL][n_pages][page_size][Hkv][d / 2]
    k_scale, v_scale:    bf16 scales, the same index order with d / 32 in the last place; any strides
                         that step over rows alike in codes and scales
    T:                   rows cached (default: all there is room for); may be assigned as the cache grows, as `length` may
    pages:               int32 device tensor of a paged cache (the sequence's block table); may be assigned as well, a
                         table that has room for T rows
    length:              optional int32 device tensor of one element: CacheBack.attend reads the first
                         min(T, length) rows, as it is when the kernel runs
    `capacity` is the number of rows there is room for (pack writes below it).  The arrays themselves are the
    cache's for good (k, v, k_scale and v_scale cannot be assigned): other arrays are another PackedKV.
    """

    GROUP = 32

    def __init__(self, k, v, k_scale, v_scale, T: Optional[int] = None, pages=None, length=None):
        paged = pages is not None
        dims = 5 if paged else 4
        _require(all(x.dim() == dims for x in (k, v, k_scale, v_scale)), "codes and scales need %d dimensions" % dims)
        _require(k.element_size() == v.element_size() == 1 and _is_bf16(k_scale) and _is_bf16(v_scale),
                 "codes are bytes and scales bf16")
        _require(k.shape == v.shape and k_scale.shape == v_scale.shape and k.shape[:-1] == k_scale.shape[:-1] and
                 k.shape[-1] == 16 * k_scale.shape[-1], "codes hold d / 2 and scales d / 32 elements of the same rows")
        kd, sd = k.shape[-1], k_scale.shape[-1]
        shape, kt, st = k.shape, k.stride(), k_scale.stride()
        like = v.stride() == kt and v_scale.stride() == st and kt[-1] == st[-1] == 1     # (nearly always)
        for a, b, c in zip(shape[:-1], kt, st):
            like = like and b % kd == 0 and b // kd * sd == c
        for x, n in () if like else ((k, kd), (v, kd), (k_scale, sd), (v_scale, sd)):
            _require(x.stride(-1) == 1, "rows are contiguous")
            # (the stride of a dimension of one entry says nothing)
            _require(all(a == 1 or (s % n == 0 and s // n == t // kd) for a, s, t in zip(shape[:-1], x.stride()[:-1], kt[:-1])),
                     "codes and scales of K and V need the same strides in rows")
        self._arrays = (k, v, k_scale, v_scale)
        self.head_dim = 2 * kd
        self.device = k.device
        if paged:
            self.page_size, self.n_pages = shape[2], shape[1]
            _require(self.page_size & (self.page_size - 1) == 0, "page_size must be a power of two")
            self.n_layers, self.n_kv_heads = shape[0], shape[3]
            order = (0, 3, 2)
        else:
            self.n_layers, self.n_kv_heads, self.capacity = shape[:3]
            order = (0, 1, 2)
        row = [kt[i] // kd * self.head_dim if shape[i] > 1 else self.head_dim for i in order]
        self._page = (kt[1] // kd * self.head_dim if shape[1] > 1 else self.head_dim) if paged else 0
        # the description with its T left open (bytes of a cb_packed are copied faster than fields are set)
        d = cb_packed(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), 0, row[0], row[1], row[2])
        if paged:
            d.page_size, d.s_page, d.n_pages = self.page_size, self._page, self.n_pages
        self._desc = d
        # the rows cached, and what _described makes of them once it is asked: an assignment puts a new list in its
        # place, so that a call of another thread never leaves the bytes of one state in the next
        self._state = [0, None]
        self._pages = None
        if paged:
            self._set_pages(pages)
        self.length = length
        self._shape = (self.n_layers, self.n_kv_heads, self.head_dim)
        self.T = self.capacity if T is None else T

    @classmethod
    def empty(cls, n_layers: int, n_kv_heads: int, T: int, head_dim: int, device=None) -> "PackedKV":
        """Room for T rows (whose contents are undefined until they are packed)."""
        import torch
        row = (n_layers, n_kv_heads, T)
        return cls(*[torch.empty(row + (head_dim // 2,), dtype=torch.uint8, device=device) for _ in range(2)],
                   *[torch.empty(row + (head_dim // 32,), dtype=torch.bfloat16, device=device) for _ in range(2)])

    @property
    def bytes(self) -> int:
        """Bytes that T rows take (codes and scales of K and V, every layer and head)."""
        return 2 * self.n_layers * self.n_kv_heads * self.T * (self.head_dim // 2 + self.head_dim // 16)

    # what a description holds the addresses of (`p.k_scale *= 2` puts back the array it took)
    def _put_back(self, x, i):
        if x is not self._arrays[i]:
            raise AttributeError("a cache's arrays are its own for good: make another PackedKV")

    k, v, k_scale, v_scale = (property(lambda self, i=i: self._arrays[i], lambda self, x, i=i: self._put_back(x, i))
                              for i in range(4))

    @property
    def pages(self):
        return self._pages

    @pages.setter
    def pages(self, pages):
        _require(self._pages is not None and pages is not None, "a cache is paged, or not, for good")
        self._set_pages(pages)

    def _set_pages(self, pages):
        _require(_is_int32(pages) and pages.dim() == 1 and pages.is_contiguous(), "pages are a row of int32")
        _require(self.T <= pages.numel() * self.page_size, "the block table has no room for T rows")
        self._pages = pages
        self.capacity = pages.numel() * self.page_size
        self._desc.pages = pages.data_ptr()
        self._state = [self.T, None]

    @property
    def T(self) -> int:
        return self._state[0]

    @T.setter
    def T(self, T: int):
        if not 0 <= T <= self.capacity:
            raise ValueError("T = %d not in [0, %d]" % (T, self.capacity))
        self._state = [int(T), None]

    @property
    def length(self):
        return self._length

    @length.setter
    def length(self, x):
        _require(x is None or (_is_int32(x) and x.numel() == 1), "length is one int32")
        self._length = x
        self._desc.length = None if x is None else x.data_ptr()
        self._state = [self.T, None]

    def _described(self) -> bytes:
        """The bytes of desc(): a call joins those of its caches."""
        state = self._state
        if state[1] is None:
            state[1] = bytes(self.desc(state[0]))
        return state[1]

    def desc(self, T: Optional[int] = None) -> cb_packed:
        """A description of its own, with T rows (default: those cached)."""
        d = cb_packed.from_buffer_copy(self._desc)
        d.T = self.T if T is None else T
        return d


class Rotary:
    """A rotary embedding (cb_rope): base, pairs as "halves" (k, k + dims / 2) or "pairs" (2k, 2k + 1),
    `dims` rotary elements of a head (0: all), scaling "none", "linear" or "yarn" (by parts) by `factor`
    over `original` positions; attention 0 takes the scaling's own factor of cosine and sine."""

    STYLES = {"halves": 0, "pairs": 1, 0: 0, 1: 1}
    SCALINGS = {"none": 0, "linear": 1, "yarn": 2}

    def __init__(self, base: float, style="halves", dims: int = 0, scaling: str = "none", factor: float = 1.0,
                 original: int = 0, beta_fast: float = 0.0, beta_slow: float = 0.0, attention: float = 0.0):
        if style not in self.STYLES or scaling not in self.SCALINGS:
            raise ValueError("style is one of halves, pairs; scaling one of none, linear, yarn")
        self._c = [cb_rope(base, self.STYLES[style], dims, self.SCALINGS[scaling], factor, original, beta_fast, beta_slow,
                           attention, inverse) for inverse in (0, 1)]

    def desc(self, inverse: bool = False) -> cb_rope:
        return self._c[1 if inverse else 0]


def _require(ok: bool, message: str):
    if not ok:
        raise ValueError(message)


_half = None


def _is_bf16(x) -> bool:
    """A tensor of 16-bit storage that does not say it holds fp16."""
    global _half
    if _half is None:
        import torch
        _half = torch.float16
    return x.element_size() == 2 and x.dtype is not _half


def _is_int32(x) -> bool:
    return x.element_size() == 4 and not x.dtype.is_floating_point


class CacheBack:
    """One cb_ctx.  Methods enqueue work on a CUDA stream (default: torch's current stream)."""

    _create = "cb_create"

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_query_tokens: int,
                 max_positions: int, max_senders: int = 1, p: float = 2.0, alpha: float = 2.0,
                 pool_width: int = 7, span_width: int = 16, n_sink: int = 1, n_latent: int = 40,
                 softmax_scale: float = 0.0, score_kernel: int = 0, lib_path: Optional[str] = None):
        self.lib = load_library(lib_path)
        cfg = cb_config()
        self.lib.cb_config_init(ctypes.byref(cfg))
        cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        cfg.max_query_tokens, cfg.max_positions, cfg.max_senders = max_query_tokens, max_positions, max_senders
        cfg.softmax_scale, cfg.p, cfg.alpha = softmax_scale, p, alpha
        cfg.pool_width, cfg.span_width, cfg.n_sink, cfg.n_latent = pool_width, span_width, n_sink, n_latent
        cfg.score_kernel = score_kernel
        self.cfg = cfg
        self._shape = (n_layers, n_kv_heads, head_dim)
        h = ctypes.c_void_p()
        st = getattr(self.lib, self._create)(ctypes.byref(cfg), ctypes.byref(h))
        if st != CB_OK:
            raise CBError(st, self.lib.cb_last_error(None).decode())
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.cb_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != CB_OK:
            raise CBError(st, self.lib.cb_last_error(self.h).decode())

    @property
    def scratch_bytes(self) -> int:
        return int(self.lib.cb_scratch_bytes(self.h))

    def score_path(self) -> int:
        """Logit-pass kernels of the last score call: 2 tcgen05, 1 mma.sync, 0 none yet."""
        return int(self.lib.cb_score_path(self.h))

    # -- the three steps ----------------------------------------------------
    def score(self, Ks: Sequence, Qs: Sequence, scores: Sequence, stream=None, Kselfs: Optional[Sequence] = None):
        """Kselfs (optional): per sender, the query tokens' own keys (or None) that join each
        query token's softmax causally."""
        n = len(Ks)
        kv = (cb_kv * n)(*[kv_desc(K) for K in Ks])
        Kselfs = Kselfs or [None] * n
        qq = (cb_query * n)(*[query_desc(Q, Kq) for Q, Kq in zip(Qs, Kselfs)])
        out = _ptr_array([s.data_ptr() for s in scores])
        self._check(self.lib.cb_score(self.h, n, kv, qq, out, _stream_handle(stream)))

    def select(self, scores: Sequence, Ts: Sequence[int], budgets: Sequence[int], idx: Sequence, stream=None):
        n = len(scores)
        sp = _ptr_array([s.data_ptr() for s in scores])
        Ta = _ptr_array(list(map(int, Ts)), ctypes.c_int64)
        Ba = _ptr_array(list(map(int, budgets)), ctypes.c_int64)
        ip = _ptr_array([x.data_ptr() for x in idx])
        self._check(self.lib.cb_select(self.h, n, sp, Ta, Ba, ip, _stream_handle(stream)))

    def compact(self, Ks: Sequence, Vs: Sequence, idx: Sequence, budgets: Sequence[int], k_out, v_out,
                offsets: Sequence[int], stream=None):
        """k_out, v_out: bf16 [nL][Hkv][capacity][d] (contiguous rows)."""
        n = len(Ks)
        kv = (cb_kv * n)(*[kv_desc(K, V) for K, V in zip(Ks, Vs)])
        ip = _ptr_array([x.data_ptr() for x in idx])
        Ba = _ptr_array(list(map(int, budgets)), ctypes.c_int64)
        Oa = _ptr_array(list(map(int, offsets)), ctypes.c_int64)
        ost = k_out.stride()
        assert ost[3] == 1 and ost[2] == k_out.size(3) and v_out.stride() == ost
        self._check(self.lib.cb_compact(self.h, n, kv, ip, Ba, k_out.data_ptr(), v_out.data_ptr(),
                                        k_out.size(2), Oa, ost[0], ost[1],
                                        _stream_handle(stream)))

    def compact_rope(self, Ks: Sequence, Vs: Sequence, idx: Sequence, budgets: Sequence[int], k_out, v_out,
                     offsets: Sequence[int], base: float, style: int = 0, pos0: int = 0, stream=None):
        """compact with K moved to receiver positions pos0 + offset + j by the rotary embedding
        (style 0: pairs (k, k + d/2); 1: pairs (2k, 2k + 1))."""
        n = len(Ks)
        kv = (cb_kv * n)(*[kv_desc(K, V) for K, V in zip(Ks, Vs)])
        ip = _ptr_array([x.data_ptr() for x in idx])
        Ba = _ptr_array(list(map(int, budgets)), ctypes.c_int64)
        Oa = _ptr_array(list(map(int, offsets)), ctypes.c_int64)
        ost = k_out.stride()
        assert ost[3] == 1 and ost[2] == k_out.size(3) and v_out.stride() == ost
        self._check(self.lib.cb_compact_rope(self.h, n, kv, ip, Ba, k_out.data_ptr(), v_out.data_ptr(),
                                             k_out.size(2), Oa, ost[0], ost[1], float(base),
                                             int(style), int(pos0), _stream_handle(stream)))

    def gather(self, tables: Sequence, idx: Sequence, counts: Sequence[int], out, offsets: Sequence[int],
               stream=None):
        """Message rows (App. C.3): out row offsets[i] + j = tables[i][idx[i][j]], j < counts[i].
        tables: per-sender [T_i][...] device tensors with one row per position (same row size and
        row stride); out: [capacity][...] with the same row size; idx: int32 device tensors."""
        n = len(tables)
        row_bytes = tables[0][0].numel() * tables[0].element_size()
        src_stride = tables[0].stride(0) * tables[0].element_size()
        for t in tables:
            assert t[0].is_contiguous() and t.stride(0) * t.element_size() == src_stride
            assert t[0].numel() * t.element_size() == row_bytes
        assert out[0].numel() * out.element_size() == row_bytes and out[0].is_contiguous()
        sp = _ptr_array([t.data_ptr() for t in tables])
        Ta = _ptr_array([int(t.shape[0]) for t in tables], ctypes.c_int64)
        ip = _ptr_array([x.data_ptr() for x in idx])
        Ca = _ptr_array([int(c) for c in counts], ctypes.c_int64)
        Oa = _ptr_array(list(map(int, offsets)), ctypes.c_int64)
        self._check(self.lib.cb_gather(self.h, n, sp, Ta, src_stride, row_bytes, ip, Ca, out.data_ptr(),
                                       out.shape[0], Oa, out.stride(0) * out.element_size(),
                                       _stream_handle(stream)))

    # -- the receiver's side: rotary positions, rows in 4 bits, attention over them -----------------
    def rotary(self, xs: Sequence, rope: Rotary, ys: Optional[Sequence] = None, pos=None, pos0: int = 0,
               inverse: bool = False, stream=None):
        """Turn bf16 vectors [nL][tokens][heads][d] (or [tokens][heads][d]) to their positions: ys[i] from
        xs[i], in place where ys or ys[i] is None.  pos: int32 device tensor of every token's position,
        or a list of one (or None) per set; else token r is at pos0 + r.  inverse: the transposed turn
        (the gradient of the forward one).  Returns ys."""
        n = len(xs)
        _require(ys is None or len(ys) == n, "one y (or None) per x")
        ys = [x if y is None else y for x, y in zip(xs, ys or [None] * n)]
        pos = list(pos) if isinstance(pos, (list, tuple)) else [pos] * n
        _require(len(pos) == n, "one pos (or None) per x")
        fields = array("q")                   # of the header's cb_vectors, eight bytes each (the counts of layers and heads share them)
        for x, y, p in zip(xs, ys, pos):
            shape, xt = x.shape, x.stride()
            yt = xt if y is x else y.stride()
            if not (shape == y.shape and len(shape) in (3, 4) and shape[-1] == self.cfg.head_dim):
                raise ValueError("vectors are [nL][tokens][heads][d]")
            if not (_is_bf16(x) and (y is x or _is_bf16(y)) and xt[-1] == yt[-1] == 1):
                raise ValueError("vectors are bf16 and contiguous")
            if p is not None and not (_is_int32(p) and p.is_contiguous() and p.numel() == shape[-3]):
                raise ValueError("pos holds one int32 a token")
            nl, xl, yl = (shape[0], xt[0], yt[0]) if len(shape) == 4 else (1, 0, 0)
            fields.extend((x.data_ptr(), y.data_ptr(), nl | shape[-2] << 32, shape[-3], xl, xt[-3], xt[-2], yl, yt[-3], yt[-2],
                           0 if p is None else p.data_ptr(), pos0))
        self._check(self.lib.cb_rotary(self.h, n, fields.buffer_info()[0], ctypes.byref(rope.desc(inverse)),
                                      _stream_on(stream, xs[0]) if n else 0))
        return ys

    def pack(self, Ks: Sequence, Vs: Sequence, caches: Sequence, offsets: Optional[Sequence[int]] = None,
             idx: Optional[Sequence] = None, counts: Optional[Sequence[int]] = None, rows: Optional[Sequence] = None,
             layer: int = 0, stream=None):
        """Rows of bf16 K and V [layers][Hkv][T][d] (or PagedKV) into 4-bit caches: row idx[i][j] (row j
        without idx) of sender i becomes row rows[i][j] (offsets[i] + j without rows) of caches[i], in the
        layers from `layer` on.  counts: rows of each sender (default: all of idx, or of K)."""
        n = len(Ks)
        idx, rows = idx or [None] * n, rows or [None] * n
        counts = counts or [int(K.shape[2]) if x is None else int(x.numel()) for K, x in zip(Ks, idx)]
        if not (0 < n == len(Vs) == len(caches) == len(idx) == len(rows) == len(counts) and (offsets is None or len(offsets) == n)):
            raise ValueError("one entry per sender in every list")
        layers = Ks[0].shape[0]
        for K, V, x, r, c, p in zip(Ks, Vs, idx, rows, counts, caches):
            for t in (x, r):
                if t is not None and not (_is_int32(t) and t.is_contiguous() and t.numel() >= c):
                    raise ValueError("idx and rows hold an int32 a row")
            shape = K.shape
            if not (_is_bf16(K.k_pool) and _is_bf16(K.v_pool) if isinstance(K, PagedKV) else
                    _is_bf16(K) and K.dtype == V.dtype and shape == V.shape):
                raise ValueError("K and V are bf16 of one shape")
            self._fits(p)
            if not (shape[1] == p.n_kv_heads and shape[3] == p.head_dim and shape[0] == layers):
                raise ValueError("K and V do not match the cache")
        kv = b"".join([bytes(kv_desc(K, V)) for K, V in zip(Ks, Vs)])
        held = b"".join([bytes(p.desc(p.capacity)) for p in caches])
        # idx, counts, offsets and rows of the call, one array of eight-byte numbers
        parts = array("q", [0 if x is None else x.data_ptr() for x in idx])
        parts.extend(map(int, counts))
        parts.extend(map(int, offsets or ()))
        parts.extend([0] * (3 * n - len(parts)))
        parts.extend([0 if x is None else x.data_ptr() for x in rows])
        at = parts.buffer_info()[0]
        self._check(self.lib.cb_pack(self.h, n, kv, at, at + 8 * n, held, None if offsets is None else at + 16 * n, at + 24 * n,
                                     int(layer), int(layers), _stream_on(stream, caches[0].k)))

    def unpack(self, caches: Sequence, k_out, v_out, offsets: Optional[Sequence[int]] = None, idx: Optional[Sequence] = None,
               counts: Optional[Sequence[int]] = None, stream=None):
        """Rows of 4-bit caches as bf16, all layers: row idx[i][j] (row j without idx) of caches[i] becomes row
        offsets[i] + j of k_out, v_out [nL][Hkv][capacity][d]; by default every cached row, caches back to
        back."""
        n = len(caches)
        idx = idx or [None] * n
        counts = counts or [p.T if x is None else int(x.numel()) for p, x in zip(caches, idx)]
        offsets = offsets or [sum(counts[:i]) for i in range(n)]
        _require(len(idx) == len(counts) == len(offsets) == n, "one entry per cache in every list")
        for p, x, c in zip(caches, idx, counts):
            self._fits(p)
            _require(x is None or (_is_int32(x) and x.is_contiguous() and x.numel() >= c), "idx holds an int32 a row")
        shape, ost = k_out.shape, k_out.stride()
        if not (len(shape) == 4 and ost[3] == 1 and ost[2] == shape[3] == self.cfg.head_dim and v_out.stride() == ost and
                v_out.shape == shape and _is_bf16(k_out) and _is_bf16(v_out) and
                shape[0] == self.cfg.n_layers and shape[1] == self.cfg.n_kv_heads):
            raise ValueError("k_out, v_out are bf16 [nL][Hkv][capacity][d]")
        held = b"".join([p._state[1] or p._described() for p in caches])
        parts = array("q", [0 if x is None else x.data_ptr() for x in idx])
        parts.extend(map(int, counts))
        parts.extend(map(int, offsets))
        at = parts.buffer_info()[0]
        self._check(self.lib.cb_unpack(self.h, n, held, at, at + 8 * n, k_out.data_ptr(), v_out.data_ptr(), shape[2], at + 16 * n,
                                       ost[0], ost[1], _stream_on(stream, k_out)))

    def attend(self, caches: Sequence, Qs: Sequence, outs: Sequence, layer: int = 0, causal: bool = True, window: int = 0,
               lses: Optional[Sequence] = None, stream=None):
        """One layer's attention over 4-bit caches: outs[i] (bf16 [m][Hq][d]) of query tokens Qs[i] (bf16
        [m][Hq][d]), the last m positions of caches[i] (causal: each sees the rows up to its own, the last
        `window` of them where window > 0; otherwise all); lses[i] (fp32 [m][Hq], contiguous) receives the
        log-sum-exp.  Qs, outs and lses may be tensors with the sequences in their first dimension."""
        n = len(caches)
        cfg, like = self.cfg, self._shape
        for p in caches:
            if p._shape != like:
                self._fits(p)
        held = b"".join([p._state[1] or p._described() for p in caches])
        if n and hasattr(Qs, "data_ptr") and hasattr(outs, "data_ptr") and (lses is None or hasattr(lses, "data_ptr")):
            # one tensor each: the sequences' addresses by arithmetic
            shape, qt, ot = Qs.shape, Qs.stride(), outs.stride()
            if not (len(shape) == 4 and shape == outs.shape and shape[0] == n and shape[2] == cfg.n_q_heads and
                    shape[3] == cfg.head_dim and qt[3] == ot[3] == 1 and _is_bf16(Qs) and _is_bf16(outs)):
                raise ValueError("queries and outputs are bf16 [sequences][m][Hq][d]")
            m, a, o, e = shape[1], Qs.data_ptr(), outs.data_ptr(), 0
            steps = [(0, a, 2 * qt[0]), (1, o, 2 * ot[0])]
            if lses is not None:
                lt = lses.stride()
                if not (lses.shape == shape[:3] and lses.element_size() == 4 and lses.dtype.is_floating_point and
                        (m == 0 or (lt[2] == 1 and (m == 1 or lt[1] == shape[2])))):
                    raise ValueError("lse is fp32 [sequences][m][Hq]")
                e = lses.data_ptr()
                steps.append((2, e, 4 * lt[0]))
            fields = array("q", (a, o, e, m, qt[1], qt[2], ot[1], ot[2])) * n      # of the header's cb_attend_query, eight bytes each
            for at, first, step in steps:
                if n > 1 and step:
                    fields[at::8] = array("q", range(first, first + n * step, step))
        else:
            _require(len(Qs) == len(outs) == n and (lses is None or len(lses) == n), "one query and output per cache")
            fields = array("q")
            for i in range(n):
                fields.extend(self._queries(Qs[i], outs[i], None if lses is None else lses[i]))
        self._check(self.lib.cb_attend(self.h, int(layer), n, held, fields.buffer_info()[0], 1 if causal else 0, int(window),
                                       _stream_on(stream, caches[0].k) if n else 0))

    def _queries(self, Q, out, lse):
        """One sequence's fields of a cb_attend_query, looked over."""
        qt, ot = Q.stride(), out.stride()
        m, heads, d = shape = Q.shape
        if not (out.shape == shape and heads == self.cfg.n_q_heads and d == self.cfg.head_dim and qt[2] == ot[2] == 1 and
                _is_bf16(Q) and _is_bf16(out)):
            raise ValueError("queries and outputs are bf16 [m][Hq][d]")
        if lse is None:
            e = 0
        else:
            _require(lse.shape == (m, heads) and lse.is_contiguous() and lse.element_size() == 4 and lse.dtype.is_floating_point,
                     "lse is fp32 [m][Hq]")
            e = lse.data_ptr()
        return Q.data_ptr(), out.data_ptr(), e, m, qt[0], qt[1], ot[0], ot[1]

    def _fits(self, p: PackedKV):
        _require(p._shape == self._shape, "the cache's layers, heads or head dimension are not the context's")

    def set_wait_limit(self, limit_ns: int = 0, stall_next_score: bool = False, stall_next_attend: bool = False):
        """cb_set_wait_limit: limit of one bounded device wait (0: the 1 s default); with
        stall_next_score (stall_next_attend) the next tcgen05 cb_score (cb_attend) makes one wait run out
        (failure-detection test)."""
        _require(not (stall_next_score and stall_next_attend), "one stall at a time")
        self._check(self.lib.cb_set_wait_limit(self.h, int(limit_ns), 1 if stall_next_score else 2 if stall_next_attend else 0))

    def set_score_sms(self, n_sms: int = 0):
        """cb_set_score_sms: SMs the persistent score kernels occupy (0: all)."""
        self._check(self.lib.cb_set_score_sms(self.h, int(n_sms)))

    STAGES = ("row_statistics", "statistics_combine", "normalised_accumulation", "finalize")

    def enable_stage_timing(self, enable=True):
        """True / 1: time every score kernel; 2: only the second logit pass; False / 0: off."""
        mode = int(enable) if not isinstance(enable, bool) else (1 if enable else 0)
        self._check(self.lib.cb_enable_stage_timing(self.h, mode))

    def stage_times(self):
        """(dict stage -> summed ms, number of cb_score calls) since the previous read."""
        ms = (ctypes.c_float * 4)()
        calls = ctypes.c_int32()
        self._check(self.lib.cb_stage_times(self.h, ms, ctypes.byref(calls)))
        return dict(zip(self.STAGES, list(ms))), int(calls.value)

    def sync_status(self, stream=None):
        self._check(self.lib.cb_sync_status(self.h, _stream_handle(stream)))


class Receiver(CacheBack):
    """A context without the scratch of score and select (cb_create_receiver): rotary, pack, unpack,
    attend, compact and gather, with max_positions and n_layers free."""

    _create = "cb_create_receiver"

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_query_tokens: int,
                 max_positions: int, max_senders: int = 1, softmax_scale: float = 0.0, lib_path: Optional[str] = None):
        super().__init__(n_layers, n_q_heads, n_kv_heads, head_dim, max_query_tokens, max_positions, max_senders,
                         softmax_scale=softmax_scale, lib_path=lib_path)
