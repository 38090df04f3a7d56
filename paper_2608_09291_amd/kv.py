"""Python binding of the 8-bit key/value cache (include/us_kv.h).

Argument marshalling and the checks that only the tensors can answer (types,
shapes, strides); every computation happens in the native library.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

from . import binding
from .binding import _check, _stream_handle

BLOCK = 64           # US_KV_BLOCK: tokens of a block
HEAD_DIM_MAX = 256   # US_KV_HEAD_DIM_MAX

#: Every symbol us_kv.h declares.
EXPORTS = ("us_kv_row", "us_kv_append", "us_kv_read", "us_kv_attend_workspace_size", "us_kv_attend", "us_kv_evict")


class CacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n_blocks", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class SeqsStruct(ctypes.Structure):
    _fields_ = [("blocks", ctypes.c_void_p), ("stride", ctypes.c_int64), ("width", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("lens", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("max_new", ctypes.c_int32)]


class RowsStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("tokens", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class AttendOpts(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("weights", ctypes.c_void_p), ("weights_stride", ctypes.c_int64)]


class KeptStruct(ctypes.Structure):
    _fields_ = [("blocks", ctypes.c_void_p), ("stride", ctypes.c_int64), ("width", ctypes.c_int32),
                ("lens", ctypes.c_void_p), ("weights", ctypes.c_void_p), ("weights_stride", ctypes.c_int64),
                ("index", ctypes.c_void_p)]


_ready = None


def lib():
    """The native library with the signatures of us_kv.h; raises if it was not built."""
    global _ready
    if _ready is None:
        L = binding.lib()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        pc, ps, pr, po = (ctypes.POINTER(t) for t in (CacheStruct, SeqsStruct, RowsStruct, AttendOpts))
        L.us_kv_row.argtypes = [i32]
        L.us_kv_append.argtypes = [pc, ps, pr, pr, vp]
        L.us_kv_read.argtypes = [pc, ps, pr, pr, vp]
        L.us_kv_attend_workspace_size.argtypes = [pc, ps, i32, i32, po, ctypes.POINTER(sz)]
        L.us_kv_attend.argtypes = [pc, ps, i32, pr, pr, po, vp, sz, vp]
        L.us_kv_evict.argtypes = [pc, ps, vp, i64, i32, i32, i32, ctypes.POINTER(KeptStruct), vp]
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        _ready = L
    return _ready


def row(head_dim: int) -> int:
    """us_kv_row: bytes of a head's key (or value) per token."""
    r = lib().us_kv_row(head_dim)
    if r == 0:
        raise ValueError(f"head_dim {head_dim} is outside [1, {HEAD_DIM_MAX}]")
    return r


def _dtype(t):
    import torch
    codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    if t.dtype not in codes:
        raise TypeError(f"{t.dtype} rows: float32, bfloat16 or float16 are wanted")
    return codes[t.dtype]


def _want(t, name, dtype, ndim):
    if t.dtype != dtype or t.dim() != ndim or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise TypeError(f"{name}: a {dtype} tensor of {ndim} dimensions, the last one contiguous, is wanted")
    return t


@dataclass
class Cache:
    """A pool of blocks: uint8 codes (n_blocks, heads, BLOCK * row(head_dim)) and float32 scales (n_blocks, heads)."""

    k: "object"
    v: "object"
    k_scale: "object"
    v_scale: "object"
    head_dim: int

    @property
    def n_blocks(self): return self.k.shape[0]

    @property
    def heads(self): return self.k.shape[1]

    def struct(self) -> CacheStruct:
        import torch
        shape = (self.n_blocks, self.heads, BLOCK * row(self.head_dim))
        for t in (self.k, self.v):
            if t.dtype != torch.uint8 or tuple(t.shape) != shape or not t.is_contiguous():
                raise TypeError(f"codes: contiguous uint8 tensors of shape {shape} are wanted")
        for t in (self.k_scale, self.v_scale):
            if t.dtype != torch.float32 or tuple(t.shape) != shape[:2] or not t.is_contiguous():
                raise TypeError(f"scales: contiguous float32 tensors of shape {shape[:2]} are wanted")
        return CacheStruct(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                           shape[0], shape[1], self.head_dim)


def new_cache(n_blocks: int, heads: int, head_dim: int, device="cuda") -> Cache:
    """An empty pool of n_blocks blocks per head."""
    import torch
    shape = (n_blocks, heads, BLOCK * row(head_dim))
    codes = [torch.full(shape, 128, dtype=torch.uint8, device=device) for _ in range(2)]
    scales = [torch.zeros(shape[:2], dtype=torch.float32, device=device) for _ in range(2)]
    return Cache(*codes, *scales, head_dim)


def _seqs(blocks, lens, starts, max_new) -> SeqsStruct:
    import torch
    _want(blocks, "blocks", torch.int32, 2)
    _want(lens, "lens", torch.int32, 1)
    batch = blocks.shape[0]
    if lens.shape[0] != batch:
        raise ValueError("lens: one length per row of blocks is wanted")
    if starts is not None:
        _want(starts, "starts", torch.int32, 1)
        if starts.shape[0] != batch + 1:
            raise ValueError("starts: one entry more than sequences is wanted")
    return SeqsStruct(blocks.data_ptr(), blocks.stride(0) if batch > 1 else blocks.shape[1], blocks.shape[1], batch,
                      lens.data_ptr(), None if starts is None else starts.data_ptr(), max_new)


def _rows(t, heads, head_dim, name) -> RowsStruct:
    if t.dim() != 3 or tuple(t.shape[1:]) != (heads, head_dim) or (head_dim > 1 and t.stride(2) != 1):
        raise TypeError(f"{name}: (tokens, {heads}, {head_dim}) with contiguous values is wanted")
    return RowsStruct(t.data_ptr(), t.stride(0), t.stride(1), t.shape[0], _dtype(t))


def append(cache: Cache, blocks, lens, k, v, starts=None, max_new: int = 1, stream=None) -> None:
    """us_kv_append: quantise the sequences' last tokens (rows of k and v) into their blocks."""
    c, s = cache.struct(), _seqs(blocks, lens, starts, max_new)
    kr, vr = (_rows(t, cache.heads, cache.head_dim, n) for t, n in ((k, "k"), (v, "v")))
    _check("us_kv_append", lib().us_kv_append(ctypes.byref(c), ctypes.byref(s), ctypes.byref(kr), ctypes.byref(vr),
                                              _stream_handle(stream)))


def read(cache: Cache, blocks, lens, k_out, v_out, starts=None, max_new: int = 1, stream=None) -> None:
    """us_kv_read: the sequences' last tokens as dense rows."""
    c, s = cache.struct(), _seqs(blocks, lens, starts, max_new)
    kr, vr = (_rows(t, cache.heads, cache.head_dim, n) for t, n in ((k_out, "k_out"), (v_out, "v_out")))
    _check("us_kv_read", lib().us_kv_read(ctypes.byref(c), ctypes.byref(s), ctypes.byref(kr), ctypes.byref(vr),
                                          _stream_handle(stream)))


def _opts(scale, causal, window, max_len, weights, batch, heads) -> AttendOpts:
    import torch
    if weights is not None:
        _want(weights, "weights", torch.float32, 3)
        if tuple(weights.shape[:2]) != (batch, heads) or not weights.is_contiguous():
            raise ValueError("weights: a contiguous (sequences, cache heads, tokens) tensor is wanted")
    return AttendOpts(0.0 if scale is None else scale, int(bool(causal)), window, max_len or 0,
                      None if weights is None else weights.data_ptr(), 0 if weights is None else weights.shape[2])


def attend_workspace_size(cache: Cache, q_heads: int, tokens: int, blocks, lens=None, starts=None, max_q: int = 1,
                          max_len=None, causal: bool = True, window: int = 0, weights=None) -> int:
    """us_kv_attend_workspace_size: device bytes us_kv_attend needs for these sizes."""
    c = cache.struct()
    # (the lengths themselves are not looked at)
    s = SeqsStruct(blocks.data_ptr(), blocks.stride(0) if blocks.shape[0] > 1 else blocks.shape[1], blocks.shape[1],
                   blocks.shape[0], blocks.data_ptr(), None if starts is None else starts.data_ptr(), max_q)
    o = _opts(None, causal, window, max_len, weights, blocks.shape[0], cache.heads)
    n = ctypes.c_size_t(0)
    _check("us_kv_attend_workspace_size", lib().us_kv_attend_workspace_size(
        ctypes.byref(c), ctypes.byref(s), q_heads, tokens, ctypes.byref(o), ctypes.byref(n)))
    return n.value


def attend_workspace(cache: Cache, q, blocks, starts=None, max_q: int = 1, max_len=None, causal: bool = True,
                     window: int = 0, weights=None):
    """A zero-filled workspace for attend calls of these sizes (lengths up to max_len, or the table's)."""
    import torch
    n = attend_workspace_size(cache, q.shape[1], q.shape[0], blocks, None, starts, max_q, max_len, causal, window,
                              weights)
    return torch.zeros((n + 3) // 4, dtype=torch.int32, device=q.device)


def attend(cache: Cache, blocks, lens, q, out, starts=None, max_q: int = 1, max_len=None, scale=None,
           causal: bool = True, window: int = 0, weights=None, ws=None, stream=None) -> None:
    """us_kv_attend: out = softmax(scale q k) v over the cache; weights (if given) gain each token's probabilities."""
    c, s = cache.struct(), _seqs(blocks, lens, starts, max_q)
    heads = q.shape[1] if q.dim() == 3 else 0
    qr, outr = (_rows(t, heads, cache.head_dim, n) for t, n in ((q, "q"), (out, "out")))
    o = _opts(scale, causal, window, max_len, weights, s.batch, cache.heads)
    _check("us_kv_attend", lib().us_kv_attend(
        ctypes.byref(c), ctypes.byref(s), heads, ctypes.byref(qr), ctypes.byref(outr), ctypes.byref(o),
        None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel() * ws.element_size(),
        _stream_handle(stream)))


def evict(cache: Cache, blocks, lens, weights, keep: int, recent: int, to_blocks, to_lens, to_weights, index,
          max_len=None, stream=None) -> None:
    """us_kv_evict: the recent and the most attended tokens of every sequence, moved to to_blocks."""
    import torch
    c, s = cache.struct(), _seqs(blocks, lens, None, 1)
    for t, name in ((weights, "weights"), (to_weights, "to_weights")):
        if t is not None:
            _want(t, name, torch.float32, 3)
            if tuple(t.shape[:2]) != (s.batch, cache.heads) or not t.is_contiguous():
                raise ValueError(f"{name}: a contiguous (sequences, cache heads, tokens) tensor is wanted")
    _want(to_blocks, "to_blocks", torch.int32, 2)
    _want(to_lens, "to_lens", torch.int32, 1)
    _want(index, "index", torch.int32, 3)
    if to_blocks.shape[0] != s.batch or to_lens.shape[0] != s.batch:
        raise ValueError("to_blocks, to_lens: one row per sequence is wanted")
    if tuple(index.shape) != (s.batch, cache.heads, keep) or not index.is_contiguous():
        raise ValueError("index: a contiguous (sequences, cache heads, keep) tensor is wanted")
    to = KeptStruct(to_blocks.data_ptr(), to_blocks.stride(0) if s.batch > 1 else to_blocks.shape[1],
                    to_blocks.shape[1], to_lens.data_ptr(), None if to_weights is None else to_weights.data_ptr(),
                    0 if to_weights is None else to_weights.shape[2], index.data_ptr())
    _check("us_kv_evict", lib().us_kv_evict(ctypes.byref(c), ctypes.byref(s), weights.data_ptr(), weights.shape[2],
                                            max_len or 0, keep, recent, ctypes.byref(to), _stream_handle(stream)))
