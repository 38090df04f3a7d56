"""Python binding of the 8-bit key/value cache (include/us_kv.h).

Argument marshalling and the checks that only the tensors can answer (types,
shapes, strides); every computation happens in the native library. A decode
step's calls take the GPU a few microseconds, so tensors are looked at in
compiled code (csrc/python), one call for each argument, and the structs are
packed without ctypes objects.
"""
from __future__ import annotations

import ctypes
import importlib
import struct

import torch

from . import binding
from .binding import _check

BLOCK = 64           # US_KV_BLOCK: tokens of a block
HEAD_DIM_MAX = 256   # US_KV_HEAD_DIM_MAX
AXES_MAX = 4         # US_KV_AXES_MAX
CHOSEN_MAX = 1 << 16  # US_KV_CHOSEN_MAX

#: Every symbol us_kv.h declares.
EXPORTS = ("us_kv_row", "us_kv_append", "us_kv_read", "us_kv_attend_workspace_size", "us_kv_attend_route",
           "us_kv_attend", "us_kv_evict", "us_kv_rotate", "us_kv_fork_workspace_size", "us_kv_fork",
           "us_kv_attend_shared_workspace_size", "us_kv_attend_shared", "us_kv_summarise", "us_kv_choose_workspace_size",
           "us_kv_choose", "us_kv_attend_chosen_workspace_size", "us_kv_attend_chosen")


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


class AttendRouteInfo(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("prompt", "tile_rows", "split_keys", "part_blocks")]


class KeptStruct(ctypes.Structure):
    _fields_ = [("blocks", ctypes.c_void_p), ("stride", ctypes.c_int64), ("width", ctypes.c_int32),
                ("lens", ctypes.c_void_p), ("weights", ctypes.c_void_p), ("weights_stride", ctypes.c_int64),
                ("index", ctypes.c_void_p)]


class RotationStruct(ctypes.Structure):
    _fields_ = [("freq", ctypes.c_void_p), ("pairs", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("positions", ctypes.c_void_p), ("positions_stride", ctypes.c_int64), ("offset", ctypes.c_int32),
                ("adjacent", ctypes.c_int32), ("norm", ctypes.c_int32), ("eps", ctypes.c_float),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p)]


class ForkedStruct(ctypes.Structure):
    _fields_ = [("blocks", ctypes.c_void_p), ("stride", ctypes.c_int64), ("width", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("lens", ctypes.c_void_p)]


class GroupsStruct(ctypes.Structure):
    _fields_ = [("starts", ctypes.c_void_p), ("shared", ctypes.c_void_p), ("groups", ctypes.c_int32),
                ("max_group", ctypes.c_int32), ("max_shared", ctypes.c_int32)]


class ChoiceStruct(ctypes.Structure):
    _fields_ = [("scores", ctypes.c_void_p), ("scores_stride", ctypes.c_int64), ("chosen", ctypes.c_void_p),
                ("top", ctypes.c_int32), ("sinks", ctypes.c_int32), ("recent", ctypes.c_int32), ("max_len", ctypes.c_int32)]


_ready = _args = None


def lib():
    """The native library with the signatures of us_kv.h; raises if it (or the tensors' checks) was not built."""
    global _ready, _args
    if _ready is None:
        L = binding.lib()
        try:
            _args = importlib.import_module("._kv_args", __package__)
        except ModuleNotFoundError as e:
            raise RuntimeError("_kv_args.so is missing: run `python -m paper_2608_09291_amd.build_args`") from e
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        # (structs go as void pointers: byref() of the classes above, or their packed bytes)
        L.us_kv_row.argtypes = [i32]
        L.us_kv_append.argtypes = [vp, vp, vp, vp, vp]
        L.us_kv_read.argtypes = [vp, vp, vp, vp, vp]
        L.us_kv_attend_workspace_size.argtypes = [vp, vp, i32, i32, vp, ctypes.POINTER(sz)]
        L.us_kv_attend_route.argtypes = [vp, vp, i32, i32, i32, vp, ctypes.POINTER(AttendRouteInfo)]
        L.us_kv_attend.argtypes = [vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.us_kv_evict.argtypes = [vp, vp, vp, i64, i32, i32, i32, vp, vp]
        L.us_kv_rotate.argtypes = [i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.us_kv_fork_workspace_size.argtypes = [vp, i32, i32, ctypes.POINTER(sz)]
        L.us_kv_fork.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.us_kv_attend_shared_workspace_size.argtypes = [vp, vp, i32, i32, vp, vp, ctypes.POINTER(sz)]
        L.us_kv_attend_shared.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.us_kv_summarise.argtypes = [vp, vp, vp, vp]
        L.us_kv_choose_workspace_size.argtypes = [vp, vp, i32, i32, ctypes.POINTER(sz)]
        L.us_kv_choose.argtypes = [vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.us_kv_attend_chosen_workspace_size.argtypes = [vp, vp, i32, i32, i32, ctypes.POINTER(sz)]
        L.us_kv_attend_chosen.argtypes = [vp, vp, i32, vp, vp, vp, i32, vp, vp, sz, vp]
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        _ready = L
    return _ready


# The structs' layouts, padded to their size in C.
_pack_cache = struct.Struct("@PPPPiii4x").pack
_pack_seqs = struct.Struct("@PqiiPPi4x").pack
_pack_rows = struct.Struct("@Pqqii").pack
_pack_opts = struct.Struct("@fiii Pq").pack
_pack_kept = struct.Struct("@Pqi4xPPqP").pack
_pack_rotation = struct.Struct("@PiiPqiiifPP").pack
_pack_forked = struct.Struct("@PqiiP").pack
_pack_groups = struct.Struct("@PPiii4x").pack
_pack_choice = struct.Struct("@PqPiiii").pack

_I32, _F32 = torch.int32, torch.float32
_ROWS = {}      # us_kv_row by head_dim


def row(head_dim: int) -> int:
    """us_kv_row: bytes of a head's key (or value) per token."""
    r = _ROWS.get(head_dim)
    if r is None:
        r = lib().us_kv_row(head_dim)
        if r == 0:
            raise ValueError(f"head_dim {head_dim} is outside [1, {HEAD_DIM_MAX}]")
        _ROWS[head_dim] = r
    return r


def _stream(stream, cache) -> int:
    """A call's stream. The library launches on the current device, which has to be the cache's and the stream's."""
    return _stream_on(stream, cache.device, "the cache")


def _stream_on(stream, device: int, what: str) -> int:
    now = torch.cuda.current_device()
    if device >= 0 and now != device:
        raise ValueError(f"{what} is on cuda:{device}, the current device is cuda:{now}")
    if stream is None:
        # (the handle alone: building torch's stream object takes as long as a launch)
        return torch._C._cuda_getCurrentRawStream(now)
    if stream.device.index != now:
        raise ValueError(f"a stream of cuda:{now}, the current device, is wanted")
    return stream.cuda_stream


class Cache:
    """A pool of blocks: uint8 codes (n_blocks, heads, BLOCK * row(head_dim)) and float32 scales (n_blocks, heads)."""

    def __init__(self, k, v, k_scale, v_scale, head_dim: int):
        size = BLOCK * row(head_dim)
        ak, av, aks, avs, n, heads, bytes_, self.device = _args.cache(k, v, k_scale, v_scale)
        if bytes_ != size:
            raise TypeError(f"codes: contiguous uint8 tensors (blocks, heads, {size}) are wanted")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_blocks, self.heads, self.head_dim = n, heads, head_dim
        self._packed = _pack_cache(ak, av, aks, avs, n, heads, head_dim)
        # what calls are given: they refuse None, a cache that is not on one GPU
        self._there = self._packed if self.device >= 0 else None

    def struct(self) -> CacheStruct:
        return CacheStruct.from_buffer_copy(self._packed)


def new_cache(n_blocks: int, heads: int, head_dim: int, device="cuda") -> Cache:
    """An empty pool of n_blocks blocks per head."""
    shape = (n_blocks, heads, BLOCK * row(head_dim))
    codes = [torch.full(shape, 128, dtype=torch.uint8, device=device) for _ in range(2)]
    scales = [torch.zeros(shape[:2], dtype=_F32, device=device) for _ in range(2)]
    return Cache(*codes, *scales, head_dim)


def _table(t, name):
    """(rows, columns, row stride) of an int32 table with contiguous rows."""
    rows, width = t.shape
    stride, one = t.stride()
    if t.dtype is not _I32 or (one != 1 and width > 1):
        raise TypeError(f"{name}: an int32 table with contiguous rows is wanted")
    return rows, width, stride if rows > 1 else width


def _numbers(t, n, name):
    if t.dtype is not _I32 or t.shape != (n,) or not t.is_contiguous():
        raise TypeError(f"{name}: {n} contiguous int32 numbers are wanted")
    return t.data_ptr()


def _on(t, device) -> bool:
    """Whether t is on GPU `device`, or on any where that is negative."""
    return t.is_cuda and (device < 0 or t.get_device() == device)


def _seqs(blocks, lens, starts, max_new, device) -> bytes:
    at, stride, width, batch, at_lens, at_starts = _args.seqs(blocks, lens, starts, device)
    return _pack_seqs(at, stride, width, batch, at_lens, at_starts, max_new)


def _rows(t, heads, head_dim, name, device) -> bytes:
    return _pack_rows(*_args.rows(t, heads, head_dim, name, device))


def _weights(t, batch, heads, name, device):
    """Address and row length of a float32 (sequences, heads, tokens) tensor."""
    b, h, n = t.shape
    if b != batch or h != heads or t.dtype is not _F32 or not t.is_contiguous():
        raise TypeError(f"{name}: a contiguous float32 tensor ({batch}, {heads}, tokens) is wanted")
    if not _on(t, device):
        raise TypeError(f"{name}: a tensor on the cache's GPU is wanted")
    return t.data_ptr(), n


def append(cache: Cache, blocks, lens, k, v, starts=None, max_new: int = 1, stream=None) -> None:
    """us_kv_append: quantise the sequences' last tokens (rows of k and v) into their blocks."""
    h, d, on = cache.heads, cache.head_dim, cache.device
    _check("us_kv_append", lib().us_kv_append(cache._there, _seqs(blocks, lens, starts, max_new, on), _rows(k, h, d, "k", on),
                                              _rows(v, h, d, "v", on), _stream(stream, cache)))


def read(cache: Cache, blocks, lens, k_out, v_out, starts=None, max_new: int = 1, stream=None) -> None:
    """us_kv_read: the sequences' last tokens as dense rows."""
    h, d, on = cache.heads, cache.head_dim, cache.device
    _check("us_kv_read", lib().us_kv_read(cache._there, _seqs(blocks, lens, starts, max_new, on), _rows(k_out, h, d, "k_out", on),
                                          _rows(v_out, h, d, "v_out", on), _stream(stream, cache)))


def _opts(scale, causal, window, max_len, weights, batch, heads, device):
    if weights is None:
        if scale is None and causal and not window and not max_len:
            return None
        at, n = 0, 0
    else:
        at, n = _weights(weights, batch, heads, "weights", device)
    return _pack_opts(0.0 if scale is None else scale, 1 if causal else 0, window, max_len or 0, at, n)


def _sizes(blocks, starts, max_q) -> bytes:
    """The sequences of a call whose sizes alone matter: what the lengths and starts are is not looked at."""
    batch, width, stride = _table(blocks, "blocks")
    return _pack_seqs(blocks.data_ptr(), stride, width, batch, blocks.data_ptr(),
                      0 if starts is None else starts.data_ptr(), max_q)


def attend_workspace_size(cache: Cache, q_heads: int, tokens: int, blocks, starts=None, max_q: int = 1, max_len=None,
                          causal: bool = True, window: int = 0, weights=None) -> int:
    """us_kv_attend_workspace_size: device bytes us_kv_attend needs for these sizes."""
    s, batch, n = _sizes(blocks, starts, max_q), blocks.shape[0], ctypes.c_size_t(0)
    _check("us_kv_attend_workspace_size", lib().us_kv_attend_workspace_size(
        cache._packed, s, q_heads, tokens, _opts(None, causal, window, max_len, weights, batch, cache.heads, cache.device),
        ctypes.byref(n)))
    return n.value


_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # us_dtype


def attend_route(cache: Cache, q, blocks, starts=None, max_q: int = 1, max_len=None, causal: bool = True, window: int = 0,
                 weights=None) -> dict:
    """us_kv_attend_route: what attend launches for these sizes."""
    r, s, batch = AttendRouteInfo(), _sizes(blocks, starts, max_q), blocks.shape[0]
    _check("us_kv_attend_route", lib().us_kv_attend_route(
        cache._packed, s, q.shape[1], q.shape[0], _TYPES[q.dtype],
        _opts(None, causal, window, max_len, weights, batch, cache.heads, cache.device), ctypes.byref(r)))
    return {name: getattr(r, name) for name, _ in AttendRouteInfo._fields_}


def attend_workspace(cache: Cache, q, blocks, starts=None, max_q: int = 1, max_len=None, causal: bool = True,
                     window: int = 0, weights=None):
    """A zero-filled workspace for attend calls of these sizes (lengths up to max_len, or the table's)."""
    n = attend_workspace_size(cache, q.shape[1], q.shape[0], blocks, starts, max_q, max_len, causal, window, weights)
    return torch.zeros((n + 3) // 4, dtype=_I32, device=q.device)


def attend(cache: Cache, blocks, lens, q, out, starts=None, max_q: int = 1, max_len=None, scale=None,
           causal: bool = True, window: int = 0, weights=None, ws=None, stream=None) -> None:
    """us_kv_attend: out = softmax(scale q k) v over the cache; weights (if given) gain each token's probabilities."""
    heads, d, on = q.shape[1], cache.head_dim, cache.device
    if ws is not None and not (_on(ws, on) and ws.is_contiguous()):
        raise TypeError("ws: a contiguous tensor on the cache's GPU is wanted")
    _check("us_kv_attend", lib().us_kv_attend(
        cache._there, _seqs(blocks, lens, starts, max_q, on), heads, _rows(q, heads, d, "q", on),
        _rows(out, heads, d, "out", on), _opts(scale, causal, window, max_len, weights, blocks.shape[0], cache.heads, on),
        0 if ws is None else ws.data_ptr(), 0 if ws is None else ws.nbytes, _stream(stream, cache)))


def evict(cache: Cache, blocks, lens, weights, keep: int, recent: int, to_blocks, to_lens, to_weights, index,
          max_len=None, stream=None) -> None:
    """us_kv_evict: the recent and the most attended tokens of every sequence, moved to to_blocks; to_weights gets
    their weights, and zeros for the tokens still to come."""
    heads, batch, on = cache.heads, blocks.shape[0], cache.device
    w, w_stride = _weights(weights, batch, heads, "weights", on)
    ow, ow_stride = (0, 0) if to_weights is None else _weights(to_weights, batch, heads, "to_weights", on)
    rows, width, stride = _table(to_blocks, "to_blocks")
    if rows != batch:
        raise ValueError("to_blocks: one row per sequence is wanted")
    if index.dtype is not _I32 or index.shape != (batch, heads, keep) or not index.is_contiguous():
        raise TypeError(f"index: a contiguous int32 tensor {(batch, heads, keep)} is wanted")
    if not (_on(to_blocks, on) and _on(to_lens, on) and _on(index, on)):
        raise TypeError("to_blocks, to_lens, index: tensors on the cache's GPU are wanted")
    to = _pack_kept(to_blocks.data_ptr(), stride, width, _numbers(to_lens, batch, "to_lens"), ow, ow_stride, index.data_ptr())
    _check("us_kv_evict", lib().us_kv_evict(cache._there, _seqs(blocks, lens, None, 1, on), w, w_stride, max_len or 0,
                                            keep, recent, to, _stream(stream, cache)))


def _workspace(ws, device):
    """Address and bytes of a workspace."""
    if ws is None:
        return 0, 0
    if not (_on(ws, device) and ws.is_contiguous()):
        raise TypeError("ws: a contiguous tensor on the cache's GPU is wanted")
    return ws.data_ptr(), ws.nbytes


def _zeros(n: int, device):
    """A zero-filled workspace of n bytes."""
    return torch.zeros((n + 3) // 4, dtype=_I32, device=device)


def _vector(t, n, dtype, name, device) -> int:
    """Address of n contiguous numbers on GPU `device`; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise TypeError(f"{name}: {n} contiguous {str(dtype)[6:]} numbers are wanted")
    if not _on(t, device):
        raise TypeError(f"{name}: a tensor on the call's GPU is wanted")
    return t.data_ptr()


def rotate(q, k, freq, positions, q_out=None, k_out=None, adjacent: bool = False, norm: bool = False, q_weight=None,
           k_weight=None, eps: float = 1e-6, offset: int = 0, stream=None) -> None:
    """us_kv_rotate: norms (norm=True) of query and key heads, and their rotation by freq (axes, pairs) times
    positions (axes, tokens); in place where no q_out and k_out are given (not for a head that is expanded over several).
    k may be None, and freq (no rotation)."""
    L = lib()
    tokens, heads, d = q.shape
    on = q.get_device() if q.is_cuda else -1
    if on < 0:
        raise TypeError("q: a tensor on a GPU is wanted")
    rows = _rows(q, heads, d, "q", on)
    rows_out = rows if q_out is None else _rows(q_out, heads, d, "q_out", on)
    k_heads, k_rows, k_rows_out = 0, None, None
    if k is not None:
        k_heads = k.shape[1]
        k_rows = _rows(k, k_heads, d, "k", on)
        k_rows_out = k_rows if k_out is None else _rows(k_out, k_heads, d, "k_out", on)
    elif k_out is not None:
        raise TypeError("k_out: there is no k")
    at, pairs, axes, at_pos, stride = _args.turns(freq, positions, tokens, on)
    how = _pack_rotation(at, pairs, axes, at_pos, stride, offset, 1 if adjacent else 0, 1 if norm else 0, eps,
                         _vector(q_weight, d, _F32, "q_weight", on), _vector(k_weight, d, _F32, "k_weight", on))
    _check("us_kv_rotate", L.us_kv_rotate(heads, k_heads, d, rows, rows_out, k_rows, k_rows_out, how,
                                          _stream_on(stream, on, "q")))


def fork_workspace(cache: Cache, blocks, to_blocks):
    """A zero-filled workspace for fork calls between tables of these sizes."""
    n = ctypes.c_size_t(0)
    _check("us_kv_fork_workspace_size", lib().us_kv_fork_workspace_size(cache._packed, blocks.shape[0], to_blocks.shape[0],
                                                                        ctypes.byref(n)))
    return _zeros(n.value, cache.k.device)


def fork(cache: Cache, refs, blocks, lens, parents, to_blocks, to_lens, missing, room=None, ws=None, stream=None) -> None:
    """us_kv_fork: new sequences (to_blocks, to_lens) that go on from the old ones `parents` (None: each from its own),
    with blocks for `room` more tokens each; refs counts the tables' references to every block."""
    on = cache.device
    batch, width, stride = _table(to_blocks, "to_blocks")
    seqs = _seqs(blocks, lens, None, 1, on)
    if not _on(to_blocks, on):
        raise TypeError("to_blocks: a tensor on the cache's GPU is wanted")
    to = _pack_forked(to_blocks.data_ptr(), stride, width, batch, _vector(to_lens, batch, _I32, "to_lens", on))
    at, n = _workspace(ws, on)
    _check("us_kv_fork", lib().us_kv_fork(
        cache._there, _vector(refs, cache.n_blocks, _I32, "refs", on), seqs, _vector(parents, batch, _I32, "parents", on),
        _vector(room, batch, _I32, "room", on), to, _vector(missing, 1, _I32, "missing", on), at, n, _stream(stream, cache)))


def _groups(group_starts, shared, max_group, max_shared, device) -> bytes:
    n = group_starts.shape[0] - 1
    return _pack_groups(_vector(group_starts, n + 1, _I32, "group_starts", device), _vector(shared, n, _I32, "shared", device),
                        n, max_group, max_shared or 0)


def attend_shared_workspace(cache: Cache, q, blocks, group_starts, starts=None, max_q: int = 1, max_group=None,
                            max_shared=None, max_len=None, causal: bool = True):
    """A workspace for attend_shared calls of these sizes. Without max_group every group is taken to be as large as the
    batch, without max_shared as long as the table: the workspace and the launch grow with both."""
    batch, n = blocks.shape[0], ctypes.c_size_t(0)
    at, count = group_starts.data_ptr(), group_starts.shape[0] - 1
    _check("us_kv_attend_shared_workspace_size", lib().us_kv_attend_shared_workspace_size(
        cache._packed, _sizes(blocks, starts, max_q), q.shape[1], q.shape[0],
        _pack_groups(at, at, count, max_group or batch, max_shared or 0),
        _opts(None, causal, 0, max_len, None, batch, cache.heads, cache.device), ctypes.byref(n)))
    return _zeros(n.value, cache.k.device)


def attend_shared(cache: Cache, blocks, lens, q, out, group_starts, shared, starts=None, max_q: int = 1, max_group=None,
                  max_shared=None, max_len=None, scale=None, causal: bool = True, ws=None, stream=None) -> None:
    """us_kv_attend_shared: attend, with the first shared[g] blocks of group g's sequences (group_starts[g] ..
    group_starts[g + 1] - 1) read once for all of them. max_group and max_shared as for the workspace: they also choose
    the kernel."""
    heads, d, on, batch = q.shape[1], cache.head_dim, cache.device, blocks.shape[0]
    at, n = _workspace(ws, on)
    _check("us_kv_attend_shared", lib().us_kv_attend_shared(
        cache._there, _seqs(blocks, lens, starts, max_q, on), heads, _rows(q, heads, d, "q", on), _rows(out, heads, d, "out", on),
        _groups(group_starts, shared, max_group or batch, max_shared, on),
        _opts(scale, causal, 0, max_len, None, batch, cache.heads, on), at, n, _stream(stream, cache)))


def new_summary(cache: Cache):
    """Room for the extremes of every block's keys: uint8 (n_blocks, heads, 2, row(head_dim))."""
    return torch.full((cache.n_blocks, cache.heads, 2, row(cache.head_dim)), 128, dtype=torch.uint8, device=cache.k.device)


def _summary(t, cache) -> int:
    return _args.summary(t, cache.n_blocks, cache.heads, row(cache.head_dim), cache.device)


def summarise(cache: Cache, blocks, lens, summary, starts=None, max_new: int = 1, stream=None) -> None:
    """us_kv_summarise: the extremes of the keys of the blocks that the sequences' last tokens are in, after append."""
    L = lib()
    _check("us_kv_summarise", L.us_kv_summarise(cache._there, _seqs(blocks, lens, starts, max_new, cache.device),
                                                    _summary(summary, cache), _stream(stream, cache)))


def choose_workspace(cache: Cache, blocks, chosen, starts=None, max_q: int = 1):
    """A zero-filled workspace for choose calls of these sizes."""
    n = ctypes.c_size_t(0)
    _check("us_kv_choose_workspace_size", lib().us_kv_choose_workspace_size(
        cache._packed, _sizes(blocks, starts, max_q), chosen.shape[0], chosen.shape[2], ctypes.byref(n)))
    return _zeros(n.value, cache.k.device)


def choose(cache: Cache, summary, blocks, lens, q, scores, chosen, starts=None, max_q: int = 1, max_len=None, sinks: int = 1,
           recent: int = 1, ws=None, stream=None) -> None:
    """us_kv_choose: for every row of q and cache head, the first `sinks`, the last `recent` and else the blocks of
    highest possible score, ascending, then -1: chosen (tokens, heads, top); the scores of all: (tokens, heads, blocks)."""
    L, on = lib(), cache.device
    tokens, heads, _ = q.shape
    at, top = _args.ints(chosen, tokens, cache.heads, "chosen", on)
    at_scores, stride = _args.floats(scores, tokens, cache.heads, "scores", on)
    at_ws, n = _workspace(ws, on)
    _check("us_kv_choose", L.us_kv_choose(
        cache._there, _seqs(blocks, lens, starts, max_q, on), _summary(summary, cache), heads,
        _rows(q, heads, cache.head_dim, "q", on), _pack_choice(at_scores, stride, at, top, sinks, recent, max_len or 0), at_ws, n,
        _stream(stream, cache)))


def attend_chosen_workspace(cache: Cache, q, blocks, chosen, starts=None, max_q: int = 1):
    """A zero-filled workspace for attend_chosen calls of these sizes."""
    n = ctypes.c_size_t(0)
    _check("us_kv_attend_chosen_workspace_size", lib().us_kv_attend_chosen_workspace_size(
        cache._packed, _sizes(blocks, starts, max_q), q.shape[1], q.shape[0], chosen.shape[2], ctypes.byref(n)))
    return _zeros(n.value, cache.k.device)


def attend_chosen(cache: Cache, blocks, lens, q, out, chosen, starts=None, max_q: int = 1, scale=None, ws=None,
                  stream=None) -> None:
    """us_kv_attend_chosen: attend over the blocks chosen[t, h] alone, for row t and cache head h."""
    L, d, on = lib(), cache.head_dim, cache.device
    tokens, heads, _ = q.shape
    at, top = _args.ints(chosen, tokens, cache.heads, "chosen", on)
    at_ws, n = _workspace(ws, on)
    _check("us_kv_attend_chosen", L.us_kv_attend_chosen(
        cache._there, _seqs(blocks, lens, starts, max_q, on), heads, _rows(q, heads, d, "q", on), _rows(out, heads, d, "out", on),
        at, top, None if scale is None else _pack_opts(scale, 1, 0, 0, 0, 0), at_ws, n, _stream(stream, cache)))
