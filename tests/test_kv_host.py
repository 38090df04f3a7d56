"""The 8-bit key/value cache without a GPU: exported symbols, the layout, refusals before any work, and the oracle's pins."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from oracle import kv as ref
from paper_2608_09291_amd import binding, kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, SHAPE = -1, -2
P = 1 << 20     # an address that nothing here reads: every call below is refused


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "us_kv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(us_kv_[a-z0-9_]+)\s*\(", text))
    assert declared == set(kv.EXPORTS)
    for name in declared:
        assert hasattr(binding.lib(), name), name


def test_row():
    for d in range(1, 257):
        assert kv.row(d) == ref.row_of(d)
    for d in (0, -1, 257, 1 << 30):
        assert kv.lib().us_kv_row(d) == 0
        with pytest.raises(ValueError):
            kv.row(d)


@pytest.mark.parametrize("row", [64, 96, 128, 192, 256])
def test_layout_has_a_byte_for_every_value(row):
    for keys in (True, False):
        assert sorted(ref.places(row, keys).ravel()) == list(range(64 * row))


def _valid():
    return (kv.CacheStruct(P, P, P, P, 8, 2, 128), kv.SeqsStruct(P, 4, 4, 3, P, P, 5),
            kv.RowsStruct(P, 256, 128, 9, 1), kv.RowsStruct(P, 256, 128, 9, 1))


# field of which struct (cache, seqs, first rows, second rows), value, status
BAD = [
    (0, "k", None, ARG), (0, "v", None, ARG), (0, "k_scale", None, ARG), (0, "v_scale", None, ARG),
    (0, "k", P + 8, ARG), (0, "v", P + 1, ARG), (0, "k_scale", P + 2, ARG), (0, "v_scale", P + 1, ARG),
    (0, "n_blocks", 0, SHAPE), (0, "heads", 0, SHAPE), (0, "heads", 65536, SHAPE), (0, "head_dim", 0, SHAPE),
    (0, "head_dim", 257, SHAPE),
    (1, "blocks", None, ARG), (1, "lens", None, ARG), (1, "blocks", P + 2, ARG), (1, "lens", P + 1, ARG),
    (1, "starts", P + 2, ARG), (1, "starts", None, SHAPE), (1, "batch", 0, SHAPE), (1, "batch", 65536, SHAPE),
    (1, "width", 0, SHAPE), (1, "width", 1 << 26, SHAPE), (1, "stride", 3, SHAPE), (1, "max_new", 0, SHAPE),
    (2, "data", None, ARG), (2, "data", P + 1, ARG), (2, "dtype", 3, ARG), (2, "dtype", -1, ARG), (2, "dtype", 0, ARG),
    (2, "tokens", 0, SHAPE), (2, "tokens", 8, SHAPE), (2, "token_stride", -1, SHAPE), (3, "head_stride", -1, SHAPE),
    (3, "data", None, ARG), (3, "dtype", 2, ARG),
]


@pytest.mark.parametrize("which,field,value,status", BAD)
def test_refusals_of_all_calls(which, field, value, status):
    L = kv.lib()
    a = _valid()
    setattr(a[which], field, value)
    r = [ctypes.byref(x) for x in a]
    assert L.us_kv_append(*r, None) == status
    assert L.us_kv_read(*r, None) == status
    assert L.us_kv_attend(r[0], r[1], 2, r[2], r[3], None, P, 1 << 40, None) == status
    if which < 2:
        n = ctypes.c_size_t(7)
        assert L.us_kv_attend_workspace_size(r[0], r[1], 2, 9, None, ctypes.byref(n)) == status
        assert n.value == 7
    if which < 2 and field not in ("starts", "max_new"):
        to = kv.KeptStruct(P, 4, 4, P, P, 256, P)
        assert L.us_kv_evict(r[0], r[1], P, 256, 0, 8, 2, ctypes.byref(to), None) == status


def test_null_structs():
    L = kv.lib()
    for hole in range(4):
        r = [ctypes.byref(x) for x in _valid()]
        r[hole] = None
        assert L.us_kv_append(*r, None) == ARG and L.us_kv_read(*r, None) == ARG
        assert L.us_kv_attend(r[0], r[1], 2, r[2], r[3], None, P, 1 << 40, None) == ARG


@pytest.mark.parametrize("field,value,status", [
    ("scale", -1.0, ARG), ("scale", math.nan, ARG), ("scale", math.inf, ARG), ("causal", 2, ARG), ("causal", -1, ARG),
    ("window", -1, ARG), ("max_len", -1, SHAPE), ("weights", P + 2, ARG), ("weights_stride", 255, SHAPE)])
def test_attend_refuses_options(field, value, status):
    L = kv.lib()
    a = [ctypes.byref(x) for x in _valid()]
    o = kv.AttendOpts(0.0, 1, 0, 0, P, 256)
    setattr(o, field, value)
    n = ctypes.c_size_t(0)
    assert L.us_kv_attend(a[0], a[1], 2, a[2], a[3], ctypes.byref(o), P, 1 << 40, None) == status
    assert L.us_kv_attend_workspace_size(a[0], a[1], 2, 9, ctypes.byref(o), ctypes.byref(n)) == status


def test_attend_refuses_heads_windows_and_workspaces():
    L = kv.lib()
    a = [ctypes.byref(x) for x in _valid()]
    for heads in (0, 1, 3, -2, 65538):
        assert L.us_kv_attend(a[0], a[1], heads, a[2], a[3], None, P, 1 << 40, None) == SHAPE
    o = kv.AttendOpts(0.0, 0, 5, 0, None, 0)                # a window without the causal mask
    assert L.us_kv_attend(a[0], a[1], 2, a[2], a[3], ctypes.byref(o), P, 1 << 40, None) == ARG
    o = kv.AttendOpts(0.0, 1, 0, 0, P, 256)
    n = ctypes.c_size_t(0)
    assert L.us_kv_attend_workspace_size(a[0], a[1], 2, 9, ctypes.byref(o), ctypes.byref(n)) == 0 and n.value > 0
    for ws, size in ((None, n.value), (P + 4, n.value), (P, n.value - 1)):
        assert L.us_kv_attend(a[0], a[1], 2, a[2], a[3], ctypes.byref(o), ws, size, None) == ARG
    assert L.us_kv_attend_workspace_size(a[0], a[1], 2, 9, ctypes.byref(o), None) == ARG
    assert L.us_kv_attend_workspace_size(a[0], a[1], 2, 0, ctypes.byref(o), ctypes.byref(n)) == SHAPE


@pytest.mark.parametrize("change,status", [
    (dict(weights=None), ARG), (dict(weights=P + 1), ARG), (dict(to=None), ARG), (dict(blocks=None), ARG),
    (dict(lens=None), ARG), (dict(index=None), ARG), (dict(blocks=P + 2), ARG), (dict(index=P + 1), ARG),
    (dict(to_weights=P + 2), ARG), (dict(lens=P + 3), ARG), (dict(keep=0), SHAPE), (dict(recent=-1), SHAPE), (dict(recent=101), SHAPE),
    (dict(max_len=-1), SHAPE), (dict(width=1), SHAPE), (dict(width=0), SHAPE), (dict(stride=1), SHAPE),
    (dict(w_stride=255), SHAPE), (dict(to_w_stride=99), SHAPE)])
def test_evict_refuses(change, status):
    a = dict(weights=P, w_stride=256, max_len=0, keep=100, recent=10, blocks=P, stride=2, width=2, lens=P, to_weights=P,
             to_w_stride=100, index=P)
    a.update(change)
    to = kv.KeptStruct(a["blocks"], a["stride"], a["width"], a["lens"], a["to_weights"], a["to_w_stride"], a["index"])
    c, s, _, _ = _valid()
    r = kv.lib().us_kv_evict(ctypes.byref(c), ctypes.byref(s), a["weights"], a["w_stride"], a["max_len"], a["keep"],
                             a["recent"], None if "to" in change else ctypes.byref(to), None)
    assert r == status


def test_evict_refuses_tables_wider_than_any():
    c, s, _, _ = _valid()
    for width in ((1 << 22) + 1, 1 << 25, 1 << 26, (1 << 31) - 1):
        to = kv.KeptStruct(P, width, width, P, P, 256, P)
        assert kv.lib().us_kv_evict(ctypes.byref(c), ctypes.byref(s), P, 256, 0, 100, 10, ctypes.byref(to), None) == SHAPE


def test_evict_refuses_to_write_what_it_reads():
    """Lengths and weights of what is kept have places of their own: other workgroups still read the sequences'."""
    c, s, _, _ = _valid()
    s.lens = 2 * P
    for lens, weights in ((2 * P, 4 * P), (2 * P, None), (5 * P, 3 * P)):
        to = kv.KeptStruct(P, 4, 4, lens, weights, 256, 6 * P)
        assert kv.lib().us_kv_evict(ctypes.byref(c), ctypes.byref(s), 3 * P, 256, 0, 100, 10, ctypes.byref(to), None) == ARG


def test_binding_refuses_tensors():
    torch = pytest.importorskip("torch")
    c = kv.new_cache(4, 2, 80, device="cpu")
    blocks, lens = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    x = torch.zeros((3, 2, 80))
    for bad in (dict(blocks=blocks.long()), dict(blocks=blocks[0]), dict(blocks=blocks.t()), dict(lens=lens[:2]),
                dict(lens=lens.float()), dict(k=x.double()), dict(k=x[:, :1]), dict(k=x[..., :79]),
                dict(k=x.transpose(1, 2).contiguous().transpose(1, 2)), dict(starts=lens), dict(starts=lens.long())):
        a = dict(blocks=blocks, lens=lens, k=x, v=x)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            kv.append(c, **a)
    with pytest.raises(TypeError):
        kv.Cache(c.k.float(), c.v, c.k_scale, c.v_scale, 80).struct()
    with pytest.raises(TypeError):
        kv.Cache(c.k, c.v, c.k_scale[:, :1], c.v_scale, 80).struct()
    with pytest.raises(TypeError):
        kv.Cache(c.k, c.v, c.k_scale, c.v_scale, 128).struct()


def test_binding_refuses_host_tensors():
    """Nothing on the host gets as far as a launch."""
    torch = pytest.importorskip("torch")
    c = kv.new_cache(4, 2, 80, device="cpu")
    blocks, lens = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    x, w = torch.zeros((3, 2, 80)), torch.zeros((3, 2, 128))
    for call in (lambda: kv.append(c, blocks, lens, x, x), lambda: kv.read(c, blocks, lens, x, x),
                 lambda: kv.attend(c, blocks, lens, x, x), lambda: kv.attend(c, blocks, lens, x, x, weights=w),
                 lambda: kv.attend(c, blocks, lens, x, x, ws=w),
                 lambda: kv.evict(c, blocks, lens, w, 64, 1, blocks, lens, None, torch.zeros((3, 2, 64), dtype=torch.int32)),
                 lambda: kv.append(c, blocks, None, x, x), lambda: kv.append(c, blocks, lens, x, 3)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(TypeError):
        kv.Cache(c.k, c.v[:3], c.k_scale, c.v_scale, 80)
    with pytest.raises(TypeError):
        kv.Cache(c.k, c.v.transpose(0, 1), c.k_scale, c.v_scale, 80)
    with pytest.raises(TypeError):
        kv.Cache(c.k, c.v, c.k_scale, c.v_scale.half(), 80)
    # a cache on the host is refused by the library
    assert c._there is None
    _, s, r, _ = _valid()
    assert kv.lib().us_kv_read(c._there, ctypes.byref(s), ctypes.byref(r), ctypes.byref(r), None) == ARG


# --- the oracle against hand-worked cases --------------------------------------

def test_oracle_append_by_hand():
    codes, scales = np.full((2, 1, 64 * 64), 77, np.uint8), np.zeros((2, 1), np.float32)
    x = np.zeros((2, 1, 3), np.float32)
    x[0, 0] = [127.0, -63.5, 0.5]            # scale 1; halves to even: -64 and 0
    ref.append(codes, scales, 3, True, [[1]], [1], None, x[:1])
    assert scales[1, 0] == 1.0
    assert [codes[1, 0, ref.key_byte(0, d)] for d in range(3)] == [255, 64, 128]
    x[1, 0] = [254.0, np.nan, -np.inf]       # scale 2: 127 -> 64 (63.5), -64 -> -32
    ref.append(codes, scales, 3, True, [[1]], [2], None, x[1:])
    assert scales[1, 0] == 2.0
    assert [codes[1, 0, ref.key_byte(0, d)] for d in range(3)] == [192, 96, 128]
    assert [codes[1, 0, ref.key_byte(1, d)] for d in range(3)] == [255, 128, 1]
    assert codes[0].min() == 77              # the other block is untouched


def test_oracle_attend_by_hand():
    codes, scales = np.full((1, 1, 64 * 64), 128, np.uint8), np.ones((1, 1), np.float32)
    v = codes.copy()
    codes[0, 0, ref.key_byte(0, 0)], codes[0, 0, ref.key_byte(1, 0)] = 128, 129
    v[0, 0, ref.value_byte(0, 0)], v[0, 0, ref.value_byte(1, 0)] = 128 + 10, 128 - 30
    q = np.full((2, 1, 1), math.log(3.0))
    out, _, w, _ = ref.attend(codes, scales, v, scales, 1, [[0]], [2], [0, 2], q, scale=1.0)
    assert out[:, 0, 0] == pytest.approx([10.0, 0.25 * 10 - 0.75 * 30])
    assert w[0][0] == pytest.approx([1.25, 0.75])
    out, _, _, _ = ref.attend(codes, scales, v, scales, 1, [[0]], [2], [0, 2], q, scale=1.0, causal=False)
    assert out[0, 0, 0] == pytest.approx(out[1, 0, 0]) == pytest.approx(-20.0)
    out, _, _, _ = ref.attend(codes, scales, v, scales, 1, [[0]], [2], [0, 3], np.ones((3, 1, 1)), window=1)
    assert list(out[:, 0, 0]) == [0.0, 10.0, -30.0]   # a query before the first key; windows of one


def test_oracle_kept_by_hand():
    assert ref.kept([1.0, 5.0, 5.0, 5.0, 9.0, 0.0], 6, 4, 1) == [1, 2, 4, 5]
    assert ref.kept([math.nan, -math.inf, 1.0], 3, 2, 0) == [1, 2]
    assert ref.kept([3.0, 1.0], 2, 5, 1) == [0, 1]
    assert ref.kept([3.0, 1.0, 2.0], 3, 2, 2) == [1, 2]


def test_workspace_sizes_of_edge_shapes():
    """Sizes exist from one token to long tables and many units, and grow with what has to be kept."""
    L = kv.lib()
    n = ctypes.c_size_t(0)
    for batch, heads, width, max_new, q_heads in ((1, 1, 1, 1, 1), (1, 8, 1 << 14, 1, 64), (65535, 8, 2000, 1, 8),
                                                  (3, 2, 100, 5000, 16), (1, 1, 1 << 20, 100, 1)):
        c = kv.CacheStruct(P, P, P, P, 8, heads, 128)
        s = kv.SeqsStruct(P, width, width, batch, P, P, max_new)
        for weights in (None, P):
            o = kv.AttendOpts(0.0, 1, 0, 0, weights, width * 64)
            r = L.us_kv_attend_workspace_size(ctypes.byref(c), ctypes.byref(s), q_heads, batch * max_new, ctypes.byref(o),
                                              ctypes.byref(n))
            assert r == 0 and (n.value >= 4 * q_heads * batch * max_new or not weights), (batch, heads, width)
            assert n.value < 1 << 42


@pytest.mark.parametrize("batch,heads,width,max_new,tokens,q_heads", [
    (65535, 128, 10, 1, 65535, 128), (65535, 65535, 1, 1, 65535, 65535),   # single tokens: as many as batch and heads allow
    (1, 8, 1000, 1 << 25, 100, 8), (3, 64, 4000, 1 << 20, 50, 64),         # a high bound of the new tokens, few rows
    (2, 4, 2000, 1 << 23, 1000, 16)])
def test_large_calls_have_a_plan(batch, heads, width, max_new, tokens, q_heads):
    c = kv.CacheStruct(P, P, P, P, 8, heads, 128)
    s = kv.SeqsStruct(P, width, width, batch, P, P, max_new)
    n = ctypes.c_size_t(0)
    assert kv.lib().us_kv_attend_workspace_size(ctypes.byref(c), ctypes.byref(s), q_heads, tokens, None, ctypes.byref(n)) == 0


def test_route():
    """Single tokens go to the kernel for few rows, whole prompts to the other; refusals as elsewhere."""
    torch = pytest.importorskip("torch")
    c = kv.new_cache(4, 8, 128, device="cpu")
    blocks, starts = torch.zeros((2, 100), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        r = kv.attend_route(c, torch.zeros((2, 32, 128), dtype=dtype), blocks)
        assert r["prompt"] == 0 and r["tile_rows"] == 16 and (r["split_keys"] - 1) * r["part_blocks"] < 100
        r = kv.attend_route(c, torch.zeros((8000, 32, 128), dtype=dtype), blocks, starts=starts, max_q=6000)
        assert r == dict(prompt=1, tile_rows=256, split_keys=1, part_blocks=100)
    a, out = _valid(), kv.AttendRouteInfo()
    r = [ctypes.byref(x) for x in a]
    f = kv.lib().us_kv_attend_route
    assert f(r[0], r[1], 2, 9, 1, None, ctypes.byref(out)) == 0
    assert f(r[0], r[1], 2, 9, 1, None, None) == ARG and f(r[0], r[1], 2, 9, 3, None, ctypes.byref(out)) == ARG
    assert f(None, r[1], 2, 9, 1, None, ctypes.byref(out)) == ARG and f(r[0], None, 2, 9, 1, None, ctypes.byref(out)) == ARG
    assert f(r[0], r[1], 3, 9, 1, None, ctypes.byref(out)) == SHAPE and f(r[0], r[1], 2, 0, 1, None, ctypes.byref(out)) == SHAPE


def test_packed_structs_are_the_c_structs():
    for pack, struct, values in ((kv._pack_cache, kv.CacheStruct, (1 << 40, 2, 3, 4, 5, 6, 7)),
                                 (kv._pack_seqs, kv.SeqsStruct, (1, 1 << 40, 3, 4, 5, 6, 7)),
                                 (kv._pack_rows, kv.RowsStruct, (1, 1 << 40, 3, 4, 2)),
                                 (kv._pack_opts, kv.AttendOpts, (0.5, 1, 2, 3, 4, 1 << 40)),
                                 (kv._pack_kept, kv.KeptStruct, (1, 1 << 40, 3, 4, 5, 6, 1 << 41))):
        raw = pack(*values)
        assert len(raw) == ctypes.sizeof(struct)
        s = struct.from_buffer_copy(raw)
        assert tuple(getattr(s, name) for name, _ in struct._fields_) == values
