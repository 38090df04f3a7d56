"""Rotations, forks, shared and sparse attention without a GPU: refusals before any work, and the oracle's pins."""
import ctypes
import math

import numpy as np
import pytest

from oracle import kv as ref
from paper_2608_09291_amd import kv
from test_kv_host import BAD

ARG, SHAPE = -1, -2
P = 1 << 20     # an address that nothing here reads: every call below is refused
BIG = 1 << 40
at = ctypes.byref


def _cache():
    return kv.CacheStruct(P, P, P, P, 8, 2, 128)


def _seqs():
    return kv.SeqsStruct(P, 4, 4, 3, P, P, 5)


def _rows():
    return kv.RowsStruct(P, 256, 128, 9, 1)


def _groups():
    return kv.GroupsStruct(P, P, 2, 3, 4)


def _choice():
    return kv.ChoiceStruct(P, 4, P, 3, 1, 1, 0)


def _forked():
    return kv.ForkedStruct(2 * P, 4, 4, 3, 2 * P)


def _calls(cache, seqs, q, out):
    """Every call that takes these, and its status."""
    L, n = kv.lib(), ctypes.c_size_t(7)
    r = [None if x is None else at(x) for x in (cache, seqs, q, out)]
    yield "shared", L.us_kv_attend_shared(*r[:2], 2, *r[2:], at(_groups()), None, P, BIG, None)
    yield "chosen", L.us_kv_attend_chosen(*r[:2], 2, *r[2:], P, 3, None, P, BIG, None)
    yield "choose", L.us_kv_choose(*r[:2], P, 2, r[2], at(_choice()), P, BIG, None)
    yield "summarise", L.us_kv_summarise(*r[:2], P, None)
    yield "fork", L.us_kv_fork(
        r[0], P, r[1], P, P, at(_forked()), P, P, BIG, None)
    yield "shared size", L.us_kv_attend_shared_workspace_size(*r[:2], 2, 9, at(_groups()), None, at(n))
    yield "chosen size", L.us_kv_attend_chosen_workspace_size(*r[:2], 2, 9, 3, at(n))
    yield "choose size", L.us_kv_choose_workspace_size(*r[:2], 9, 3, at(n))
    yield "fork size", L.us_kv_fork_workspace_size(r[0], 3, 3, at(n))


TAKES = {"cache": {"shared", "chosen", "choose", "summarise", "fork", "shared size", "chosen size", "choose size", "fork size"},
         "seqs": {"shared", "chosen", "choose", "summarise", "fork", "shared size", "chosen size", "choose size"},
         "q": {"shared", "chosen", "choose"}, "out": {"shared", "chosen"}}


@pytest.mark.parametrize("which,field,value,status", BAD)
def test_refusals_of_all_calls(which, field, value, status):
    a = [_cache(), _seqs(), _rows(), _rows()]
    setattr(a[which], field, value)
    if field == "dtype" and value == 0 or field == "tokens" and value == 8 or field == "dtype" and value == 2:
        takes = TAKES["out"]                                # (rows that differ from the other ones)
    else:
        takes = TAKES[("cache", "seqs", "q", "out")[which]]
    got = dict(_calls(*a))
    assert {k: got[k] for k in takes} == {k: status for k in takes}


def test_null_structs():
    for hole, name in enumerate(("cache", "seqs", "q", "out")):
        a = [_cache(), _seqs(), _rows(), _rows()]
        a[hole] = None
        got = dict(_calls(*a))
        assert all(got[k] == ARG for k in TAKES[name]), name


# --- rotations -------------------------------------------------------------------------

def _rotate(q_heads=2, k_heads=2, head_dim=128, q=None, q_out=None, k=None, k_out=None, drop=(), **how):
    a = dict(freq=P, pairs=64, axes=1, positions=P, positions_stride=9, offset=0, adjacent=0, norm=1, eps=1e-6, q_weight=P, k_weight=P)
    a.update(how)
    r = dict(q=q or _rows(), q_out=q_out or _rows(), k=k or _rows(), k_out=k_out or _rows())
    r = {name: None if name in drop else at(x) for name, x in r.items()}
    s = kv.RotationStruct(*[a[name] for name, _ in kv.RotationStruct._fields_])
    return kv.lib().us_kv_rotate(q_heads, k_heads, head_dim, r["q"], r["q_out"], r["k"], r["k_out"], None if "how" in drop else at(s), None)


@pytest.mark.parametrize("change,status", [
    (dict(drop=("how",)), ARG), (dict(drop=("q",)), ARG), (dict(drop=("q_out",)), ARG), (dict(drop=("k",)), ARG),
    (dict(drop=("k_out",)), ARG), (dict(drop=("k", "k_out")), SHAPE), (dict(k_heads=0), SHAPE), (dict(q_heads=0), SHAPE),
    (dict(q_heads=65536), SHAPE), (dict(k_heads=-1), SHAPE), (dict(k_heads=65536), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(head_dim=257), SHAPE), (dict(pairs=-1), SHAPE), (dict(pairs=65), SHAPE), (dict(axes=0), SHAPE), (dict(axes=5), SHAPE),
    (dict(axes=2, positions_stride=8), SHAPE), (dict(freq=None), ARG), (dict(positions=None), ARG), (dict(freq=P + 2), ARG),
    (dict(positions=P + 1), ARG), (dict(adjacent=2), ARG), (dict(norm=2), ARG), (dict(norm=-1), ARG), (dict(eps=0.0), ARG),
    (dict(eps=-1.0), ARG), (dict(eps=math.nan), ARG), (dict(eps=math.inf), ARG), (dict(norm=0), ARG),
    (dict(norm=0, q_weight=None), ARG), (dict(norm=0, q_weight=None, k_weight=None, pairs=0), ARG), (dict(q_weight=P + 1), ARG),
    (dict(k_weight=P + 2), ARG), (dict(q=kv.RowsStruct(P, 256, 128, 8, 1)), SHAPE), (dict(k=kv.RowsStruct(P, 256, 128, 8, 1)), SHAPE),
    (dict(k_out=kv.RowsStruct(P, 256, 128, 10, 1)), SHAPE), (dict(q_out=kv.RowsStruct(P, 256, 128, 9, 0)), ARG),
    (dict(k=kv.RowsStruct(P, 256, 128, 9, 2)), ARG), (dict(k_out=kv.RowsStruct(P + 1, 256, 128, 9, 1)), ARG),
    (dict(q=kv.RowsStruct(P, -1, 128, 9, 1)), SHAPE), (dict(q_out=kv.RowsStruct(P, 256, -128, 9, 1)), SHAPE)])
def test_rotate_refuses(change, status):
    assert _rotate(**change) == status


# --- forks -----------------------------------------------------------------------------

@pytest.mark.parametrize("change,status", [
    (dict(refs=None), ARG), (dict(refs=P + 2), ARG), (dict(parents=P + 1), ARG), (dict(room=P + 1), ARG), (dict(missing=None), ARG),
    (dict(missing=P + 2), ARG), (dict(to=None), ARG), (dict(blocks=None), ARG), (dict(blocks=2 * P + 2), ARG), (dict(lens=None), ARG),
    (dict(lens=2 * P + 1), ARG), (dict(width=3), SHAPE), (dict(width=(1 << 22) + 1, stride=1 << 23), SHAPE), (dict(stride=3), SHAPE),
    (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(blocks=P), ARG), (dict(lens=P), ARG), (dict(ws=None), ARG),
    (dict(ws=P + 8), ARG), (dict(ws_bytes=-1), ARG), (dict(heads=32768), SHAPE)])
def test_fork_refuses(change, status):
    L, n = kv.lib(), ctypes.c_size_t(0)
    assert L.us_kv_fork_workspace_size(at(_cache()), 3, 3, at(n)) == 0 and n.value > 0
    a = dict(refs=P, parents=P, room=P, missing=P, blocks=2 * P, lens=2 * P, width=4, stride=4, batch=3, ws=P, ws_bytes=BIG, heads=2)
    a.update(change)
    if a["ws_bytes"] < 0:
        a["ws_bytes"] = n.value - 1
    c = _cache()
    c.heads = a["heads"]
    to = kv.ForkedStruct(a["blocks"], a["stride"], a["width"], a["batch"], a["lens"])
    r = L.us_kv_fork(at(c), a["refs"], at(_seqs()), a["parents"], a["room"], None if "to" in change else at(to), a["missing"], a["ws"],
                     a["ws_bytes"], None)
    assert r == status


@pytest.mark.parametrize("at_first,stride,width,batch,meets", [
    (24, 6, 4, 3, False), (23, 6, 4, 3, False), (15, 6, 4, 3, True), (16, 9, 6, 2, False), (-4, 9, 5, 1, True), (-5, 9, 5, 1, False),
    (4, 10, 6, 3, False), (4, 10, 7, 3, True), (3, 10, 6, 3, True), (-6, 10, 6, 3, False), (-6, 10, 7, 2, True), (4, 11, 6, 2, True)])
def test_fork_refuses_tables_that_share_memory(at_first, stride, width, batch, meets):
    # The old table: 3 rows of 4 entries, as far apart as the new ones' are, or 6. (What is refused after it: SHAPE.)
    seqs, c = _seqs(), _cache()
    seqs.stride = stride if stride > 9 and stride != 11 else 6
    c.heads = 32768
    seqs.blocks = 2 * P
    own = {seqs.stride * i + j for i in range(3) for j in range(4)}
    assert meets == bool(own & {at_first + stride * i + j for i in range(batch) for j in range(width)})
    to = kv.ForkedStruct(2 * P + 4 * at_first, stride, width, batch, 4 * P)
    assert kv.lib().us_kv_fork(at(c), P, at(seqs), P, P, at(to), P, P, BIG, None) == (ARG if meets else SHAPE)


def test_fork_workspace_refuses():
    L, n = kv.lib(), ctypes.c_size_t(7)
    for batch, to_batch in ((0, 3), (3, 0), (65536, 3), (3, 65536), (-1, 3)):
        assert L.us_kv_fork_workspace_size(at(_cache()), batch, to_batch, at(n)) == SHAPE
    assert L.us_kv_fork_workspace_size(at(_cache()), 3, 3, None) == ARG and n.value == 7


# --- shared and sparse attention -----------------------------------------------------------

OPTS = [("scale", -1.0, ARG), ("scale", math.nan, ARG), ("scale", math.inf, ARG), ("causal", 2, ARG), ("window", -1, ARG),
        ("window", 5, ARG), ("max_len", -1, SHAPE), ("weights", P, ARG)]


@pytest.mark.parametrize("field,value,status", OPTS + [("causal", 0, None)])
def test_options_are_refused(field, value, status):
    L, n = kv.lib(), ctypes.c_size_t(0)
    o = kv.AttendOpts(0.0, 1, 0, 0, None, 256)
    setattr(o, field, value)
    c, s, q = at(_cache()), at(_seqs()), at(_rows())
    if status is not None:
        assert L.us_kv_attend_shared(c, s, 2, q, q, at(_groups()), at(o), P, BIG, None) == status
        assert L.us_kv_attend_shared_workspace_size(c, s, 2, 9, at(_groups()), at(o), at(n)) == status
    assert L.us_kv_attend_chosen(c, s, 2, q, q, P, 3, at(o), P, BIG, None) == (status or ARG)


@pytest.mark.parametrize("field,value,status", [
    ("starts", None, ARG), ("shared", None, ARG), ("starts", P + 2, ARG), ("shared", P + 1, ARG), ("groups", 0, SHAPE),
    ("groups", 65536, SHAPE), ("max_group", 0, SHAPE), ("max_group", 65536, SHAPE), ("max_shared", -1, SHAPE), ("max_shared", 5, SHAPE)])
def test_groups_are_refused(field, value, status):
    L, n = kv.lib(), ctypes.c_size_t(0)
    g = _groups()
    setattr(g, field, value)
    c, s, q = at(_cache()), at(_seqs()), at(_rows())
    assert L.us_kv_attend_shared(c, s, 2, q, q, at(g), None, P, BIG, None) == status
    assert L.us_kv_attend_shared_workspace_size(c, s, 2, 9, at(g), None, at(n)) == status


def test_shared_refuses_heads_rows_and_workspaces():
    L, n = kv.lib(), ctypes.c_size_t(0)
    c, s, q, g = at(_cache()), at(_seqs()), at(_rows()), at(_groups())
    for heads in (0, 1, 3, -2, 65538):
        assert L.us_kv_attend_shared(c, s, heads, q, q, g, None, P, BIG, None) == SHAPE
        assert L.us_kv_attend_chosen(c, s, heads, q, q, P, 3, None, P, BIG, None) == SHAPE
        assert L.us_kv_choose(c, s, P, heads, q, at(_choice()), P, BIG, None) == SHAPE
    assert L.us_kv_attend_shared(c, s, 2, q, q, None, None, P, BIG, None) == ARG
    many = kv.SeqsStruct(P, 4, 4, 3, P, P, 1 << 24)
    assert L.us_kv_attend_shared(c, at(many), 2, q, q, g, None, P, BIG, None) == SHAPE
    assert L.us_kv_attend_shared_workspace_size(c, s, 2, 9, g, None, at(n)) == 0 and n.value > 0
    for ws, size in ((None, n.value), (P + 4, n.value), (P, n.value - 1)):
        assert L.us_kv_attend_shared(c, s, 2, q, q, g, None, ws, size, None) == ARG
    assert L.us_kv_attend_shared_workspace_size(c, s, 2, 9, g, None, None) == ARG
    assert L.us_kv_attend_shared_workspace_size(c, s, 2, 0, g, None, at(n)) == SHAPE


@pytest.mark.parametrize("change,status", [
    (dict(chosen=None), ARG), (dict(chosen=P + 2), ARG), (dict(top=0), SHAPE), (dict(top=-1), SHAPE), (dict(top=(1 << 16) + 1), SHAPE),
    (dict(tokens=65536), SHAPE), (dict(ws=None), ARG), (dict(ws=P + 4), ARG), (dict(ws_bytes=-1), ARG)])
def test_chosen_refuses(change, status):
    L, n = kv.lib(), ctypes.c_size_t(0)
    a = dict(chosen=P, top=400, tokens=9, ws=P, ws_bytes=BIG)
    a.update(change)
    q = kv.RowsStruct(P, 256, 128, a["tokens"], 1)
    c, s = at(_cache()), at(_seqs())
    assert L.us_kv_attend_chosen_workspace_size(c, s, 2, 9, 400, at(n)) == 0 and n.value > 0
    size = n.value - 1 if a["ws_bytes"] < 0 else a["ws_bytes"]
    assert L.us_kv_attend_chosen(c, s, 2, at(q), at(q), a["chosen"], a["top"], None, a["ws"], size, None) == status
    if "top" in change or "tokens" in change:
        assert L.us_kv_attend_chosen_workspace_size(c, s, 2, a["tokens"], a["top"], at(n)) == status
    assert L.us_kv_attend_chosen_workspace_size(c, s, 2, 9, 400, None) == ARG


@pytest.mark.parametrize("change,status", [
    (dict(choice=None), ARG), (dict(scores=None), ARG), (dict(scores=P + 2), ARG), (dict(chosen=None), ARG), (dict(chosen=P + 1), ARG),
    (dict(scores_stride=3), SHAPE), (dict(top=0), SHAPE), (dict(top=(1 << 16) + 1), SHAPE), (dict(sinks=-1), SHAPE),
    (dict(recent=-1), SHAPE), (dict(sinks=2, recent=2), SHAPE), (dict(sinks=(1 << 31) - 1, recent=(1 << 31) - 1), SHAPE),
    (dict(max_len=-1), SHAPE), (dict(summary=None), ARG), (dict(summary=P + 8), ARG), (dict(ws=None), ARG), (dict(ws=P + 8), ARG),
    (dict(ws_bytes=-1), ARG), (dict(tokens=65536), SHAPE)])
def test_choose_refuses(change, status):
    L, n = kv.lib(), ctypes.c_size_t(0)
    a = dict(scores=P, scores_stride=4, chosen=P, top=3, sinks=1, recent=1, max_len=0, summary=P, ws=P, ws_bytes=BIG, tokens=9)
    a.update(change)
    c, s = at(_cache()), at(_seqs())
    assert L.us_kv_choose_workspace_size(c, s, 9, 3, at(n)) == 0 and n.value > 0
    size = n.value - 1 if a["ws_bytes"] < 0 else a["ws_bytes"]
    choice = kv.ChoiceStruct(*[a[name] for name, _ in kv.ChoiceStruct._fields_])
    q = kv.RowsStruct(P, 256, 128, a["tokens"], 1)
    assert L.us_kv_choose(c, s, a["summary"], 2, at(q), None if "choice" in change else at(choice), a["ws"], size, None) == status
    if "summary" in change:
        assert L.us_kv_summarise(c, s, a["summary"], None) == status
    assert L.us_kv_choose_workspace_size(c, s, 9, 3, None) == ARG
    assert L.us_kv_choose_workspace_size(c, s, 0, 3, at(n)) == SHAPE


def test_binding_refuses_host_tensors():
    """Nothing on the host gets as far as a launch."""
    torch = pytest.importorskip("torch")
    i32 = torch.int32
    c = kv.new_cache(4, 2, 80, device="cpu")
    blocks, lens, refs = torch.zeros((3, 2), dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(4, dtype=i32)
    x, one, chosen = torch.zeros((3, 2, 80)), torch.zeros(1, dtype=i32), torch.zeros((3, 2, 2), dtype=i32)
    summary, scores, groups = kv.new_summary(c), torch.zeros((3, 2, 2)), torch.zeros(2, dtype=i32)
    for call in (lambda: kv.rotate(x, x, torch.zeros((1, 40)), lens), lambda: kv.rotate(x, None, None, None, norm=True),
                 lambda: kv.fork(c, refs, blocks, lens, None, blocks.clone(), lens.clone(), one),
                 lambda: kv.attend_shared(c, blocks, lens, x, x, groups, one), lambda: kv.summarise(c, blocks, lens, summary),
                 lambda: kv.choose(c, summary, blocks, lens, x, scores, chosen),
                 lambda: kv.attend_chosen(c, blocks, lens, x, x, chosen)):
        with pytest.raises(TypeError):
            call()


# --- the oracle against hand-worked cases -----------------------------------------------

def test_oracle_rotation_by_hand():
    x = np.array([[[3.0, 4.0, 5.0, 7.0]]], np.float32)
    f = np.array([[0.0, 0.0], [math.pi / 2, 0.0]], np.float32)
    pos = np.array([[9], [1]])
    assert np.allclose(ref.rotate(x, f, pos), [[[-5, 4, 3, 7]]], atol=1e-6)
    assert np.allclose(ref.rotate(x, f, pos, adjacent=True), [[[-4, 3, 5, 7]]], atol=1e-6)
    assert np.allclose(ref.rotate(x, f, pos, offset=1), [[[-3, 4, -5, 7]]], atol=1e-6)      # two quarters
    n = ref.rotate(x[..., :2], eps=1e-30)
    assert np.allclose(n, np.array([3, 4]) / math.sqrt(12.5))
    assert np.allclose(ref.rotate(x[..., :2], eps=1e-30, weight=np.array([2, 0.5])), np.array([6, 2]) / math.sqrt(12.5))


def test_oracle_fork_by_hand():
    refs, blocks = [1, 1, 0, 1, 0, 0], [[0, 1], [3, -1]]                # sequences of 70 and 10 tokens
    to, lens, after, copies, missing = ref.fork(refs, blocks, [70, 10], [0, 0, -1], [0, 60, 1], 3)
    assert to == [[0, 1, -1], [0, 2, 4], [5, -1, -1]] and lens == [70, 70, 0] and missing == 0
    assert after == [2, 1, 1, 0, 1, 1] and copies == [(1, 2)]
    assert ref.fork(refs, blocks, [70, 10], [0, 0, 0, 0, 1], [0, 0, 0, 100, 0], 3)[4] == 1
    assert ref.fork([2, 1, 0], [[0]], [64], [0], [1], 2)[0] == [[0, 2]]


def test_oracle_choice_by_hand():
    s = [5.0, 1.0, 9.0, 9.0, math.nan, 2.0]
    all_ = [True] * 6
    assert ref.choose(s, all_, 2, 0, 0) == [2, 3] and ref.choose(s, all_, 1, 0, 0) == [2]
    assert ref.choose(s, all_, 3, 0, 1) == [2, 3, 5] and ref.choose(s, all_, 3, 2, 1) == [0, 1, 5]
    assert ref.choose(s, all_, 9, 0, 0) == [0, 1, 2, 3, 4, 5] and ref.choose(s, all_, 5, 0, 0) == [0, 1, 2, 3, 5]
    assert ref.choose(s, [True, True, False, True, True, False], 2, 0, 1) == [0, 3]
    q = np.array([[1.0, -2.0], [math.nan, 0.0]])
    summary = np.array([[128 - 5, 128 - 7], [128 + 4, 128 + 6]], np.uint8)
    assert ref.score(summary, 0.5, q) == np.float32(0.5 * (4 + 14))
    assert ref.score(summary, 0.5, q[1:]) == -np.inf
