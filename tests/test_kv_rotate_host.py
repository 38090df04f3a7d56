"""Rotations whose outputs share memory are refused before any work: rows that lie on each other would be turned more
than once, or by another row's position."""
import ctypes
import random

import pytest

from paper_2608_09291_amd import kv

ARG, SHAPE = -1, -2
P = 1 << 20     # an address that nothing here reads: every call below is refused
at = ctypes.byref
T, H, D = 9, 2, 128


def _rotate(q=(P, 256, 128), q_out=(P, 256, 128), k=(2 * P, 256, 128), k_out=(2 * P, 256, 128), tokens=T, q_heads=H, k_heads=H, head_dim=D):
    rows = [kv.RowsStruct(*r, tokens, 1) for r in (q, q_out, k, k_out)]
    # (axes of a stride that is too short: refused, but after the rows)
    s = kv.RotationStruct(P, 64, 2, P, 0, 0, 0, 0, 0.0, None, None)
    return kv.lib().us_kv_rotate(q_heads, k_heads, head_dim, *map(at, rows), at(s), None)


@pytest.mark.parametrize("change", [
    dict(q=(P, 256, 0), q_out=(P, 256, 0)), dict(q=(P, 0, 128), q_out=(P, 0, 128)), dict(k=(2 * P, 256, 0), k_out=(2 * P, 256, 0)),
    dict(q_out=(3 * P, 256, 0)), dict(q_out=(3 * P, 0, 128)), dict(k_out=(3 * P, 256, 127)), dict(k_out=(3 * P, 127, 128 * 9)),
    dict(q_out=(P, 512, 128)), dict(q_out=(P, 256, 256)), dict(q=(P, 0, 128)), dict(k=(2 * P, 256, 0)), dict(k=(2 * P, 128, 128 * 9))])
def test_outputs_that_share_memory(change):
    assert _rotate(**change) == ARG


@pytest.mark.parametrize("change", [
    dict(), dict(q=(3 * P, 0, 0)), dict(k=(3 * P, 256, 0)), dict(q_out=(3 * P, 128, 128 * 9)), dict(tokens=1, q=(P, 7, 128), q_out=(P, 0, 128)),
    dict(q_heads=1, q=(P, 128, 3), q_out=(P, 128, 0)), dict(k_heads=1, k=(2 * P, 128, 0), k_out=(2 * P, 128, 0))])
def test_rows_that_do_not(change):
    """Inputs may be one row for all; a stride between one row and none does not count. (Refused for another reason.)"""
    assert _rotate(**change) == SHAPE


def test_strides_against_the_rows_themselves():
    rng = random.Random(1)
    met = 0
    for _ in range(4000):
        tokens, heads, head_dim = rng.randint(1, 6), rng.randint(1, 6), rng.choice([2, 5, 16])
        strides = [rng.choice([0, rng.randint(0, 3), rng.randint(0, 5)]) * head_dim + rng.randint(0, head_dim) for _ in range(2)]
        first = sorted(t * strides[0] + h * strides[1] for t in range(tokens) for h in range(heads))
        meets = any(b - a < head_dim for a, b in zip(first, first[1:]))
        met += meets
        s = kv.RotationStruct(P, 1, 2, P, 0, 0, 0, 0, 0.0, None, None)
        q, out = kv.RowsStruct(3 * P, 0, 0, tokens, 0), kv.RowsStruct(P, *strides, tokens, 0)
        got = kv.lib().us_kv_rotate(heads, 0, head_dim, at(q), at(out), None, None, at(s), None)
        assert got == (ARG if meets else SHAPE), (tokens, heads, head_dim, strides)
    assert 1000 < met < 3500


def test_far_strides():
    far = (1 << 63) - 1
    for out, status in (((P, far, 128), SHAPE), ((P, 256, far), SHAPE), ((P, far, far), ARG), ((P, far, far - 127), ARG), ((P, far, far - 128), SHAPE)):
        assert _rotate(q_out=out, q=(3 * P, 256, 128)) == status, out
