"""Rotations with weights of queries and of keys. Bounds are those of test_gpu_kv_more.py."""
import numpy as np
import pytest

from oracle import kv as ref
from paper_2608_09291_amd import kv
from test_gpu_kv import DTYPES, _torch_dtype
from test_gpu_kv_more import _rotate_bound
from test_gpu_spmm import announce, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

WEIGHTS = [  # tokens, q heads, k heads, head_dim, pairs, adjacent: passes of a token's rows, one with both, and parts of them
    (1, 32, 32, 128, 64, False), (1, 70, 9, 128, 64, True), (5, 8, 2, 128, 64, True), (3, 3, 1, 80, 40, False), (2050, 37, 30, 64, 32, False),
    (4100, 64, 8, 96, 20, True), (9, 2, 1, 255, 127, False), (17, 2, 2, 13, 6, True), (1200, 40, 9, 256, 128, False), (300, 1, 1, 64, 0, False),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("aligned", [False, True])
@pytest.mark.parametrize("which", ["both", "keys", "queries"])
@pytest.mark.parametrize("T,H,Hk,D,pairs,adjacent", WEIGHTS)
def test_rotate_weights(torch_cuda, T, H, Hk, D, pairs, adjacent, which, aligned, dtype):
    torch = torch_cuda
    announce(f"kv rotate weights of {which} T={T} {H}+{Hk} D={D} pairs={pairs} adjacent={adjacent} aligned={aligned} {dtype}")
    rng = np.random.default_rng(T + H + D)
    pad, dt = 0 if aligned else 3, _torch_dtype(torch, dtype)
    wide = torch.from_numpy(rng.normal(0, 1.5, size=(T, H + Hk, D + pad)).astype(np.float32)).to(dt).cuda()
    rows = [wide[:, :H, pad // 2:pad // 2 + D], wide[:, H:, pad // 2:pad // 2 + D]]
    freq = positions = None
    if pairs:
        freq = rng.uniform(0, 1, size=(1, pairs)).astype(np.float32) ** 4
        positions = rng.integers(0, 5000, size=(1, T)).astype(np.int32)
    weights = [rng.uniform(a, a + 1, size=D).astype(np.float32) for a in (0.5, 2.0)]
    if which != "both":
        weights[which == "queries"] = None
    qw, kw = (None if w is None else torch.from_numpy(w).cuda() for w in weights)
    out = [torch.empty((T, n, D), dtype=dt, device="cuda") for n in (H, Hk)]
    kv.rotate(*rows, None if freq is None else torch.from_numpy(freq).cuda(), None if freq is None else torch.from_numpy(positions).cuda(),
              q_out=out[0], k_out=out[1], adjacent=adjacent, norm=True, q_weight=qw, k_weight=kw, eps=1e-5)
    torch.cuda.synchronize()
    # (all rows of a few tokens, the first and the last among them: the oracle turns them one by one)
    some = np.unique(np.linspace(0, T - 1, 40).astype(int))
    pos = None if freq is None else positions[:, some]
    for x, y, w in zip(rows, out, weights):
        x, y = (z[torch.from_numpy(some).cuda()].double().cpu().numpy() for z in (x, y))
        want = ref.rotate(x, freq, pos, 0, adjacent, w, 1e-5)
        over = np.abs(y - want) - _rotate_bound(x, want, freq, pos, 0, adjacent, 1e-5, dtype, w)
        assert (over <= 0).all(), (np.unravel_index(over.argmax(), over.shape), over.max())


def test_rotate_a_head_that_is_there_once(torch_cuda):
    """One key head for all: turned into an output of its own, not in place."""
    torch = torch_cuda
    announce("kv rotate a broadcast head")
    one, freq, pos = torch.randn((20, 1, 64), device="cuda"), torch.rand(32, device="cuda"), torch.arange(20, dtype=torch.int32, device="cuda")
    q, k, before = torch.randn((20, 8, 64), device="cuda"), one.expand(20, 4, 64), one.clone()
    with pytest.raises((RuntimeError, ValueError)):
        kv.rotate(q.clone(), k, freq, pos)
    out, alone = torch.empty((20, 4, 64), device="cuda"), torch.empty_like(one)
    kv.rotate(q, k, freq, pos, k_out=out)
    kv.rotate(one, None, freq, pos, q_out=alone)
    torch.cuda.synchronize()
    assert torch.equal(one, before) and torch.equal(out, alone.expand(20, 4, 64))


def test_rotate_as_many_rows_as_there_can_be(torch_cuda):
    """2^31 - 1 rows of one value, whose number and that of a workgroup's rows add up to more than 32 bits hold."""
    torch = torch_cuda
    announce("kv rotate 2^31 - 1 rows")
    x = torch.full((2 ** 31 - 1, 1, 1), 2.0, dtype=torch.float16, device="cuda")
    x[-1], x[12345] = -3.0, 0.5
    kv.rotate(x, None, None, None, norm=True, q_weight=torch.tensor([4.0], device="cuda"))
    torch.cuda.synchronize()
    assert x[-1].item() == -4.0                             # (1 - eps / (2 x^2) times 4, to half a step of 2^-9)
    assert (x[:-1] == 4.0).all()
