"""The choice of blocks where a cache head has more query heads than are laid out together (16), over one and several
chunks of blocks to a workgroup, and where no query head is finite. Bounds are those of test_gpu_kv_more.py, whose cases and oracle these share."""
import math

import pytest

from paper_2608_09291_amd import kv
from test_gpu_kv import DTYPES
from test_gpu_kv_more import _attend_chosen, _choose_case
from test_gpu_spmm import announce, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

# Tables of at most 128 blocks take 64 blocks a chunk, wider ones 128; up to two chunks are one workgroup's.
MANY_HEADS = [  # lens, queries, q heads, cache heads, head_dim
    ([5000, 4096, 70], [1, 2, 1], 17, 1, 64), ([4200], [2], 40, 2, 256), ([8192, 4161], [1, 1], 32, 1, 128),
    ([6000], [1], 71, 1, 80), ([9000, 8193, 300], [1, 1, 1], 34, 2, 128), ([16384], [1], 32, 1, 64),
    ([10000], [3], 71, 1, 13), ([8200], [1], 20, 1, 192), ([8300], [1], 33, 1, 256), ([20000], [1], 20, 1, 64),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,new,H,Hk,D", MANY_HEADS)
def test_choose_with_many_query_heads(torch_cuda, lens, new, H, Hk, D, dtype):
    torch = torch_cuda
    announce(f"kv choose of many heads lens={lens} new={new} {H}/{Hk} D={D} {dtype}")
    p, cache, q, chosen, starts = _choose_case(torch, lens, new, H, Hk, D, 9, 1, 2, dtype)
    if dtype == "bf16":
        _attend_chosen(torch, p, cache, q, chosen, lens, new, starts, dtype)


def test_choose_with_many_query_heads_and_rows(torch_cuda):
    """So many rows that a workgroup takes several chunks of one with more than two."""
    announce("kv choose of many heads and rows")
    _choose_case(torch_cuda, [17000], [700], 17, 1, 64, 5, 0, 1, "f16")


def test_choose_with_many_query_heads_and_blocks_that_are_not_there(torch_cuda):
    announce("kv choose of many heads over holes")
    _choose_case(torch_cuda, [7000], [2], 24, 1, 64, 6, 1, 1, "f32", holes=[(0, 0), (0, 64), (0, 90), (0, 109)])


@pytest.mark.parametrize("blocks,top", [(1, 1), (20, 4), (140, 9), (5000, 70)])
def test_choose_without_a_finite_query(torch_cuda, blocks, top):
    """Scores are -infinity, of blocks of scale 0 as well, and the first blocks are taken."""
    torch = torch_cuda
    announce(f"kv choose without a finite query blocks={blocks}")
    cache = kv.new_cache(blocks, 2, 64)
    cache.k_scale[::3, 0] = 0.5                             # (zeros are what a block of zeros has)
    cache.k_scale[1:, 1] = 0.25
    i32 = dict(dtype=torch.int32, device="cuda")
    table, lens = torch.arange(blocks, **i32)[None], torch.tensor([64 * blocks], **i32)
    for bad in (math.nan, math.inf, -math.inf):
        q = torch.randn((1, 6, 64), device="cuda")
        q[0, :, 5] = bad
        scores, chosen = torch.zeros((1, 2, blocks), device="cuda"), torch.zeros((1, 2, top), **i32)
        kv.choose(cache, kv.new_summary(cache), table, lens, q, scores, chosen, sinks=0, recent=0, ws=kv.choose_workspace(cache, table, chosen))
        assert (scores == -math.inf).all()
        assert chosen.tolist() == [[list(range(top))] * 2]
