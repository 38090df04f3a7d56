"""Shared attention where the queries' own table is out of order: no part of another row is looked at, and groups that
are in order keep their results. Bounds are those of test_gpu_kv.py."""
import math

import numpy as np
import pytest

from paper_2608_09291_amd import kv
from test_gpu_kv import _check
from test_gpu_kv_more import Groups
from test_gpu_spmm import announce, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("queries", [4, 150])               # joined by the workgroups that leave parts, and by a launch of its own
def test_attend_shared_with_queries_out_of_order(torch_cuda, queries):
    torch = torch_cuda
    announce(f"kv shared queries out of order {queries}")
    rng = np.random.default_rng(queries)
    n, H, Hk, D = queries, 4, 2, 64
    p = Groups(torch, rng, [2, 2], [3, 2], [n, n, n + 9, n], Hk, D)
    cache, groups = p.cache(), p.dev([0, 2, 4])
    q = torch.from_numpy(rng.normal(0, 1.5, size=(4 * n, H, D)).astype(np.float32)).cuda()
    args = dict(max_q=n, max_group=2, max_shared=3)
    ws = kv.attend_shared_workspace(cache, q, p.dev(p.blocks), groups, starts=p.dev([i * n for i in range(5)]), **args)
    for first in (2 * n, 2 ** 31 - 1, -2 ** 31):            # of the first group's first sequence, which has no rows then
        starts = p.dev([first, n, 2 * n, 3 * n, 4 * n])
        out = torch.full_like(q, math.nan)
        kv.attend_shared(cache, p.dev(p.blocks), p.dev(p.lens_), q, out, groups, p.dev([3, 2]), starts=starts, ws=ws, **args)
        torch.cuda.synchronize()
        assert torch.isfinite(out[n:]).all()
        _check(torch, p, p.lens_, [0, 0, n, n], q[2 * n:], out[2 * n:], "f32")
        assert not ws[:16384].any()                         # the tickets
