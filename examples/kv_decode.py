#!/usr/bin/env python3
"""One attention layer, decoded with the library's own operators.

    python examples/kv_decode.py [--batch B] [--tokens T] [--budget N]

Per token and sequence: the QKV projection of pruned INT4 weights (us_spmm with
its dequant epilogue, N = batch), the new keys and values into the 8-bit cache
(us_kv_append), attention over it that also adds up each token's weight
(us_kv_attend), the activations quantised to INT4 again, and the output
projection (us_spmm). When a sequence's cache has reached the budget, half of it
is evicted: the recent tokens stay, and those that were attended to most
(us_kv_evict). Weights and inputs are synthetic. Prints one line per eviction and,
at the end, how far the last step's attention is from the same attention in
float64 over the cached values (us_kv_read).
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_09291_amd import binding, kv, synth  # noqa: E402

HIDDEN, HEADS, KV_HEADS, HEAD_DIM = 512, 8, 2, 64


def pack_int4(x, step):
    """(N, K) values -> packed INT4 of x / step, on the GPU."""
    q = torch.clamp(torch.round(x / step), -8, 7).to(torch.int16) & 15
    return (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)


class Layer:
    """The layer's weights, a pool of cache blocks, and what the sequences hold of it."""

    def __init__(self, batch, budget, seed=0):
        rows = (HEADS + 2 * KV_HEADS) * HEAD_DIM
        self.batch, self.budget = batch, budget
        self.qkv = binding.to_device(binding.encode(synth.random_problem(rows, HIDDEN, 1, 0.5, seed)[0]))
        self.proj = binding.to_device(binding.encode(synth.random_problem(HIDDEN, HEADS * HEAD_DIM, 1, 0.5, seed + 1)[0]))
        # dequant: weight scale times activation step, one per output channel
        self.qkv_scale = torch.full((rows,), 0.02, device="cuda")
        self.proj_scale = torch.full((HIDDEN,), 0.02, device="cuda")
        # Twice the blocks a full cache takes: evictions move to the half that is free.
        width = (budget + kv.BLOCK - 1) // kv.BLOCK
        self.cache = kv.new_cache(2 * batch * width, KV_HEADS, HEAD_DIM)
        halves = torch.arange(2 * batch * width, dtype=torch.int32, device="cuda").view(2, batch, width)
        self.tables = [halves[0].contiguous(), halves[1].contiguous()]
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.weights = torch.zeros((batch, KV_HEADS, width * kv.BLOCK), device="cuda")
        self.index = torch.empty((batch, KV_HEADS, budget // 2), dtype=torch.int32, device="cuda")
        self.length = 0                                    # of every sequence, known here without asking the GPU
        y = torch.empty((batch, rows), device="cuda")
        self.y, self.yi = y, torch.empty((batch, rows), dtype=torch.int32, device="cuda")
        parts = y.view(batch, HEADS + 2 * KV_HEADS, HEAD_DIM)
        self.q, self.k, self.v = parts[:, :HEADS], parts[:, HEADS:HEADS + KV_HEADS], parts[:, HEADS + KV_HEADS:]
        self.attended = torch.empty((batch, HEADS, HEAD_DIM), device="cuda")
        self.out = torch.empty((batch, HIDDEN), device="cuda")
        self.outi = torch.empty((batch, HIDDEN), dtype=torch.int32, device="cuda")
        self.ws = kv.attend_workspace(self.cache, self.q, self.tables[0], weights=self.weights)

    def step(self, x):
        """One token of every sequence: x (batch, HIDDEN) packed INT4 -> (batch, HIDDEN)."""
        binding.spmm(self.qkv, x, self.batch, self.yi, self.qkv_scale, self.y)
        self.lens.add_(1)
        self.length += 1
        kv.append(self.cache, self.tables[0], self.lens, self.k, self.v)
        kv.attend(self.cache, self.tables[0], self.lens, self.q, self.attended, weights=self.weights, ws=self.ws)
        binding.spmm(self.proj, pack_int4(self.attended.view(self.batch, -1), 0.25), self.batch, self.outi, self.proj_scale,
                     self.out)
        return self.out

    def evict(self):
        """Half of the budget stays, a quarter of that for being recent."""
        keep = self.budget // 2
        lens, weights = torch.empty_like(self.lens), torch.empty_like(self.weights)
        kv.evict(self.cache, self.tables[0], self.lens, self.weights, keep, keep // 4, self.tables[1], lens, weights, self.index)
        self.tables.reverse()
        self.lens, self.weights, self.length = lens, weights, min(self.length, keep)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=700)
    ap.add_argument("--budget", type=int, default=256)
    a = ap.parse_args(argv)
    layer = Layer(a.batch, a.budget)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    evictions = 0
    for t in range(a.tokens):
        if layer.length == a.budget:
            layer.evict()
            evictions += 1
            print(f"token {t}: {a.budget} cached tokens -> {layer.length}", flush=True)
        x = torch.randint(-8, 8, (a.batch, HIDDEN), generator=g, device="cuda").float()
        out = layer.step(pack_int4(x, 1.0))
    if not torch.isfinite(out).all():
        raise AssertionError("the layer's output is not finite")
    # The last step's attention again, over the dense values of the cache.
    n = layer.length
    dense = [torch.empty((a.batch * n, KV_HEADS, HEAD_DIM), device="cuda") for _ in range(2)]
    starts = torch.arange(0, a.batch * n + 1, n, dtype=torch.int32, device="cuda")
    kv.read(layer.cache, layer.tables[0], layer.lens, *dense, starts=starts, max_new=n)
    k, v = (d.view(a.batch, n, KV_HEADS, HEAD_DIM).double().repeat_interleave(HEADS // KV_HEADS, dim=2) for d in dense)
    s = (layer.q.double()[:, None] * k).sum(-1) / math.sqrt(HEAD_DIM)
    want = (torch.softmax(s, dim=1)[..., None] * v).sum(1)
    off = ((layer.attended.double() - want).norm() / want.norm()).item()
    print(f"{a.tokens} tokens, {evictions} evictions, attention off by {off:.1e} of its norm", flush=True)
    return off, evictions


if __name__ == "__main__":
    main()
