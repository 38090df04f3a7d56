#!/usr/bin/env python3
"""Several samples of one prompt, decoded over a cache that they share.

    python examples/kv_samples.py [--samples S] [--prompt P] [--tokens T] [--blocks K]

One attention layer with the library's own operators. The prompt's rows come out of
the QKV projection of pruned INT4 weights (us_spmm), are rotated by their positions
(us_kv_rotate) and go into the 8-bit cache (us_kv_append) once; us_kv_fork then
makes S sequences of it, which share its full blocks. Every step projects and
rotates a token of each sample, asks for its block (us_kv_fork again, which now and
then lets a sample go on from another), and attends to the common blocks once for
all of them (us_kv_attend_shared). At the end the last tokens attend to the K blocks
alone whose keys can matter most to them (us_kv_summarise, us_kv_choose,
us_kv_attend_chosen). Weights and inputs are synthetic. Prints how far the last
step is from us_kv_attend over the same cache, and what the blocks left out change.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_09291_amd import binding, kv, synth  # noqa: E402

HIDDEN, HEADS, KV_HEADS, HEAD_DIM = 512, 8, 2, 64
ROWS = (HEADS + 2 * KV_HEADS) * HEAD_DIM


def pack_int4(x):
    """(N, K) whole numbers in [-8, 7] -> packed INT4, on the GPU."""
    q = x.to(torch.int16) & 15
    return (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)


class Layer:
    """The layer's weights, a pool of cache blocks with their references, and the samples' tables."""

    def __init__(self, samples, most_tokens, seed=0):
        self.qkv = binding.to_device(binding.encode(synth.random_problem(ROWS, HIDDEN, 1, 0.5, seed)[0]))
        self.scale = torch.full((ROWS,), 0.02, device="cuda")
        width = most_tokens // kv.BLOCK + 2
        n_blocks = width + 2 * samples * 4
        ints = dict(dtype=torch.int32, device="cuda")
        self.cache = kv.new_cache(n_blocks, KV_HEADS, HEAD_DIM)
        self.summary = kv.new_summary(self.cache)
        self.refs, self.missing = torch.zeros(n_blocks, **ints), torch.zeros(1, **ints)
        self.tables = [torch.full((samples, width), -1, **ints) for _ in range(2)]
        self.lens = [torch.zeros(samples, **ints) for _ in range(2)]
        self.ws = kv.fork_workspace(self.cache, *self.tables)
        self.freq = (10000.0 ** (-torch.arange(HEAD_DIM // 2, device="cuda") / (HEAD_DIM // 2))).float()

    def project(self, x, positions, offset=0):
        """Rows of x (N, HIDDEN) whole numbers: rotated queries and keys, and values, (N, heads, HEAD_DIM) each."""
        n = x.shape[0]
        y, yi = torch.empty((n, ROWS), device="cuda"), torch.empty((n, ROWS), dtype=torch.int32, device="cuda")
        binding.spmm(self.qkv, pack_int4(x), n, yi, self.scale, y)
        heads = y.view(n, HEADS + 2 * KV_HEADS, HEAD_DIM)
        q, k, v = heads[:, :HEADS], heads[:, HEADS:HEADS + KV_HEADS], heads[:, HEADS + KV_HEADS:]
        kv.rotate(q, k, self.freq, positions, offset=offset)
        return q, k, v

    def fork(self, parents, room):
        """The samples go on from `parents`, with blocks for `room` more tokens of each."""
        kv.fork(self.cache, self.refs, self.tables[0], self.lens[0], parents, self.tables[1], self.lens[1], self.missing, room=room,
                ws=self.ws)
        self.tables.reverse()
        self.lens.reverse()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--samples", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--tokens", type=int, default=100)
    ap.add_argument("--blocks", type=int, default=6)
    a = ap.parse_args(argv)
    S, P = a.samples, a.prompt
    layer = Layer(S, P + a.tokens)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ints = dict(dtype=torch.int32, device="cuda")
    # The prompt: the first sample alone, in pieces as wide as a projection takes.
    first = torch.full((S,), -1, **ints)
    first[0] = 0
    layer.fork(first, P * (first >= 0).int())
    for at in range(0, P, binding.N_LIMIT):
        n = min(binding.N_LIMIT, P - at)
        x = torch.randint(-8, 8, (n, HIDDEN), generator=g, device="cuda")
        _, k, v = layer.project(x, torch.arange(at, at + n, **ints))
        layer.lens[0][0] += n
        starts = torch.tensor([0] + [n] * S, **ints)
        kv.append(layer.cache, layer.tables[0], layer.lens[0], k, v, starts=starts, max_new=n)
        kv.summarise(layer.cache, layer.tables[0], layer.lens[0], layer.summary, starts=starts, max_new=n)
    # One group of all samples, which have the prompt's full blocks in common.
    groups, shared = torch.tensor([0, S], **ints), torch.tensor([P // kv.BLOCK], **ints)
    parents, room = torch.zeros(S, **ints), torch.ones(S, **ints)
    q0 = torch.empty((S, HEADS, HEAD_DIM), device="cuda")
    ws = kv.attend_shared_workspace(layer.cache, q0, layer.tables[0], groups)
    out = torch.empty_like(q0)
    for t in range(a.tokens):
        layer.fork(parents, room)
        x = torch.randint(-8, 8, (S, HIDDEN), generator=g, device="cuda")
        layer.lens[0] += 1
        q, k, v = layer.project(x, layer.lens[0], offset=-1)
        kv.append(layer.cache, layer.tables[0], layer.lens[0], k, v)
        kv.summarise(layer.cache, layer.tables[0], layer.lens[0], layer.summary)
        kv.attend_shared(layer.cache, layer.tables[0], layer.lens[0], q, out, groups, shared, ws=ws)
        # each goes on from itself; at every 16th token the last two from the first
        parents = torch.arange(S, **ints)
        if t % 16 == 15:
            parents[-2:] = 0
    if layer.missing.item():
        raise AssertionError("too few blocks")
    want = torch.empty_like(out)
    kv.attend(layer.cache, layer.tables[0], layer.lens[0], q, want, ws=kv.attend_workspace(layer.cache, q, layer.tables[0]))
    blocks = layer.tables[0].shape[1]
    scores, chosen = torch.empty((S, KV_HEADS, blocks), device="cuda"), torch.empty((S, KV_HEADS, a.blocks), **ints)
    kv.choose(layer.cache, layer.summary, layer.tables[0], layer.lens[0], q, scores, chosen, sinks=1, recent=2,
              ws=kv.choose_workspace(layer.cache, layer.tables[0], chosen))
    part = torch.empty_like(out)
    kv.attend_chosen(layer.cache, layer.tables[0], layer.lens[0], q, part, chosen,
                     ws=kv.attend_chosen_workspace(layer.cache, q, layer.tables[0], chosen))
    off, less = ((x.double() - want.double()).norm().item() / want.double().norm().item() for x in (out, part))
    used = int((layer.refs > 0).sum())
    print(f"{S} samples of {P} + {a.tokens} tokens in {used} blocks: shared attention off by {off:.1e} of its norm, "
          f"{a.blocks} blocks of {blocks} instead of all by {less:.1e}", flush=True)
    return off, less, used


if __name__ == "__main__":
    main()
