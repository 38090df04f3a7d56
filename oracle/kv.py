"""The 8-bit key/value cache on the CPU, from the definitions in include/us_kv.h.

Pools are numpy arrays: codes uint8 (n_blocks, heads, 64 * row), scales float32
(n_blocks, heads). The stored numbers are defined in float32 and computed so
here (numpy rounds every operation once); attention is computed in float64.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 64
F32 = np.float32


def row_of(head_dim: int) -> int:
    return next(r for r in (64, 96, 128, 192, 256) if head_dim <= r)


def key_byte(t: int, d: int) -> int:
    return 2048 * (d // 32) + 1024 * (t // 32) + 64 * (t % 16) + 16 * ((d // 8) % 4) + 8 * ((t // 16) % 2) + d % 8


def value_byte(t: int, d: int) -> int:
    return 64 * d + 16 * ((t // 4) % 4) + 4 * (t // 16) + t % 4


def places(head_dim: int, keys: bool) -> np.ndarray:
    """(64, head_dim): the byte of every (token, value) of a block."""
    f = key_byte if keys else value_byte
    return np.array([[f(t, d) for d in range(head_dim)] for t in range(BLOCK)])


def rows_of(b, lens, starts):
    """First row, number of rows and first position of sequence b's new tokens."""
    r0, r1 = (b, b + 1) if starts is None else (starts[b], starts[b + 1])
    return r0, r1 - r0, lens[b] - (r1 - r0)


def append(codes, scales, head_dim, keys, blocks, lens, starts, x):
    """Quantise rows x (tokens, heads, head_dim; float32) into codes and scales, in place."""
    at = places(head_dim, keys)
    for b in range(len(lens)):
        r0, n, p0 = rows_of(b, lens, starts)
        for first in range(max(p0, 0) // BLOCK, -(-lens[b] // BLOCK)):
            t0, t1 = max(p0 - first * BLOCK, 0), min(lens[b] - first * BLOCK, BLOCK)
            if t1 <= t0 or n == 0:
                continue
            blk = blocks[b][first]
            for h in range(codes.shape[1]):
                new = x[r0 + first * BLOCK + t0 - p0:r0 + first * BLOCK + t1 - p0, h].astype(F32)
                fin = np.abs(new[np.isfinite(new)])
                amax = F32(fin.max()) if fin.size else F32(0)
                s1 = scales[blk, h] if t0 > 0 else F32(0)
                s2 = max(s1, F32(amax / F32(127)))
                if t0 > 0 and s2 != s1:
                    c = codes[blk, h][at[:t0]].astype(F32) - F32(128)
                    codes[blk, h][at[:t0]] = (np.rint(c * F32(s1 / s2)) + F32(128)).astype(np.uint8)
                with np.errstate(all="ignore"):
                    q = np.rint(new / s2) if s2 > 0 else np.where(np.isinf(new), new, F32(0))
                q = np.clip(np.nan_to_num(q, nan=0.0), -127, 127)
                codes[blk, h][at[t0:t1]] = (q + 128).astype(np.uint8)
                scales[blk, h] = s2


def tokens(codes, scales, head_dim, keys, blocks, n, h):
    """Codes and scales (float64) of a sequence's first n tokens of head h: (n, head_dim), (n,)."""
    at = places(head_dim, keys)
    ids = [blocks[i] for i in range(-(-n // BLOCK))]
    c = np.concatenate([codes[i, h][at].astype(np.float64) - 128 for i in ids] or [np.zeros((0, head_dim))])[:n]
    s = np.concatenate([np.full(BLOCK, float(scales[i, h])) for i in ids] or [np.zeros(0)])[:n]
    return c, s


def visible(i, n, length, causal, window):
    """First and end key of query i of n."""
    if not causal:
        return 0, length
    at = length - n + i
    return (max(at - window + 1, 0) if window else 0), max(at + 1, 0)


def attend(k, ks, v, vs, head_dim, blocks, lens, starts, q, scale=None, causal=True, window=0):
    """float64 attention of rows q (tokens, heads, head_dim).

    Returns (out, out_abs, weights, reach): out_abs = sum_j p_j |v_j| and reach = the largest
    scale * sum_d |q_d k_jd| of a row, which bound rounding errors; weights a list over the
    sequences of (cache heads, len)."""
    T, H, D = q.shape
    Hk = k.shape[1]
    G = H // Hk
    scale = 1 / math.sqrt(D) if scale is None else scale
    q = q.astype(np.float64)
    out, out_abs, reach = np.zeros((T, H, D)), np.zeros((T, H, D)), np.zeros((T, H))
    weights = [np.zeros((Hk, n)) for n in lens]
    for b in range(len(lens)):
        r0, n, _ = rows_of(b, lens, starts)
        for hk in range(Hk):
            kc, kscale = tokens(k, ks, D, True, blocks[b], lens[b], hk)
            vc, vscale = tokens(v, vs, D, False, blocks[b], lens[b], hk)
            key, val = kc * kscale[:, None], vc * vscale[:, None]
            for i in range(n):
                lo, hi = visible(i, n, lens[b], causal, window)
                if hi <= lo:
                    continue
                for h in range(hk * G, hk * G + G):
                    x = scale * (key[lo:hi] @ q[r0 + i, h])
                    reach[r0 + i, h] = (scale * (np.abs(key[lo:hi]) @ np.abs(q[r0 + i, h]))).max()
                    p = np.exp(x - x.max())
                    p /= p.sum()
                    weights[b][hk, lo:hi] += p
                    out[r0 + i, h] = p @ val[lo:hi]
                    out_abs[r0 + i, h] = p @ np.abs(val[lo:hi])
    return out, out_abs, weights, reach


def kept(weights, length, keep, recent):
    """The positions that stay, ascending, for one row of weights."""
    stay = min(length, keep)
    late = min(recent, stay)
    m = length - late
    w = [(-math.inf, 1) if math.isnan(x) else (float(x), 0) for x in weights[:m]]
    order = sorted(range(m), key=lambda j: (w[j][1], -w[j][0], j))   # a NaN after every number
    return sorted(order[:stay - late]) + list(range(m, length))


def evict(codes, scales, head_dim, keys, blocks, positions, to_blocks, h):
    """Move the tokens at `positions` of one sequence's head h to to_blocks, in place."""
    at = places(head_dim, keys)
    got = [(codes[blocks[p // BLOCK], h][at[p % BLOCK]].astype(F32) - F32(128), scales[blocks[p // BLOCK], h])
           for p in positions]
    for first in range(0, len(got), BLOCK):
        part = got[first:first + BLOCK]
        s2 = max(s for _, s in part)
        blk = to_blocks[first // BLOCK]
        for t, (c, s) in enumerate(part):
            r = F32(s / s2) if s2 > 0 else F32(0)
            codes[blk, h][at[t]] = (np.rint(c * r) + F32(128)).astype(np.uint8)
        scales[blk, h] = s2


# --- rotations, forks, and blocks that a query chooses ------------------------------

def rotate(x, freq=None, positions=None, offset=0, adjacent=False, weight=None, eps=None):
    """float64 norms (with eps) and rotations of rows x (tokens, heads, head_dim); freq (axes, pairs), positions (axes, tokens)."""
    x = x.astype(np.float64).copy()
    if eps is not None:
        x /= np.sqrt((x * x).mean(-1, keepdims=True) + float(F32(eps)))
        if weight is not None:
            x *= weight.astype(np.float64)
    if freq is None:
        return x
    pairs = freq.shape[1]
    for t in range(x.shape[0]):
        for i in range(pairs):
            a = math.fsum((int(positions[j][t]) + offset) * float(freq[j][i]) for j in range(freq.shape[0]))
            one, two = (2 * i, 2 * i + 1) if adjacent else (i, pairs + i)
            n1, n2 = x[t, :, one].copy(), x[t, :, two].copy()
            x[t, :, one] = n1 * math.cos(a) - n2 * math.sin(a)
            x[t, :, two] = n2 * math.cos(a) + n1 * math.sin(a)
    return x


def fork(refs, blocks, lens, parents, room, to_width):
    """A fork of the sequences in `blocks` (lists of numbers); parents a list, room one or None.

    Returns (to_blocks, to_lens, refs, copies, missing): copies a list of (from, to) blocks; with missing > 0
    empty sequences and refs as they were."""
    n_blocks, batch, width = len(refs), len(blocks), len(blocks[0])
    free = [i for i in range(n_blocks) if refs[i] == 0]
    taken = set()
    new, copies, want, to_lens = [], [], 0, []
    for b, p in enumerate(parents):
        p = p if 0 <= p < batch else None
        row = [-1] * to_width
        length = min(max(lens[p], 0), width * BLOCK) if p is not None else 0
        more = 0 if room is None else max(room[b], 0)
        need = min(-(-(length + more) // BLOCK), to_width)
        heir = p is not None and p not in taken
        taken.add(p)
        for i in range(need):
            old = blocks[p][i] if p is not None and i < width and 0 <= blocks[p][i] < n_blocks else -1
            started = i * BLOCK < length
            if i < length // BLOCK or (heir and old >= 0 and refs[old] == 1):
                row[i] = old
            elif old >= 0 or not started:
                got = free[want] if want < len(free) else None
                want += 1
                row[i] = got
                if started:
                    copies.append((old, got))
        new.append(row)
        to_lens.append(length)
    if want > len(free):
        return [[-1] * to_width for _ in parents], [0] * len(parents), list(refs), [], want - len(free)
    after = list(refs)
    for row in blocks:
        for x in row:
            if 0 <= x < n_blocks:
                after[x] -= 1
    for row in new:
        for x in row:
            if x >= 0:
                after[x] += 1
    return new, to_lens, after, copies, 0


def extremes(codes, head_dim, block, h, tokens_there):
    """Smallest and largest byte of each value over the first tokens of a key block: (2, head_dim)."""
    c = codes[block, h][places(head_dim, True)[:tokens_there]]
    return np.stack((c.min(0), c.max(0)))


def score(summary, scale, q):
    """float32 score of a block for the query heads q (heads, head_dim) of its cache head, rounded once."""
    lo, hi = summary.astype(np.float64) - 128
    q = q.astype(np.float64)
    ok = np.isfinite(q).all(-1)
    if not ok.any():
        return F32(-np.inf)
    q = q[ok]
    return F32((np.maximum(q, 0) @ hi + np.minimum(q, 0) @ lo).max() * float(scale))


def choose(scores, there, top, sinks, recent):
    """Places of the blocks to take, ascending: `there` says which of the scored blocks exist."""
    n = len(scores)

    def rank(i):
        if i < sinks or i >= n - recent:
            return (0, 0.0, i)
        return (2, 0.0, i) if math.isnan(scores[i]) else (1, -float(scores[i]), i)

    return sorted(sorted((i for i in range(n) if there[i]), key=rank)[:top])


def attend_chosen(k, ks, v, vs, head_dim, blocks, at, places_, q, h, scale=None):
    """float64 attention of one query (head_dim) at position `at` over the blocks at places_ of its sequence.

    Returns (out, out_abs, reach) as attend does."""
    scale = 1 / math.sqrt(head_dim) if scale is None else scale
    q = q.astype(np.float64)
    key, val = [], []
    for i in places_:
        n = min(BLOCK, at + 1 - i * BLOCK) if i >= 0 else 0
        if n <= 0 or i >= len(blocks) or not 0 <= blocks[i] < len(k):
            continue
        kc, kscale = tokens(k, ks, head_dim, True, [blocks[i]], n, h)
        vc, vscale = tokens(v, vs, head_dim, False, [blocks[i]], n, h)
        key.append(kc * kscale[:, None])
        val.append(vc * vscale[:, None])
    if not key:
        return np.zeros(head_dim), np.zeros(head_dim), 0.0
    key, val = np.concatenate(key), np.concatenate(val)
    x = scale * (key @ q)
    p = np.exp(x - x.max())
    p /= p.sum()
    return p @ val, p @ np.abs(val), (scale * (np.abs(key) @ np.abs(q))).max()
