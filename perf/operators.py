"""Measured cases of the 8-bit key/value cache: append, read, attention and eviction.

The cache holds keys and values in 8 bits (byte = code + 128, code in [-127, 127]) with one
float32 scale for each block of 64 tokens and head. Four operators, each through the public
binding where ``own`` is true and in elementary torch operations in 32 bits otherwise:

* ``append``  quantises new tokens into the blocks of their sequences (a started block whose
  scale grows has its older tokens requantised) and reads the touched blocks back;
* ``read``    the last tokens of every sequence as dense values, as for a move to another machine;
* ``attend``  attention of new queries over the cache: single tokens, chunks and whole prompts,
  grouped heads, causal, windowed or cross, optionally adding each cached token's weight up;
* ``evict``   keeps the recent tokens and those of largest accumulated weight, per head, in new
  blocks, and reads them back.

Sizes are those of the decoder layers whose projections the library multiplies (hidden 4096,
5120 and 8192; 128 values a head) and generic ones around them.
"""
import math
import random

import torch

own = False

BLOCK = 64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _append(name, B, Hkv, D, past, new_lo, new_hi, dtype):
    return {"name": name, "kind": "append", "B": B, "Hkv": Hkv, "D": D, "past": past, "new_lo": new_lo,
            "new_hi": new_hi, "dtype": dtype}


def _read(name, B, Hkv, D, len_lo, len_hi, dtype):
    return {"name": name, "kind": "read", "B": B, "Hkv": Hkv, "D": D, "len_lo": len_lo, "len_hi": len_hi,
            "dtype": dtype}


def _attend(name, B, H, Hkv, D, len_lo, len_hi, q_lo, q_hi, dtype, causal=True, window=0, weights=False):
    return {"name": name, "kind": "attend", "B": B, "H": H, "Hkv": Hkv, "D": D, "len_lo": len_lo,
            "len_hi": len_hi, "q_lo": q_lo, "q_hi": q_hi, "dtype": dtype, "causal": causal, "window": window,
            "weights": weights}


def _evict(name, B, Hkv, D, len_lo, len_hi, keep, recent):
    return {"name": name, "kind": "evict", "B": B, "Hkv": Hkv, "D": D, "len_lo": len_lo, "len_hi": len_hi,
            "keep": keep, "recent": recent}


def listed():
    return [
        # One decode step of 32 sequences stores its new token, grouped heads (8 of 128).
        _append("append_step_b32", 32, 8, 128, 1001, 1, 1, "bf16"),
        # Ragged prompts after a cached prefix that ends inside a block, straight
        # from the float32 output of a QKV projection (hidden 4096, 32 heads).
        _append("append_prompt_b4", 4, 32, 128, 37, 700, 4096, "f32"),
        # A preempted sequence leaves the GPU.
        _read("read_1k", 1, 8, 128, 1021, 1021, "bf16"),
        # A batch of ragged sequences does, 40 heads of 128 (hidden 5120).
        _read("read_b8", 8, 40, 128, 500, 4096, "bf16"),
        # The smallest decode step: one user, a short chat, float32 from the
        # projection's dequant epilogue, 32 heads of 128. Latency counts.
        _attend("decode_b1_200", 1, 32, 32, 128, 200, 200, 1, 1, "f32"),
        # A serving batch of ragged lengths, grouped heads (32 over 8).
        _attend("decode_b64_gqa", 64, 32, 8, 128, 300, 8192, 1, 1, "bf16"),
        # One very long context, 64 heads over 8 (hidden 8192).
        _attend("decode_128k", 1, 64, 8, 128, 131071, 131071, 1, 1, "f16"),
        # Decode that tracks the weight of cached tokens for eviction, 40 heads (hidden 5120).
        _attend("decode_weights_b16", 16, 40, 40, 128, 1500, 2048, 1, 1, "bf16", weights=True),
        # A whole prompt, causal, 32 heads (hidden 4096): the largest case.
        _attend("prompt_8k", 1, 32, 32, 128, 8192, 8192, 8192, 8192, "bf16"),
        # Chunked prefill: ragged chunks of up to 512 queries against cached
        # prefixes, grouped heads (64 over 8), tracking weights.
        _attend("chunk_512_weights", 4, 64, 8, 128, 5000, 16000, 200, 512, "f16", weights=True),
        # Eviction of a few short sequences down to 512 tokens.
        _evict("evict_b4_1k", 4, 8, 128, 700, 1100, 512, 128),
        # Eviction of a batch of long sequences to a quarter.
        _evict("evict_b16_16k", 16, 8, 128, 9000, 16384, 4096, 512),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "read", "attend", "attend", "attend", "attend", "evict"])
    D = rng.choice([64, 80, 96, 128, 128, 256])
    dtype = rng.choice(["f32", "bf16", "f16"])
    Hkv = rng.choice([1, 2, 5, 8, 8, 32])
    B = _log_int(rng, 1, 48)
    while True:
        top = _log_int(rng, 40, 60000)
        low = max(1, int(top * rng.uniform(0.1, 1.0)))
        if kind == "append":
            new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 5000)
            c = _append("", B, Hkv, D, _log_int(rng, 1, 3000), max(1, new // 3), new, dtype)
        elif kind == "read":
            c = _read("", B, Hkv, D, low, top, dtype)
        elif kind == "evict":
            keep = max(8, int(top * rng.uniform(0.1, 0.9)))
            c = _evict("", B, Hkv, D, low, top, keep, int(keep * rng.uniform(0.05, 0.5)))
        else:
            G = rng.choice([1, 1, 4, 5, 8])
            q = 1 if rng.random() < 0.5 else _log_int(rng, 2, 4096)
            q = min(q, top)
            causal = rng.random() < 0.85
            c = _attend("", B, G * Hkv, Hkv, D, max(low, q), top, max(1, q // 2), q, dtype, causal=causal,
                        window=_log_int(rng, 16, top) if causal and rng.random() < 0.2 else 0,
                        weights=rng.random() < 0.3)
        del c["name"]
        w = work(c)
        pool = B * Hkv * top * 2 * D if kind != "append" else 0
        pairs = B * c["H"] * c["q_hi"] * top if kind == "attend" else 0
        if w["bytes"] <= 5e8 and w["flops"] <= 3e11 and pool <= 6e8 and pairs <= 1e9:
            return c
        B = max(1, B // 2)


# ---------------------------------------------------------------------------
# Lengths and inputs
# ---------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, the largest first, the others spread over the logarithm."""
    return [hi] + [int(round(lo * (hi / lo) ** ((i * 0.61803398875) % 1.0))) for i in range(1, n)]


def _shape(case):
    """Lengths of the sequences (all their tokens) and the number of new tokens or queries of each."""
    B = case["B"]
    if case["kind"] == "append":
        new = _spread(case["new_lo"], case["new_hi"], B)
        return [case["past"] + 13 * (i % 5) + n for i, n in enumerate(new)], new
    lens = _spread(case["len_lo"], case["len_hi"], B)
    if case["kind"] == "attend":
        return lens, [min(n, q) for n, q in zip(lens, _spread(case["q_lo"], case["q_hi"], B))]
    return lens, lens


def _row(D):
    """Values a head takes in the cache: its width, rounded up to one the cache is laid out for."""
    return 64 if D <= 64 else 96 if D <= 96 else 128 if D <= 128 else 192 if D <= 192 else 256


def _visible(case):
    """(query, key) pairs that are not masked, and keys that some query sees, over all sequences."""
    pairs = keys = 0
    for n, q in zip(*_shape(case)):
        if not case["causal"]:
            pairs, keys = pairs + q * n, keys + n
            continue
        w = case["window"] or n
        p0 = n - q
        full = max(0, n - max(p0, w))                      # queries that see a whole window
        part = q - full
        pairs += full * w + part * p0 + part * (part + 1) // 2
        keys += n - max(0, p0 - w + 1)
    return pairs, keys


def work(case):
    lens, new = _shape(case)
    Hkv, D, B = case["Hkv"], case["D"], case["B"]
    es = 4 if case.get("dtype") == "f32" else 2
    T = sum(new)
    if case["kind"] == "append":
        back = sum(n - (n - t) // BLOCK * BLOCK for n, t in zip(lens, new))
        return {"bytes": 2 * Hkv * D * (T * es + T + back + back * es), "flops": 2 * Hkv * D * T * 2}
    if case["kind"] == "read":
        return {"bytes": 2 * Hkv * D * T * (1 + es), "flops": 2 * Hkv * D * T}
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in lens)
        # weights of all tokens; codes of the kept ones read, written and read back; indices and weights
        return {"bytes": Hkv * (4 * sum(lens) + kept * (2 * D * (3 + 2) + 8)), "flops": 2 * Hkv * D * kept}
    pairs, keys = _visible(case)
    b = 2 * Hkv * keys * D + 2 * T * case["H"] * D * es + 8 * Hkv * keys // BLOCK
    return {"bytes": b + (8 * Hkv * keys if case["weights"] else 0), "flops": 4 * case["H"] * D * pairs}


def _codes(g, shape, spread):
    return torch.randn(shape, generator=g, device=DEV).mul_(spread).round_().clamp_(-127, 127).add_(128).to(torch.uint8)


def _starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    order = random.Random(int(seed))
    lens, new = _shape(case)
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    Dp, kind = _row(D), case["kind"]
    width = (max(lens) + BLOCK - 1) // BLOCK
    used = [(n + BLOCK - 1) // BLOCK for n in lens]
    kept = [min(n, case["keep"]) for n in lens] if kind == "evict" else [0] * B
    more = [(n + BLOCK - 1) // BLOCK for n in kept]
    n_blocks = sum(used) + sum(more) + 1                   # the last one belongs to no sequence
    free = list(range(n_blocks - 1))
    order.shuffle(free)
    table = [[free.pop() for _ in range(u)] + [-1] * (width - u) for u in used]
    s = {"case": case, "ws": None, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV),
         "blocks": torch.tensor(table, dtype=torch.int32, device=DEV), "max_len": max(lens)}
    # Codes as a quantiser leaves them: about four standard deviations in 127 steps, values of about 1.
    s["k"] = _codes(g, (n_blocks, Hkv, BLOCK * Dp), 32.0)
    s["v"] = _codes(g, (n_blocks, Hkv, BLOCK * Dp), 32.0)
    s["ks"] = torch.rand((n_blocks, Hkv), generator=g, device=DEV) * 0.02 + 0.02
    s["vs"] = torch.rand((n_blocks, Hkv), generator=g, device=DEV) * 0.02 + 0.02
    starts = _starts(new)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["T"], s["max_new"] = starts[-1], max(new)
    dt = DTYPES[case.get("dtype", "bf16")]
    if kind == "attend":
        # heads of a fused projection: the rows of q are further apart than its values
        H, T = case["H"], s["T"]
        y = (torch.randn((T, (H + 2 * Hkv) * D), generator=g, device=DEV) * 1.5).to(dt)
        s["q"] = y[:, :H * D].view(T, H, D)
        s["out"] = torch.empty((T, H, D), dtype=dt, device=DEV)
        if case["weights"]:
            s["w"] = torch.rand((B, Hkv, width * BLOCK), generator=g, device=DEV)
    elif kind == "append":
        T = s["T"]
        y = (torch.randn((T, 2 * Hkv * D), generator=g, device=DEV) * 1.2).to(dt)
        s["kn"], s["vn"] = y[:, :Hkv * D].view(T, Hkv, D), y[:, Hkv * D:].view(T, Hkv, D)
        back = [n - (n - t) // BLOCK * BLOCK for n, t in zip(lens, new)]
        _dense(s, back, Hkv, D, dt)
    elif kind == "read":
        _dense(s, lens, Hkv, D, dt)
    else:
        # weights as attention leaves them: a few tokens hold most
        s["w"] = torch.rand((B, Hkv, width * BLOCK), generator=g, device=DEV).pow_(6).mul_(20.0)
        cap = max(more)
        s["to"] = torch.tensor([[free.pop() for _ in range(u)] + [-1] * (cap - u) for u in more],
                               dtype=torch.int32, device=DEV)
        s["to_lens"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        s["to_w"] = torch.zeros((B, Hkv, cap * BLOCK), device=DEV)
        s["index"] = torch.full((B, Hkv, case["keep"]), -1, dtype=torch.int32, device=DEV)
        _dense(s, kept, Hkv, D, dt)
    return s


def _dense(s, counts, Hkv, D, dt):
    """Where the last counts[b] tokens of every sequence are read to."""
    st = _starts(counts)
    s["back"] = torch.tensor(st, dtype=torch.int32, device=DEV)
    s["back_T"], s["back_max"] = st[-1], max(counts)
    s["ko"] = torch.empty((st[-1], Hkv, D), dtype=dt, device=DEV)
    s["vo"] = torch.empty((st[-1], Hkv, D), dtype=dt, device=DEV)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"append": _own_append, "read": _own_read, "attend": _own_attend, "evict": _own_evict}[kind](s)
    return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "evict": _plain_evict}[kind](s)


def _cache(s):
    from paper_2608_09291_amd import kv
    return kv, kv.Cache(s["k"], s["v"], s["ks"], s["vs"], s["case"]["D"])


def _own_append(s):
    kv, cache = _cache(s)
    kv.append(cache, s["blocks"], s["lens"], s["kn"], s["vn"], starts=s["starts"], max_new=s["max_new"])
    kv.read(cache, s["blocks"], s["lens"], s["ko"], s["vo"], starts=s["back"], max_new=s["back_max"])
    return {"k": s["ko"], "v": s["vo"]}


def _own_read(s):
    kv, cache = _cache(s)
    kv.read(cache, s["blocks"], s["lens"], s["ko"], s["vo"], starts=s["back"], max_new=s["back_max"])
    return {"k": s["ko"], "v": s["vo"]}


def _own_attend(s):
    kv, cache = _cache(s)
    c = s["case"]
    if s["ws"] is None:                                    # a serving loop keeps its workspace
        s["ws"] = kv.attend_workspace(cache, s["q"], s["blocks"], starts=s["starts"], max_q=s["max_new"],
                                      max_len=s["max_len"], weights=s.get("w"))
    kv.attend(cache, s["blocks"], s["lens"], s["q"], s["out"], starts=s["starts"], max_q=s["max_new"],
              max_len=s["max_len"], causal=c["causal"], window=c["window"], weights=s.get("w"), ws=s["ws"])
    return {"out": s["out"], "weights": s["w"]} if c["weights"] else {"out": s["out"]}


def _own_evict(s):
    kv, cache = _cache(s)
    c = s["case"]
    kv.evict(cache, s["blocks"], s["lens"], s["w"], c["keep"], c["recent"], s["to"], s["to_lens"], s["to_w"],
             s["index"], max_len=s["max_len"])
    kv.read(cache, s["to"], s["to_lens"], s["ko"], s["vo"], starts=s["back"], max_new=s["back_max"])
    return {"index": s["index"], "lens": s["to_lens"], "weights": s["to_w"], "k": s["ko"], "v": s["vo"]}


# --- plain forms ------------------------------------------------------------

def _k_tokens(k, Dp):
    """(n, heads, 64 Dp) bytes of key blocks -> (n, 64, heads, Dp), still as bytes."""
    n, h = k.shape[:2]
    x = k.view(n, h, Dp // 32, 2, 16, 4, 2, 8).permute(0, 3, 6, 4, 1, 2, 5, 7)
    return x.reshape(n, BLOCK, h, Dp)


def _k_blocks(x):
    """The inverse of _k_tokens."""
    n, _, h, Dp = x.shape
    return x.view(n, 2, 2, 16, h, Dp // 32, 4, 8).permute(0, 4, 5, 1, 3, 6, 2, 7).reshape(n, h, BLOCK * Dp)


def _v_tokens(v, Dp):
    n, h = v.shape[:2]
    return v.view(n, h, Dp, 4, 4, 4).permute(0, 4, 3, 5, 1, 2).reshape(n, BLOCK, h, Dp)


def _v_blocks(x):
    n, _, h, Dp = x.shape
    return x.view(n, 4, 4, 4, h, Dp).permute(0, 4, 5, 2, 1, 3).reshape(n, h, BLOCK * Dp)


def _values(tokens, scale):
    """(n, 64, heads, Dp) bytes and (n, heads) scales -> float32 values."""
    return (tokens.float() - 128.0) * scale[:, None, :, None]


def _where(starts, lens, T):
    """Sequence and position of each of T packed tokens, the last ones of their sequences."""
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(starts[1:].contiguous().long(), t, right=True)
    return b, lens.long()[b] - (starts.long()[b + 1] - t)


def _plain_dense(s, ids, first, lens):
    """The tokens that s["back"] names, as (T, heads, D) values, out of the blocks ids (B, n), block first[b] on."""
    D, Hkv = s["case"]["D"], s["case"]["Hkv"]
    Dp = _row(D)
    B, n = ids.shape
    b, pos = _where(s["back"], lens, s["back_T"])
    pos = pos - first[b] * BLOCK

    def dense(pool, scales, to_tokens):
        x = _values(to_tokens(pool[ids.reshape(-1)], Dp), scales[ids.reshape(-1)])
        return x.view(B, n * BLOCK, Hkv, Dp)[b, pos, :, :D].to(s["ko"].dtype)

    return {"k": dense(s["k"], s["ks"], _k_tokens), "v": dense(s["v"], s["vs"], _v_tokens)}


def _plain_read(s):
    ids = s["blocks"].long().clamp(min=0)
    return _plain_dense(s, ids, torch.zeros_like(ids[:, 0]), s["lens"])


def _requantise(new, is_new, old, scale):
    """New values (B, n, 64, heads, Dp) into blocks of old codes with old scales (0: no old tokens)."""
    amax = (new.abs() * is_new).amax(dim=(2, 4))
    s2 = torch.maximum(scale, amax / torch.full_like(amax, 127.0))
    div = torch.where(s2 > 0, s2, torch.ones_like(s2))
    kept = torch.round(old * (scale / div)[:, :, None, :, None])
    put = torch.round(new / div[:, :, None, :, None])
    return torch.where(is_new, put, kept), s2


def _plain_append(s):
    c = s["case"]
    Dp, B = _row(c["D"]), c["B"]
    lens, starts = s["lens"].long(), s["starts"].long()
    p0 = lens - (starts[1:] - starts[:-1])
    first = p0 // BLOCK
    n = (s["max_new"] + BLOCK - 2) // BLOCK + 1            # blocks that a sequence's new tokens can touch
    blk = first[:, None] + torch.arange(n, device=DEV)
    real = blk * BLOCK < lens[:, None]
    ids = torch.where(real, s["blocks"].long().gather(1, blk.clamp(max=s["blocks"].shape[1] - 1)), s["k"].shape[0] - 1)
    pos = blk[:, :, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    is_new = ((pos >= p0[:, None, None]) & (pos < lens[:, None, None]))[:, :, :, None, None]
    src = (starts[:-1, None, None] + pos - p0[:, None, None]).clamp(0, s["T"] - 1)
    started = (blk * BLOCK < p0[:, None])[:, :, None]
    pad = Dp - c["D"]

    def store(pool, scales, x, to_tokens, to_blocks):
        new = torch.nn.functional.pad(x.float()[src], (0, pad))
        old = (to_tokens(pool[ids.view(-1)], Dp).float() - 128.0).view(new.shape)
        keep = torch.where(started, scales[ids], torch.zeros((), device=DEV))
        codes, s2 = _requantise(new, is_new, old, keep)
        pool[ids.view(-1)] = to_blocks((codes + 128.0).to(torch.uint8).view(B * n, BLOCK, c["Hkv"], Dp))
        scales[ids.view(-1)] = s2.view(B * n, c["Hkv"])

    store(s["k"], s["ks"], s["kn"], _k_tokens, _k_blocks)
    store(s["v"], s["vs"], s["vn"], _v_tokens, _v_blocks)
    return _plain_dense(s, ids, first, s["lens"])


def _plain_attend(s):
    c = s["case"]
    B, H, Hkv, D = c["B"], c["H"], c["Hkv"], c["D"]
    G, Dp, n = H // Hkv, _row(D), s["max_new"]
    ids = s["blocks"].long().clamp(min=0)
    L = ids.shape[1] * BLOCK
    lens, starts = s["lens"].long(), s["starts"].long()

    def dense(pool, scales, to_tokens):
        x = _values(to_tokens(pool[ids.view(-1)], Dp), scales[ids.view(-1)])
        return x.view(B, L, Hkv, Dp).permute(0, 2, 1, 3)[..., :D].reshape(B * Hkv, L, D)

    count = starts[1:] - starts[:-1]
    i = torch.arange(n, device=DEV)
    src = (starts[:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["q"].float()[src].view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * n, D)
    keys = dense(s["k"], s["ks"], _k_tokens).transpose(1, 2).contiguous()
    x = torch.bmm(q, keys).mul_(1.0 / math.sqrt(D)).view(B, Hkv, G, n, L)
    j = torch.arange(L, device=DEV)
    at = (lens - count)[:, None] + i
    seen = (j < lens[:, None, None]) & (i[None, :, None] < count[:, None, None])
    if c["causal"]:
        seen = seen & (j <= at[:, :, None])
        if c["window"]:
            seen = seen & (j > at[:, :, None] - c["window"])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros((), device=DEV))
    x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    x.div_(torch.where(total > 0, total, torch.ones((), device=DEV)))
    o = torch.bmm(x.view(B * Hkv, G * n, L), dense(s["v"], s["vs"], _v_tokens))
    o = o.view(B, Hkv, G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    t = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    out = o[b, t - starts[b]].to(s["q"].dtype)
    if not c["weights"]:
        return {"out": out}
    s["w"] += x.sum(dim=(2, 3))
    return {"out": out, "weights": s["w"]}


def _plain_evict(s):
    c = s["case"]
    B, Hkv, D, keep, recent = c["B"], c["Hkv"], c["D"], c["keep"], c["recent"]
    Dp = _row(D)
    L = s["blocks"].shape[1] * BLOCK
    lens = s["lens"].long()
    kept = lens.clamp(max=keep)
    j = torch.arange(L, device=DEV)
    here = (j < lens[:, None])[:, None].expand(B, Hkv, L)
    late = (j >= lens[:, None] - recent)[:, None] & here
    w = s["w"]
    rank = torch.where(late, math.inf, torch.where(here, w, -math.inf))
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    slot = torch.arange(keep, device=DEV)
    order = torch.nn.functional.pad(order, (0, max(0, keep - L)), value=L)
    real = (slot < kept[:, None])[:, None].expand(B, Hkv, keep)
    index = torch.sort(torch.where(real, order, L), dim=-1).values
    cap = s["to"].shape[1] * BLOCK
    src = torch.nn.functional.pad(index, (0, max(0, cap - keep)), value=L)[..., :cap]
    real = src < L
    src = src.clamp(max=L - 1)
    s["to_w"].copy_(torch.where(real, w.gather(2, src), torch.zeros((), device=DEV)))
    s["index"].copy_(torch.where(index < L, index, torch.full_like(index, -1)))
    s["to_lens"].copy_(kept)
    ids = s["blocks"].long().clamp(min=0)
    at = ids.gather(1, (src // BLOCK).view(B, -1)).view(B, Hkv, cap)
    to = torch.where(s["to"] >= 0, s["to"].long(), s["k"].shape[0] - 1).view(-1)
    heads = torch.arange(Hkv, device=DEV)[None, :, None]

    def move(pool, scales, to_tokens, to_blocks):
        old = scales[at, heads] * real
        s2 = old.view(B, Hkv, cap // BLOCK, BLOCK).amax(dim=-1)
        div = torch.where(s2 > 0, s2, torch.ones_like(s2)).repeat_interleave(BLOCK, dim=2)
        tokens = to_tokens(pool[ids.view(-1)], Dp).view(B, L, Hkv, Dp).permute(0, 2, 1, 3)
        codes = tokens.gather(2, src[..., None].expand(B, Hkv, cap, Dp)).float() - 128.0
        codes = torch.round(codes * (old / div)[..., None]) + 128.0
        codes = codes.to(torch.uint8).view(B, Hkv, cap // BLOCK, BLOCK, Dp).permute(0, 2, 3, 1, 4)
        pool[to] = to_blocks(codes.reshape(-1, BLOCK, Hkv, Dp))
        scales[to] = s2.permute(0, 2, 1).reshape(-1, Hkv)

    move(s["k"], s["ks"], _k_tokens, _k_blocks)
    move(s["v"], s["vs"], _v_tokens, _v_blocks)
    kv = _plain_dense(s, to.view(B, -1), torch.zeros_like(lens), s["to_lens"])
    return {"index": s["index"], "lens": s["to_lens"], "weights": s["to_w"], **kv}


# ---------------------------------------------------------------------------
# The same in 64 bits, sequence by sequence, from the definition
# ---------------------------------------------------------------------------

def _places(Dp):
    """Byte of (token, value) in a block, for keys and values."""
    t = torch.arange(BLOCK, device=DEV)[:, None]
    d = torch.arange(Dp, device=DEV)[None, :]
    k = d // 32 * 2048 + t // 32 * 1024 + t % 16 * 64 + d // 8 % 4 * 16 + t // 16 % 2 * 8 + d % 8
    v = d * 64 + t // 4 % 4 * 16 + t // 16 * 4 + t % 4
    return k, v


def _one(s, b, n, which):
    """Codes (tokens, heads, D) and scales (tokens, heads) of sequence b's first n tokens, in float64."""
    D = s["case"]["D"]
    place = _places(_row(D))[0 if which == "k" else 1][:, :D]
    ids = s["blocks"][b, :(n + BLOCK - 1) // BLOCK].long()
    codes = s[which][ids][:, :, place].permute(0, 2, 1, 3).reshape(-1, s[which].shape[1], D)[:n].double() - 128
    scale = s[which + "s"][ids].double().repeat_interleave(BLOCK, dim=0)[:n]
    return codes, scale


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _shape(case)
    kind, Hkv, D = case["kind"], case["Hkv"], case["D"]
    starts = _starts(new)
    if kind == "read":
        got = {"k": [], "v": []}
        for b, n in enumerate(lens):
            for which in got:
                codes, scale = _one(s, b, n, which)
                got[which].append(codes * scale[..., None])
        return {which: torch.cat(x) for which, x in got.items()}
    if kind == "append":
        got = {"k": [], "v": []}
        for b, n in enumerate(lens):
            p0 = n - new[b]
            for which in got:
                codes, scale = _one(s, b, p0, which)
                x = s[which + "n"][starts[b]:starts[b + 1]].double()
                rows = []
                for at in range(p0 // BLOCK * BLOCK, n, BLOCK):
                    here = x[max(at - p0, 0):at + BLOCK - p0]
                    s2 = here.abs().amax(dim=(0, 2)) / 127
                    if at < p0:
                        s2 = torch.maximum(s2, scale[at])
                        rows.append(torch.round(codes[at:] * (scale[at] / s2)[:, None]) * s2[:, None])
                    rows.append(torch.round(here / s2[:, None]) * s2[:, None])
                got[which] += rows
        return {which: torch.cat(x) for which, x in got.items()}
    if kind == "evict":
        cap, keep, recent = s["to_w"].shape[2], case["keep"], case["recent"]
        got, weights = {"k": [], "v": []}, torch.zeros(s["to_w"].shape, dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            m = min(n, keep)
            rank = s["w"][b, :, :n].double()
            rank[:, max(0, n - recent):] = math.inf
            index = torch.argsort(-rank, dim=-1, stable=True)[:, :m].sort(dim=-1).values
            weights[b, :, :m] = s["w"][b, :, :n].double().gather(1, index)
            for which in got:
                codes, scale = _one(s, b, n, which)
                codes = codes.gather(0, index.t()[:, :, None].expand(m, Hkv, D))
                scale = scale.gather(0, index.t())
                for at in range(0, m, BLOCK):
                    s2 = scale[at:at + BLOCK].amax(dim=0)
                    ratio = scale[at:at + BLOCK] / s2
                    got[which].append(torch.round(codes[at:at + BLOCK] * ratio[..., None]) * s2[:, None])
        return {"index": None, "lens": None, "weights": weights, "k": torch.cat(got["k"]), "v": torch.cat(got["v"])}
    G = case["H"] // Hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    weights = s["w"].double() if case["weights"] else None
    for b, n in enumerate(lens):
        (kc, ks), (vc, vs) = _one(s, b, n, "k"), _one(s, b, n, "v")
        key, val = (kc * ks[..., None]).permute(1, 2, 0).contiguous(), (vc * vs[..., None]).permute(1, 0, 2).contiguous()
        j = torch.arange(n, device=DEV)
        step = max(1, 60_000_000 // (case["H"] * n))       # queries at a time
        for a in range(0, new[b], step):
            e = min(new[b], a + step)
            q = s["q"][starts[b] + a:starts[b] + e].double().view(e - a, Hkv, G, D).permute(1, 2, 0, 3)
            x = torch.bmm(q.reshape(Hkv, G * (e - a), D), key) / math.sqrt(D)
            x = x.view(Hkv, G, e - a, n)
            if case["causal"]:
                at = n - new[b] + torch.arange(a, e, device=DEV)[:, None]
                no = j > at
                if case["window"]:
                    no = no | (j <= at - case["window"])
                x = x.masked_fill(no, -math.inf)
            p = torch.softmax(x, dim=-1)
            if weights is not None:
                weights[b, :, :n] += p.sum(dim=(1, 2))
            o = torch.bmm(p.view(Hkv, G * (e - a), n), val).view(Hkv, G, e - a, D)
            out[starts[b] + a:starts[b] + e] = o.permute(2, 0, 1, 3).reshape(e - a, Hkv * G, D)
    return {"out": out, "weights": weights} if weights is not None else {"out": out}
