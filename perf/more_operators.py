"""Measured cases of what surrounds the 8-bit key/value cache when many sequences share it or grow long.

Six calls, each through the public binding where ``own`` is true and in elementary torch
operations otherwise (32 bits; 64 for the angles of far positions and for scores that decide
which blocks are taken):

* ``rotate``   norms of a projection's query and key heads, and the rotation by their positions on
  one or several axes, in one pass;
* ``fork``     sequences that continue others: full blocks are shared, started ones copied, blocks
  for new tokens taken from the free ones, those that nobody holds any more given back; the
  started blocks are read back;
* ``shared``   attention of new tokens over a cache whose sequences have their first blocks in
  common, group by group;
* ``choose``   the extremes of each block's keys brought up to date (``summarise``) and the blocks
  of highest possible score found for every query (``choose``);
* ``sparse``   both, then attention over the chosen blocks alone (``attend_chosen``).

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
EPS = 1e-6


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _rotate(name, T, H, Hkv, D, pairs, axes, adjacent, norm, far, dtype):
    return {"name": name, "kind": "rotate", "T": T, "H": H, "Hkv": Hkv, "D": D, "pairs": pairs, "axes": axes,
            "adjacent": adjacent, "norm": norm, "far": far, "dtype": dtype}


def _fork(name, B, parents, Hkv, D, len_lo, len_hi, room, spare, dtype):
    """B new sequences of B old ones; `parents` of these go on."""
    return {"name": name, "kind": "fork", "B": B, "parents": parents, "Hkv": Hkv, "D": D, "len_lo": len_lo,
            "len_hi": len_hi, "room": room, "spare": spare, "dtype": dtype}


def _shared(name, groups, each_lo, each_hi, pre_lo, pre_hi, own_lo, own_hi, q, H, Hkv, D, dtype):
    """`groups` groups of each_lo .. each_hi sequences, pre tokens (whole blocks) in common, own tokens after them."""
    return {"name": name, "kind": "shared", "groups": groups, "each_lo": each_lo, "each_hi": each_hi, "pre_lo": pre_lo,
            "pre_hi": pre_hi, "own_lo": own_lo, "own_hi": own_hi, "q": q, "H": H, "Hkv": Hkv, "D": D, "dtype": dtype}


def _pick(kind, name, B, H, Hkv, D, len_lo, len_hi, new, top, dtype):
    """Of each sequence's `new` last tokens (0: all) the blocks' extremes are new; the last q tokens look for `top` blocks."""
    return {"name": name, "kind": kind, "B": B, "H": H, "Hkv": Hkv, "D": D, "len_lo": len_lo, "len_hi": len_hi,
            "new": new, "top": top, "dtype": dtype}


def listed():
    return [
        # One user's next token, float32 from the projection's dequant epilogue, 32 heads. Latency counts.
        _rotate("rotate_step_b1", 1, 32, 32, 128, 64, 1, False, False, 4000, "f32"),
        # A whole prompt of hidden 8192: 64 heads over 8, normed, positions of a long context.
        _rotate("rotate_prompt_8k", 8192, 64, 8, 128, 64, 1, False, True, 1000000, "bf16"),
        # A video's tokens: time, height and width, heads of 80, adjacent pairs, an odd number of tokens.
        _rotate("rotate_video_3_axes", 5007, 16, 16, 80, 36, 3, True, True, 4000, "f16"),
        # A step of beam search, 8 beams of which 3 go on.
        _fork("fork_beams_b8", 8, 3, 32, 128, 2011, 2011, 1, 40, "f32"),
        # 64 samples of 9 prompts whose lengths differ, 40 heads (hidden 5120), room for 64 more tokens of each.
        _fork("fork_samples_b64", 64, 9, 40, 128, 400, 2000, 64, 300, "bf16"),
        # A few chats after one short instruction.
        _shared("shared_b6_1k", 1, 6, 6, 1024, 1024, 40, 300, 1, 32, 8, 128, "bf16"),
        # A serving batch after one long instruction, grouped heads (64 over 8, hidden 8192).
        _shared("shared_b64_16k", 1, 64, 64, 16384, 16384, 100, 900, 1, 64, 8, 128, "bf16"),
        # Several documents, each asked about by a few users with 3 drafted tokens, heads not grouped.
        _shared("shared_docs_b24", 5, 2, 8, 3000, 12000, 17, 500, 3, 32, 32, 128, "f16"),
        # A prompt has just been stored: the extremes of all its blocks, and the first token's choice.
        _pick("choose", "choose_prompt_32k", 1, 32, 8, 128, 32700, 32700, 0, 64, "bf16"),
        # A decode step's choice in a batch, float32 queries, heads not grouped.
        _pick("choose", "choose_step_b8", 8, 32, 32, 128, 3000, 9000, 1, 24, "f32"),
        # One very long context, 64 heads over 8 (hidden 8192), a thirtieth of it attended to.
        _pick("sparse", "sparse_128k", 1, 64, 8, 128, 131071, 131071, 1, 64, "f16"),
        # A batch of long sequences, two drafted tokens each.
        _pick("sparse", "sparse_b16_16k", 16, 32, 8, 128, 9000, 16384, 2, 48, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "fork", "shared", "shared", "choose", "sparse", "sparse"])
    D = rng.choice([64, 80, 96, 128, 128, 192, 256])
    dtype = rng.choice(["f32", "bf16", "f16"])
    Hkv = rng.choice([1, 2, 5, 8, 8, 32])
    G = rng.choice([1, 1, 4, 5, 8])
    while True:
        if kind == "rotate":
            axes = rng.choice([1, 1, 2, 3])
            c = _rotate("", _log_int(rng, 1, 8192), G * Hkv, Hkv, D, rng.choice([D // 2, D // 2, D // 4, 5]), axes,
                        rng.random() < 0.4, rng.random() < 0.6, _log_int(rng, 3000, 2000000), dtype)
        elif kind == "fork":
            B, top = _log_int(rng, 1, 128), _log_int(rng, 30, 8000)
            c = _fork("", B, rng.randint(1, B), Hkv, D, max(1, int(top * rng.uniform(0.1, 1))), top,
                      rng.choice([0, 1, 1, 70, 300]), _log_int(rng, 1, 1000), dtype)
        elif kind == "shared":
            each = _log_int(rng, 1, 64)
            pre, more = _log_int(rng, 64, 16384), _log_int(rng, 8, 2000)
            c = _shared("", rng.choice([1, 1, 2, 5]), max(1, each // 3), each, max(64, pre // 3), pre, max(8, more // 5),
                        more, rng.choice([1, 1, 1, 2, 5]), G * Hkv, Hkv, D, dtype)
        else:
            B, top = _log_int(rng, 1, 32), _log_int(rng, 200, 131000)
            new = rng.choice([1, 1, 3, 0] if kind == "choose" else [1, 1, 3])
            c = _pick(kind, "", B, G * Hkv, Hkv, D, max(100, int(top * rng.uniform(0.2, 1))), top, new,
                      _log_int(rng, 4, 128), dtype)
        del c["name"]
        w = work(c)
        if w["bytes"] <= 3e8 and w["flops"] <= 3e10 and _pool(c) <= 6e8 and _dense_work(c) <= 3e9:
            return c


# ---------------------------------------------------------------------------
# Lengths and inputs
# ---------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, the largest first, the others spread over the logarithm."""
    return [hi] + [int(round(lo * (hi / lo) ** ((i * 0.61803398875) % 1.0))) for i in range(1, n)]


def _row(D):
    """Values a head takes in the cache: its width, rounded up to one the cache is laid out for."""
    return 64 if D <= 64 else 96 if D <= 96 else 128 if D <= 128 else 192 if D <= 192 else 256


def _up(n):
    return (n + BLOCK - 1) // BLOCK


def _groups(case):
    """Of a shared case: sequences of each group, its blocks in common, and every sequence's length."""
    each = _spread(case["each_lo"], case["each_hi"], case["groups"])
    pre = [n // BLOCK for n in _spread(case["pre_lo"], case["pre_hi"], case["groups"])]
    more = _spread(case["own_lo"], case["own_hi"], sum(each))
    lens = [p * BLOCK for n, p in zip(each, pre) for _ in range(n)]
    return each, pre, [a + b for a, b in zip(lens, more)]


def _lens(case):
    if case["kind"] == "shared":
        return _groups(case)[2]
    return _spread(case["len_lo"], case["len_hi"], case["B"])


def _queries(case):
    """Query tokens of each sequence."""
    return case["q"] if case["kind"] == "shared" else max(1, case["new"])


def _parents(case):
    """Each new sequence's old one: those that go on are their own, so that the same step can follow; one has none."""
    B, rng = case["B"], random.Random(case["B"] * 1000 + case["parents"])
    stay = rng.sample(range(B), case["parents"])
    p = [i if i in stay else rng.choice(stay) for i in range(B)]
    gone = [i for i in range(B) if i not in stay]
    if len(gone) > 20:
        p[gone[-1]] = -1
    return p


def _es(case):
    return 4 if case["dtype"] == "f32" else 2


def _pool(case):
    """Bytes of the cache's blocks."""
    if case["kind"] == "rotate":
        return 0
    lens, one = _lens(case), case["Hkv"] * 2 * BLOCK * _row(case["D"])
    if case["kind"] == "shared":
        each, pre, _ = _groups(case)
        return one * (sum(_up(n) for n in lens) - sum((e - 1) * p for e, p in zip(each, pre)))
    if case["kind"] == "fork":
        return one * (sum(_up(n) for n in lens) + case["spare"] + 2 * case["B"] * _up(case["room"] + BLOCK))
    return one * sum(_up(n) for n in lens)


def _dense_work(case):
    """Values of the largest array that the plain form of an attention makes."""
    if case["kind"] == "shared":
        lens = _lens(case)
        return len(lens) * max(lens) * max(case["Hkv"] * case["D"], case["H"] * case["q"])
    if case["kind"] in ("choose", "sparse"):
        blocks, T = _up(max(_lens(case))), case["B"] * _queries(case)
        return T * case["Hkv"] * case["D"] * max(4 * blocks, BLOCK * case["top"])
    return 0


def work(case):
    kind, D, Hkv, es = case["kind"], case["D"], case["Hkv"], _es(case)
    if kind == "rotate":
        n = case["T"] * (case["H"] + Hkv) * D
        return {"bytes": 2 * n * es + 4 * case["T"] * case["axes"], "flops": n * (6 if case["norm"] else 3)}
    lens = _lens(case)
    if kind == "fork":
        seen, copies, rest, tables = set(), 0, 0, 0
        for p in _parents(case):
            if p < 0:
                continue
            copies += p in seen and lens[p] % BLOCK > 0
            seen.add(p)
            rest += lens[p] % BLOCK
            tables += 8 * _up(lens[p])
        move = 2 * copies * Hkv * 2 * BLOCK * D
        return {"bytes": move + tables + 2 * Hkv * D * rest * (1 + es), "flops": 2 * Hkv * D * rest}
    T, G = len(lens) * _queries(case), case["H"] // Hkv
    rows = 2 * T * case["H"] * D * es
    if kind == "shared":
        each, pre, _ = _groups(case)
        pairs = sum(case["q"] * n - case["q"] * (case["q"] - 1) // 2 for n in lens)
        keys = sum(p * BLOCK for p in pre) + sum(n for n in lens) - sum(e * p * BLOCK for e, p in zip(each, pre))
        return {"bytes": 2 * Hkv * keys * D + rows + 8 * Hkv * keys // BLOCK, "flops": 4 * case["H"] * D * pairs}
    blocks = [_up(n) for n in lens]
    fresh = sum(n if case["new"] == 0 else min(case["new"] + BLOCK, n) for n in lens) * D * Hkv
    b = fresh + 2 * fresh // BLOCK + 2 * sum(blocks) * D * Hkv + T * case["H"] * D * es + 4 * T * Hkv * case["top"]
    b += 4 * _queries(case) * sum(blocks) * Hkv
    f = 4 * _queries(case) * sum(blocks) * D * case["H"]
    if kind == "sparse":
        taken = _queries(case) * sum(min(n, case["top"]) for n in blocks) * BLOCK
        b += 2 * taken * Hkv * D + T * case["H"] * D * es
        f += 4 * case["H"] * D * taken
    return {"bytes": b, "flops": f}


def _codes(g, shape, spread):
    return torch.randn(shape, generator=g, device=DEV).mul_(spread).round_().clamp_(-127, 127).add_(128).to(torch.uint8)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return s


def _frequencies(case):
    """(axes, pairs): what an axis turns a pair by; each axis has a run of the pairs, of frequencies 10000^-x."""
    pairs, axes = case["pairs"], case["axes"]
    f = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], dtype=torch.float64)
    axis = torch.tensor([min(i * axes // pairs, axes - 1) for i in range(pairs)])
    return (f * (axis == torch.arange(axes)[:, None])).float().to(DEV).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    order = random.Random(int(seed))
    kind, D, Hkv = case["kind"], case["D"], case["Hkv"]
    dt = DTYPES[case["dtype"]]
    s = {"case": case, "ws": {}}
    if kind == "rotate":
        # heads of a fused projection: the rows of q and k are further apart than their values
        T, H = case["T"], case["H"]
        y = (torch.randn((T, (H + 2 * Hkv) * D), generator=g, device=DEV) * 1.5).to(dt)
        s["q"], s["k"] = y[:, :H * D].view(T, H, D), y[:, H * D:(H + Hkv) * D].view(T, Hkv, D)
        s["q_out"] = torch.empty((T, H, D), dtype=dt, device=DEV)
        s["k_out"] = torch.empty((T, Hkv, D), dtype=dt, device=DEV)
        t = torch.arange(T, device=DEV) + order.randint(0, case["far"])
        # one axis: positions in order; more: time, and places in frames of 24 by 32
        rest = [t % (24 * 32) // 32, t % 32][:case["axes"] - 1]
        s["positions"] = torch.stack([t if case["axes"] == 1 else t // (24 * 32)] + rest).int().contiguous()
        s["freq"] = _frequencies(case)
        s["qw"] = torch.rand(D, generator=g, device=DEV) + 0.5 if case["norm"] else None
        s["kw"] = torch.rand(D, generator=g, device=DEV) + 0.5 if case["norm"] else None
        return s
    lens, Dp = _lens(case), _row(D)
    B = len(lens)
    used = [_up(n) for n in lens]
    width = max(used)
    if kind == "fork":
        n_blocks = sum(used) + case["spare"] + 2 * B * _up(case["room"] + BLOCK) + 1
        width += _up(case["room"] + BLOCK)
    elif kind == "shared":
        each, pre, _ = _groups(case)
        n_blocks = sum(used) - sum((e - 1) * p for e, p in zip(each, pre)) + 1
    else:
        n_blocks = sum(used) + 1
    free = list(range(n_blocks - 1))
    order.shuffle(free)
    if kind == "shared":
        table = []
        for e, p in zip(each, pre):
            common = [free.pop() for _ in range(p)]
            for _ in range(e):
                table.append(common + [free.pop() for _ in range(used[len(table)] - p)])
        s["group_starts"], s["shared"] = _ints(_starts(each)), _ints(pre)
        s["max_group"], s["max_shared"] = max(each), max(pre)
    else:
        table = [[free.pop() for _ in range(u)] for u in used]
    s["blocks"] = _ints([row + [-1] * (width - len(row)) for row in table])
    s["lens"], s["max_len"] = _ints(lens), max(lens)
    # Codes as a quantiser leaves them: about four standard deviations in 127 steps, values of about 1.
    s["k"] = _codes(g, (n_blocks, Hkv, BLOCK * Dp), 32.0)
    s["v"] = _codes(g, (n_blocks, Hkv, BLOCK * Dp), 32.0)
    s["ks"] = torch.rand((n_blocks, Hkv), generator=g, device=DEV) * 0.02 + 0.02
    s["vs"] = torch.rand((n_blocks, Hkv), generator=g, device=DEV) * 0.02 + 0.02
    if kind == "fork":
        parents = _parents(case)
        s["parents"], s["room"] = _ints(parents), torch.full((B,), case["room"], dtype=torch.int32, device=DEV)
        refs = torch.zeros(n_blocks, dtype=torch.int32, device=DEV)
        here = s["blocks"][s["blocks"] >= 0].long()
        s["refs"] = refs.index_add_(0, here, torch.ones_like(here, dtype=torch.int32))
        s["to_blocks"] = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
        s["to_lens"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        s["missing"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        st = _starts([lens[p] % BLOCK if p >= 0 else 0 for p in parents])
        s["back"], s["back_T"] = _ints(st), max(1, st[-1])
        s["ko"] = torch.zeros((s["back_T"], Hkv, D), dtype=dt, device=DEV)
        s["vo"] = torch.zeros((s["back_T"], Hkv, D), dtype=dt, device=DEV)
        return s
    H, n = case["H"], _queries(case)
    T = B * n
    y = (torch.randn((T, (H + 2 * Hkv) * D), generator=g, device=DEV) * 1.5).to(dt)
    s["q"] = y[:, :H * D].view(T, H, D)
    s["starts"], s["n"], s["T"] = _ints(_starts([n] * B)), n, T
    s["out"] = torch.empty((T, H, D), dtype=dt, device=DEV)
    if kind != "shared":
        # the blocks' extremes; of the newest tokens' blocks they are not up to date
        s["fresh"] = _ints(_starts([m if case["new"] == 0 else min(m, case["new"]) for m in lens]))
        s["max_fresh"] = max(lens) if case["new"] == 0 else case["new"]
        s["chosen"] = torch.empty((T, Hkv, case["top"]), dtype=torch.int32, device=DEV)
        s["scores"] = torch.zeros((T, Hkv, width), device=DEV)
        s["summary"] = torch.full((n_blocks, Hkv, 2, Dp), 128, dtype=torch.uint8, device=DEV)
        _plain_summary(s, torch.zeros_like(s["lens"]).long(), max(lens))
        last = (s["lens"].long() - 1) // BLOCK
        s["summary"][s["blocks"].long().gather(1, last[:, None])[:, 0]] = 128
        if case["new"] == 0:
            s["summary"].fill_(128)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"rotate": _own_rotate, "fork": _own_fork, "shared": _own_shared, "choose": _own_choose,
                "sparse": _own_sparse}[kind](s)
    return {"rotate": _plain_rotate, "fork": _plain_fork, "shared": _plain_shared, "choose": _plain_choose,
            "sparse": _plain_sparse}[kind](s)


def _own_rotate(s):
    from paper_2608_09291_amd import kv
    c = s["case"]
    kv.rotate(s["q"], s["k"], s["freq"], s["positions"], q_out=s["q_out"], k_out=s["k_out"], adjacent=c["adjacent"],
              norm=c["norm"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS)
    return {"q": s["q_out"], "k": s["k_out"]}


def _cache(s):
    from paper_2608_09291_amd import kv
    return kv, kv.Cache(s["k"], s["v"], s["ks"], s["vs"], s["case"]["D"])


def _turn(s):
    """The next step goes on from this one's tables."""
    s["blocks"], s["to_blocks"] = s["to_blocks"], s["blocks"]
    s["lens"], s["to_lens"] = s["to_lens"], s["lens"]


def _own_fork(s):
    kv, cache = _cache(s)
    if "ws" not in s["ws"]:                                # a serving loop keeps its workspaces
        s["ws"]["ws"] = kv.fork_workspace(cache, s["blocks"], s["to_blocks"])
    kv.fork(cache, s["refs"], s["blocks"], s["lens"], s["parents"], s["to_blocks"], s["to_lens"], s["missing"],
            room=s["room"], ws=s["ws"]["ws"])
    kv.read(cache, s["to_blocks"], s["to_lens"], s["ko"], s["vo"], starts=s["back"], max_new=BLOCK)
    _turn(s)
    return {"blocks": s["blocks"], "lens": s["lens"], "refs": s["refs"], "missing": s["missing"], "k": s["ko"], "v": s["vo"]}


def _own_shared(s):
    kv, cache = _cache(s)
    if "ws" not in s["ws"]:
        s["ws"]["ws"] = kv.attend_shared_workspace(cache, s["q"], s["blocks"], s["group_starts"], starts=s["starts"],
                                                   max_q=s["n"], max_group=s["max_group"], max_shared=s["max_shared"],
                                                   max_len=s["max_len"])
    kv.attend_shared(cache, s["blocks"], s["lens"], s["q"], s["out"], s["group_starts"], s["shared"], starts=s["starts"],
                     max_q=s["n"], max_group=s["max_group"], max_shared=s["max_shared"], max_len=s["max_len"],
                     ws=s["ws"]["ws"])
    return {"out": s["out"]}


def _own_pick(s):
    kv, cache = _cache(s)
    c = s["case"]
    if "choose" not in s["ws"]:
        s["ws"]["choose"] = kv.choose_workspace(cache, s["blocks"], s["chosen"], starts=s["starts"], max_q=s["n"])
    kv.summarise(cache, s["blocks"], s["lens"], s["summary"], starts=s["fresh"], max_new=s["max_fresh"])
    kv.choose(cache, s["summary"], s["blocks"], s["lens"], s["q"], s["scores"], s["chosen"], starts=s["starts"],
              max_q=s["n"], max_len=s["max_len"], sinks=1, recent=2, ws=s["ws"]["choose"])
    return kv, cache


def _own_choose(s):
    _own_pick(s)
    return {"chosen": s["chosen"], "scores": s["scores"]}


def _own_sparse(s):
    kv, cache = _own_pick(s)
    if "ws" not in s["ws"]:
        s["ws"]["ws"] = kv.attend_chosen_workspace(cache, s["q"], s["blocks"], s["chosen"], starts=s["starts"], max_q=s["n"])
    kv.attend_chosen(cache, s["blocks"], s["lens"], s["q"], s["out"], s["chosen"], starts=s["starts"], max_q=s["n"],
                     ws=s["ws"]["ws"])
    return {"chosen": s["chosen"], "scores": s["scores"], "out": s["out"]}


# --- plain forms ------------------------------------------------------------

def _plain_rotate(s):
    c = s["case"]
    angle = (s["positions"][:, :, None].double() * s["freq"][:, None].double()).sum(0)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    P = c["pairs"]

    def one(x, w):
        x = x.float()
        if c["norm"]:
            x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w
        a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if c["adjacent"] else (x[..., :P], x[..., P:2 * P])
        lo, hi = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack((lo, hi), dim=-1).flatten(-2) if c["adjacent"] else torch.cat((lo, hi), dim=-1)
        return torch.cat((turned, x[..., 2 * P:]), dim=-1)

    s["q_out"].copy_(one(s["q"], s["qw"]))
    s["k_out"].copy_(one(s["k"], s["kw"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _k_tokens(k, Dp):
    """(n, heads, 64 Dp) bytes of key blocks -> (n, 64, heads, Dp), still as bytes."""
    n, h = k.shape[:2]
    x = k.view(n, h, Dp // 32, 2, 16, 4, 2, 8).permute(0, 3, 6, 4, 1, 2, 5, 7)
    return x.reshape(n, BLOCK, h, Dp)


def _v_tokens(v, Dp):
    n, h = v.shape[:2]
    return v.view(n, h, Dp, 4, 4, 4).permute(0, 4, 3, 5, 1, 2).reshape(n, BLOCK, h, Dp)


def _values(tokens, scale):
    """(n, 64, heads, Dp) bytes and (n, heads) scales -> float32 values."""
    return (tokens.float() - 128.0) * scale[:, None, :, None]


def _where(starts, lens, T):
    """Sequence and position of each of T packed tokens, the last ones of their sequences."""
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(starts[1:].contiguous().long(), t, right=True).clamp(max=lens.shape[0] - 1)
    return b, lens.long()[b] - (starts.long()[b + 1] - t)


def _plain_fork(s):
    c = s["case"]
    old, lens, refs = s["blocks"].long(), s["lens"].long(), s["refs"]
    B, width = old.shape
    n_blocks = refs.shape[0]
    parents = s["parents"].long()
    has = (parents >= 0) & (parents < B)
    p = parents.clamp(0, B - 1)
    before = torch.ones((B, B), dtype=torch.bool, device=DEV).tril(-1)
    first = has & ~((parents[:, None] == parents) & before).any(dim=1)
    length = torch.where(has, lens[p], 0)
    full, used = length // BLOCK, (length + BLOCK - 1) // BLOCK
    need = ((length + s["room"].long() + BLOCK - 1) // BLOCK).clamp(max=width)
    i = torch.arange(width, device=DEV)
    src = torch.where(has[:, None], old[p], -1)
    valid = (src >= 0) & (src < n_blocks)
    src = torch.where(valid, src, -1)
    late = (i >= full[:, None]) & (i < need[:, None])
    kept = late & first[:, None] & valid & (refs.long()[src.clamp(min=0)] == 1)
    fresh = late & ~kept & (valid | (i >= used[:, None]))
    copied = fresh & (i < used[:, None])
    free = refs == 0
    missing = (fresh.sum() - free.sum()).clamp(min=0)
    ids = torch.argsort(~free, stable=True)                # the free blocks first, in order
    rank = (fresh.view(-1).cumsum(0) - 1).clamp(0, n_blocks - 1).view(B, width)
    new = torch.where(fresh, ids[rank], torch.where(kept | (i < full[:, None]), src, -1))
    spare = n_blocks - 1                                   # no sequence has it: entries without a copy move it to itself
    a, b = torch.where(copied, src, spare), torch.where(copied, new, spare)
    at = full.clamp(max=width - 1)[:, None]                # a sequence copies one block at most, its started one
    a, b = a.gather(1, at)[:, 0], b.gather(1, at)[:, 0]
    for pool in (s["k"], s["v"], s["ks"], s["vs"]):
        pool[b] = pool[a]
    one = torch.ones(B * width, dtype=torch.int32, device=DEV)
    was = ((old >= 0) & (old < n_blocks)).view(-1)
    count = torch.zeros(n_blocks + 1, dtype=torch.int32, device=DEV)
    count.index_add_(0, torch.where(new >= 0, new, n_blocks).view(-1), one)
    count.index_add_(0, torch.where(was, old.view(-1), n_blocks), -one)
    enough = missing == 0
    refs += torch.where(enough, count[:-1], 0)
    s["to_blocks"].copy_(torch.where(enough, new, -1))
    s["to_lens"].copy_(torch.where(enough, length, 0))
    s["missing"].copy_(missing)
    _turn(s)
    Dp = _row(c["D"])
    t = torch.arange(s["back_T"], device=DEV)
    b, pos = _where(s["back"], s["lens"], s["back_T"])
    ok = (pos >= 0) & (t < s["back"][-1])
    pos = pos.clamp(min=0)
    blk = s["blocks"].long()[b, pos // BLOCK]
    ok = (ok & (blk >= 0))[:, None, None]
    blk = blk.clamp(min=0)
    last = s["blocks"].long().gather(1, (s["lens"].long()[:, None] // BLOCK).clamp(max=width - 1))[:, 0].clamp(min=0)

    def back(pool, scales, to_tokens, to):                 # (all of them lie in the sequences' last blocks)
        tokens = to_tokens(pool[last], Dp)[b, pos % BLOCK, :, :c["D"]].float() - 128.0
        to.copy_(torch.where(ok, tokens * scales[blk][..., None], 0.0))

    back(s["k"], s["ks"], _k_tokens, s["ko"])
    back(s["v"], s["vs"], _v_tokens, s["vo"])
    return {"blocks": s["blocks"], "lens": s["lens"], "refs": s["refs"], "missing": s["missing"], "k": s["ko"], "v": s["vo"]}


def _softmax(x, seen):
    """Over the last dimension, of the scores that are seen; zeros where there are none."""
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    x.sub_(torch.where(top > -math.inf, top, torch.zeros((), device=DEV))).exp_()
    total = x.sum(dim=-1, keepdim=True)
    return x.div_(torch.where(total > 0, total, torch.ones((), device=DEV)))


def _plain_shared(s):
    c = s["case"]
    H, Hkv, D, n = c["H"], c["Hkv"], c["D"], s["n"]
    G, Dp = H // Hkv, _row(D)
    ids = s["blocks"].long().clamp(min=0)
    B, L = ids.shape[0], ids.shape[1] * BLOCK
    lens = s["lens"].long()

    def dense(pool, scales, to_tokens):
        x = _values(to_tokens(pool[ids.view(-1)], Dp), scales[ids.view(-1)])
        return x.view(B, L, Hkv, Dp).permute(0, 2, 1, 3)[..., :D].reshape(B * Hkv, L, D)

    q = s["q"].float().reshape(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * n, D)
    x = torch.bmm(q, dense(s["k"], s["ks"], _k_tokens).transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(D))
    at = (lens - n)[:, None] + torch.arange(n, device=DEV)
    seen = torch.arange(L, device=DEV) <= at[:, :, None]
    x = _softmax(x.view(B, Hkv, G, n, L), seen[:, None, None])
    o = torch.bmm(x.view(B * Hkv, G * n, L), dense(s["v"], s["vs"], _v_tokens))
    s["out"].copy_(o.view(B, Hkv, G, n, D).permute(0, 3, 1, 2, 4).reshape(B * n, H, D))
    return {"out": s["out"]}


def _plain_summary(s, p0, most):
    """The extremes of the key codes of every block that holds tokens from p0 on, at most `most` of them."""
    Dp = _row(s["case"]["D"])
    first, lens = p0 // BLOCK, s["lens"].long()
    n = min((most + BLOCK - 2) // BLOCK + 1, s["blocks"].shape[1])
    blk = first[:, None] + torch.arange(n, device=DEV)
    real = blk * BLOCK < lens[:, None]
    ids = torch.where(real, s["blocks"].long().gather(1, blk.clamp(max=s["blocks"].shape[1] - 1)), s["k"].shape[0] - 1)
    ids = ids.view(-1)
    for a in range(0, ids.shape[0], 4096):                 # blocks at a time
        part = ids[a:a + 4096]
        tokens = _k_tokens(s["k"][part], Dp)
        t = (blk.view(-1)[a:a + 4096] * BLOCK)[:, None] + torch.arange(BLOCK, device=DEV)
        here = (t < lens.repeat_interleave(n)[a:a + 4096][:, None])[:, :, None, None]
        lo = torch.where(here, tokens, 255).amin(dim=1)
        hi = torch.where(here, tokens, 0).amax(dim=1)
        s["summary"][part] = torch.stack((lo, hi), dim=2)


def _plain_pick(s):
    c = s["case"]
    Hkv, D, n, T, top = c["Hkv"], c["D"], s["n"], s["T"], c["top"]
    G = c["H"] // Hkv
    lens = s["lens"].long()
    fresh = s["fresh"].long()
    _plain_summary(s, lens - (fresh[1:] - fresh[:-1]), s["max_fresh"])
    ids = s["blocks"].long()
    B, N = ids.shape
    ids = ids.clamp(min=0)
    ends = s["summary"][ids.view(-1)][..., :D].reshape(B, N, Hkv, 2 * D).permute(0, 2, 3, 1).double().sub_(128.0)
    q = s["q"].double().reshape(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4)
    q = torch.cat((q.clamp(max=0), q.clamp(min=0)), dim=-1).reshape(B * Hkv, n * G, 2 * D)
    x = torch.bmm(q, ends.reshape(B * Hkv, 2 * D, N)).view(B, Hkv, n, G, N).amax(dim=3)
    x = x * s["ks"][ids.view(-1)].double().view(B, N, Hkv).permute(0, 2, 1)[:, :, None]
    x = x.float().permute(0, 2, 1, 3).reshape(T, Hkv, N)
    _, at = _where(s["starts"], s["lens"], T)
    i, here = torch.arange(N, device=DEV), at // BLOCK + 1
    s["scores"].copy_(torch.where((i < here[:, None])[:, None], x, s["scores"]))
    x.masked_fill_(((i < 1) | (i >= here[:, None] - 2))[:, None], math.inf)
    x.masked_fill_((i >= here[:, None])[:, None], -math.inf)
    best = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :top]
    best = torch.nn.functional.pad(best, (0, max(0, top - N)), value=N)
    best = torch.where(torch.arange(top, device=DEV) < here[:, None, None], best, N)
    best = torch.sort(best, dim=-1).values
    s["chosen"].copy_(torch.where(best < N, best, -1))
    return at


def _plain_choose(s):
    _plain_pick(s)
    return {"chosen": s["chosen"], "scores": s["scores"]}


def _plain_sparse(s):
    at = _plain_pick(s)
    c = s["case"]
    Hkv, D, n, T, top = c["Hkv"], c["D"], s["n"], s["T"], c["top"]
    G, Dp = c["H"] // Hkv, _row(c["D"])
    chosen = s["chosen"].long()
    real = chosen >= 0
    blk = chosen.clamp(min=0)
    b = torch.arange(T, device=DEV) // n
    ids = s["blocks"].long()[b[:, None, None], blk]
    heads = torch.arange(Hkv, device=DEV)[None, :, None].expand(T, Hkv, top)

    def dense(pool, scales, to_tokens):
        x = pool[ids, heads].view(T * Hkv * top, 1, BLOCK * Dp)
        x = _values(to_tokens(x, Dp), scales[ids, heads].view(-1, 1))
        return x.view(T * Hkv, top * BLOCK, Dp)[..., :D].contiguous()

    q = s["q"].float().reshape(T * Hkv, G, D)
    x = torch.bmm(q, dense(s["k"], s["ks"], _k_tokens).transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(D))
    j = blk[..., None] * BLOCK + torch.arange(BLOCK, device=DEV)
    seen = ((j <= at[:, None, None, None]) & real[..., None]).view(T * Hkv, 1, top * BLOCK)
    x = _softmax(x, seen)
    s["out"].copy_(torch.bmm(x, dense(s["v"], s["vs"], _v_tokens)).view(T, c["H"], D))
    return {"chosen": s["chosen"], "scores": s["scores"], "out": s["out"]}


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


def _dense(s, ids, which):
    """Blocks ids (a list of numbers) as float64 values (tokens, heads, D)."""
    D = s["case"]["D"]
    place = _places(_row(D))[0 if which == "k" else 1][:, :D]
    ids = torch.as_tensor(ids, device=DEV).long()
    codes = s[which][ids][:, :, place].permute(0, 2, 1, 3).reshape(-1, s[which].shape[1], D).double() - 128
    return codes * s[which + "s"][ids].double().repeat_interleave(BLOCK, dim=0)[..., None]


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "rotate":
        return {"q": _exact_rotate(s, s["q"], s["qw"]), "k": _exact_rotate(s, s["k"], s["kw"])}
    if kind == "fork":
        rows = {"k": [], "v": []}
        for p in s["parents"].tolist():
            n = int(s["lens"][p]) if p >= 0 else 0
            if n % BLOCK:
                for which in rows:
                    rows[which].append(_dense(s, [int(s["blocks"][p, n // BLOCK])], which)[:n % BLOCK])
        zero = torch.zeros(s["ko"].shape, dtype=torch.float64, device=DEV)
        got = {which: torch.cat(x) if x else zero for which, x in rows.items()}
        return {"blocks": None, "lens": None, "refs": None, "missing": None, **got}
    H, Hkv, D, n = case["H"], case["Hkv"], case["D"], s["n"]
    G = H // Hkv
    out = torch.zeros((s["T"], H, D), dtype=torch.float64, device=DEV)
    if kind == "shared":
        for b, length in enumerate(s["lens"].tolist()):
            ids = s["blocks"][b, :_up(length)]
            k, v = (_dense(s, ids, which)[:length].permute(1, 0, 2).contiguous() for which in ("k", "v"))
            for i in range(n):
                end = length - n + i + 1
                q = s["q"][b * n + i].double().view(Hkv, G, D)
                p = torch.softmax(torch.bmm(q, k[:, :end].transpose(1, 2).contiguous()) / math.sqrt(D), dim=-1)
                out[b * n + i] = torch.bmm(p, v[:, :end].contiguous()).view(H, D)
        return {"out": out}
    scores = s["scores"].double()
    for b, length in enumerate(s["lens"].tolist()):
        ids = s["blocks"][b, :_up(length)]
        keys = _dense(s, ids, "k")
        values = _dense(s, ids, "v") if kind == "sparse" else None
        hidden = (torch.arange(keys.shape[0], device=DEV) >= length).view(-1, BLOCK, 1, 1)
        lo = keys.view(-1, BLOCK, Hkv, D).masked_fill(hidden, math.inf).amin(dim=1)
        hi = keys.view(-1, BLOCK, Hkv, D).masked_fill(hidden, -math.inf).amax(dim=1)
        for i in range(n):
            end = length - n + i + 1
            here = _up(end)
            for h in range(Hkv):
                q = s["q"][b * n + i, h * G:h * G + G].double()
                reach = torch.maximum(q[:, None] * lo[:here, h], q[:, None] * hi[:here, h]).sum(dim=-1).amax(dim=0)
                scores[b * n + i, h, :here] = reach
                if kind == "choose":
                    continue
                reach = reach.float()
                reach[:1] = math.inf
                reach[max(0, here - 2):] = math.inf
                best = torch.argsort(-reach, stable=True)[:case["top"]].sort().values
                j = (best[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)).view(-1)
                j = j[j < end]
                p = torch.softmax(q @ keys[j, h].t() / math.sqrt(D), dim=-1)
                out[b * n + i, h * G:h * G + G] = p @ values[j, h]
    return {"chosen": None, "scores": scores, "out": out} if kind == "sparse" else {"chosen": None, "scores": scores}


def _exact_rotate(s, x, weight):
    """Pairs as complex numbers times e^(i angle)."""
    c = s["case"]
    P, x = c["pairs"], x.double()
    if c["norm"]:
        x = x * (x.pow(2).sum(dim=-1, keepdim=True) / c["D"] + EPS).rsqrt() * weight.double()
    angle = torch.zeros((c["T"], P), dtype=torch.float64, device=DEV)
    for a in range(c["axes"]):
        angle += s["positions"][a].double()[:, None] * s["freq"][a].double()
    turned = x[..., :2 * P]
    z = turned.unflatten(-1, (P, 2)) if c["adjacent"] else turned.unflatten(-1, (2, P)).transpose(-1, -2)
    z = torch.complex(z[..., 0], z[..., 1]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    z = torch.view_as_real(z)
    y = z.flatten(-2) if c["adjacent"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat((y, x[..., 2 * P:]), dim=-1)
