"""Normed heads, windows, trees of drafted tokens: operators next to the 8-bit paged cache, as cases that can be timed and compared with
their plain forms.

Every case is a dict of plain values; its "kind" names the part of a user's program it stands for:

  norm       a layer's queries and keys: root-mean-square norm of each head with its weight, then the rotary positions; with "grad" also
             the gradients of the inputs and of the weights
  window     attention over a full cache in which a query sees the last `window` tokens and the first `sinks` ones
  tree       attention of drafted tokens that form a tree: a node sees the sequence before the tree, its ancestors and itself
  slide      pages that no window will see again given back
  stream     a model generating with a window, layer by layer: norm with rotation, append, attention; after every token the pages slide
  speculate  one step of speculative decoding: a fork of each sequence takes the drafted tree, all layers are run on it, the fork is
             given up and the accepted branch appended to the original

`run` computes them in elementary torch operations while `own` is false and with the library's calls where it is true.  Shapes are those of
the repository's workloads: 28 query and 4 key/value heads at 28 layers, 32 and 4 at 48; two-second chunks of 350 tokens.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D, BLOCK = 128, 32
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the smallest call: one new token of eight sequences, between a layer's projections and its append
        {"name": "norm step", "kind": "norm", "dtype": "fp16", "batch": 8, "new": 1, "q_heads": 32, "kv_heads": 4,
         "sections": "24,20,20", "interleaved": True, "heads_inner": True, "grad": False, "start": 16384},
        # a layer of a prompt of odd length
        {"name": "norm prompt", "kind": "norm", "dtype": "bf16", "batch": 1, "new": 32767, "q_heads": 32, "kv_heads": 4,
         "sections": "24,20,20", "interleaved": True, "heads_inner": True, "grad": False, "start": 0},
        # training in 16 bits: forwards, backwards, gradients of both weights
        {"name": "norm train", "kind": "norm", "dtype": "bf16", "batch": 3, "new": 4095, "q_heads": 32, "kv_heads": 4,
         "sections": "16,24,24", "interleaved": False, "heads_inner": True, "grad": True, "start": 1000003},
        # the smallest attention with a window: one sequence, one key/value head, two seconds of sight
        {"name": "window tiny", "kind": "window", "dtype": "fp16", "layers": 1, "batch": 1, "q_heads": 7, "kv_heads": 1,
         "tokens": 2048, "new": 1, "ragged": False, "page": 64, "window": 350, "sinks": 4},
        # a layer of a large decode batch with a long window over long sequences
        {"name": "window batch", "kind": "window", "dtype": "bf16", "layers": 1, "batch": 16, "q_heads": 32, "kv_heads": 4,
         "tokens": 32768, "new": 1, "ragged": False, "page": 64, "window": 4096, "sinks": 64},
        # several queries per sequence, sequences of all lengths (one empty, one of a single token), all layers in one call
        {"name": "window ragged", "kind": "window", "dtype": "fp16", "layers": 28, "batch": 8, "q_heads": 28, "kv_heads": 4,
         "tokens": 1357, "new": 5, "ragged": True, "page": 32, "window": 511, "sinks": 1},
        # a prompt's second piece
        {"name": "window prompt", "kind": "window", "dtype": "bf16", "layers": 1, "batch": 1, "q_heads": 28, "kv_heads": 4,
         "tokens": 8192, "new": 2048, "ragged": False, "page": 64, "window": 1400, "sinks": 4},
        # a small tree behind one short sequence
        {"name": "tree tiny", "kind": "tree", "dtype": "fp16", "layers": 1, "batch": 1, "q_heads": 7, "kv_heads": 1,
         "tokens": 2048, "new": 7, "ragged": False, "page": 64},
        # trees of up to 64 nodes behind sequences of all lengths
        {"name": "tree batch", "kind": "tree", "dtype": "bf16", "layers": 1, "batch": 8, "q_heads": 28, "kv_heads": 4,
         "tokens": 16384, "new": 64, "ragged": True, "page": 64},
        # many long sequences after a long absence of housekeeping
        {"name": "slide", "kind": "slide", "dtype": "fp16", "layers": 28, "batch": 64, "q_heads": 4, "kv_heads": 1,
         "tokens": 2800, "new": 1, "ragged": True, "page": 32, "window": 700, "sinks": 4},
        # a model generating with a window
        {"name": "stream", "kind": "stream", "dtype": "fp16", "layers": 28, "batch": 4, "q_heads": 28, "kv_heads": 4,
         "tokens": 4090, "steps": 4, "page": 64, "window": 2047, "sinks": 4},
        # four sequences with 16 drafted tokens each, all layers
        {"name": "speculate", "kind": "speculate", "dtype": "fp16", "layers": 28, "batch": 8, "q_heads": 28, "kv_heads": 4,
         "tokens": 4090, "new": 16, "page": 64},
    ]


MOST_NORM = 36 * 32767 * 2           # elements / 128 x bytes of the largest listed case
MOST_TOKENS = 16 * 4 * 32768         # token-heads of a cache
MOST_SCORES = 28 * 2048 * 8192       # query heads x queries x keys
MOST_STREAM = 28 * 4 * 4 * 4096


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(lo * (max(hi, lo) / lo) ** rng.random()))))


def _heads(rng):
    kv, group = rng.choice([(1, 7), (2, 8), (4, 7), (4, 8), (4, 5), (8, 4), (8, 1), (3, 2)])
    return {"q_heads": kv * group, "kv_heads": kv}


def _half(rng):
    return {"dtype": rng.choice(["fp16", "bf16"]), "page": rng.choice([32, 64, 128, 256])}


def _sight(rng, tokens):
    return {"window": _log(rng, 1, 2 * tokens + 1), "sinks": rng.choice([0, 1, 4, 64, _log(rng, 1, tokens)])}


def draw(rng):
    kind = rng.choice(["norm"] * 4 + ["window"] * 5 + ["tree"] * 4 + ["slide", "stream", "speculate"])
    if kind == "norm":
        c = {"kind": kind, "dtype": rng.choice(["fp16", "bf16", "fp32"]), "batch": _log(rng, 1, 32), **_heads(rng)}
        grad = rng.random() < 0.5
        top = MOST_NORM // ((c["q_heads"] + c["kv_heads"]) * c["batch"] * (4 if c["dtype"] == "fp32" else 2) * (3 if grad else 1))
        sections, interleaved = rng.choice([("16,24,24", False), ("24,20,20", True), ("64,0,0", False), ("16,8,8", False), ("12,10,10", True), ("", False)])
        return {**c, "new": _log(rng, 1, top), "sections": sections, "interleaved": interleaved, "heads_inner": rng.random() < 0.5,
                "grad": grad, "start": _log(rng, 1, 2000000)}
    if kind in ("window", "tree"):
        c = {"kind": kind, "layers": rng.choice([1, 1, 1, rng.randint(2, 28)]), "batch": _log(rng, 1, 32), **_heads(rng), **_half(rng)}
        form = rng.choice(["one", "one", "few", "prompt"])
        new = _log(rng, 2, 128) if kind == "tree" else 1 if form == "one" else rng.randint(2, 16) if form == "few" else _log(rng, 17, 2048)
        top = MOST_TOKENS // (c["layers"] * c["batch"] * c["kv_heads"])
        if new > 1:
            top = min(top, MOST_SCORES // (c["layers"] * c["batch"] * c["q_heads"] * new))
        tokens = _log(rng, 1, max(1, min(131072, top)))
        return {**c, "tokens": tokens, "new": min(new, tokens), "ragged": rng.random() < 0.4, **(_sight(rng, tokens) if kind == "window" else {})}
    if kind == "slide":
        c = {"kind": kind, "layers": rng.choice([1, 28]), "batch": _log(rng, 1, 64), **_heads(rng), **_half(rng)}
        tokens = _log(rng, 1, max(1, min(32768, MOST_TOKENS // (c["layers"] * c["batch"] * c["kv_heads"]))))
        return {**c, "tokens": tokens, "new": 1, "ragged": rng.random() < 0.5, **_sight(rng, tokens)}
    if kind == "stream":
        c = {"kind": kind, "layers": rng.randint(1, 28), "batch": _log(rng, 1, 16), **_heads(rng), **_half(rng)}
        top = MOST_STREAM // (c["layers"] * c["batch"] * c["kv_heads"])
        tokens = _log(rng, 1, max(1, min(16384, top - 4)))
        return {**c, "tokens": tokens, "steps": rng.randint(1, 4), **_sight(rng, tokens)}
    c = {"kind": kind, "layers": rng.randint(1, 28), "batch": 2 * _log(rng, 1, 8), **_heads(rng), **_half(rng)}
    new = _log(rng, 2, 64)
    top = min(MOST_STREAM // (c["layers"] * c["batch"] * c["kv_heads"]) - 64, MOST_SCORES // (c["layers"] * c["batch"] * c["q_heads"] * new))
    return {**c, "tokens": _log(rng, 1, max(1, min(16384, top))), "new": new}


# ------------------------------------------------------------------------------------------------ sizes of a case
def _lens(case):
    """Tokens of each sequence: all alike, or of all lengths with an empty one and one of a single token among them.  Of speculate the
    sequences; their forks, which are the second half, are empty."""
    top, n = case["tokens"], case["batch"]
    if case["kind"] == "speculate":
        return [max(1, top - 13 * b) for b in range(n // 2)] + [0] * (n // 2)
    if not case.get("ragged"):
        return [top] * n
    return [top if b == 0 else 0 if b == 1 else min(1, top) if b == 2 else top * ((37 * b) % 64 + 1) // 64 for b in range(n)]


def _news(case):
    """Queries of each sequence."""
    if case["kind"] == "speculate":
        return [0] * (case["batch"] // 2) + [case["new"]] * (case["batch"] // 2)
    if not case.get("ragged"):
        return [case["new"]] * case["batch"]
    news = [case["new"] - (b * 29) % case["new"] if b != 3 else 0 for b in range(case["batch"])]
    return [min(n, m) for n, m in zip(news, _lens(case))] if case["kind"] == "tree" else news


def _pages_of(tokens, page):
    return (tokens + page - 1) // page


def _accepted(case):
    """Nodes of the accepted branch at most."""
    return min(4, case["new"])


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + 20261208)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _positions(batch, n, start):
    """int32 [3, batch, n]: in chunks of 350 tokens 300 of video (a grid of 15 x 20 at one time) and 50 of audio or text."""
    i = torch.arange(n, device="cuda")
    j = i % 350
    first, video = i - j, j < 300
    p = torch.stack([torch.where(video, first, i), torch.where(video, first + j // 20, i), torch.where(video, first + j % 20, i)])
    return (p + start).to(torch.int32)[:, None, :].expand(3, batch, n).contiguous()


def _sections(case):
    return case.get("sections", "24,20,20")


def _frequencies(case):
    """float64 [pairs]: theta^(-2 c / rotary channels)"""
    if not _sections(case):
        return None
    half = sum(int(x) for x in _sections(case).split(","))
    return 1000000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)


def _heads_in(case, x):
    """The same numbers as a projection [batch, token, head * 128] leaves them."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if case["heads_inner"] else x


def _weight(g, dt, *shape):
    """A norm's weight as training leaves it: around one, some channels several times as large."""
    w = 1 + 0.3 * _randn(g, *shape, D)
    w[..., torch.randint(0, D, (4,), generator=g, device="cuda")] *= 6
    return w.to(dt)


def _fill(x, g):
    """Keys of a recording in place of noise: a slow walk over time, four channels at ten times the size."""
    step = max(1, (1 << 26) // x[0].numel())
    for part in x.split(step):
        part.copy_(_randn(g, *part.shape).mul_(0.05).cumsum_(-2).add_(_randn(g, *part.shape)))
    x[..., torch.randint(0, D, (4,), generator=g, device="cuda")] *= 10
    return x


def _store(case, g, pages, width, lens, room):
    """A cache's buffers: pages in an order of their own, `lens` tokens per sequence and tables with room for `room` more of each."""
    L, B, H, P, dt = case["layers"], case["batch"], case["kv_heads"], case["page"], TYPES[case["dtype"]]
    codes = torch.empty(L, pages, H, 2, P, D, dtype=torch.int8, device="cuda")
    scales = torch.empty(L, pages, H, 2, P // BLOCK, device="cuda")
    for l in range(L):
        x = torch.empty(pages, H, 2, P // BLOCK, BLOCK, D, device="cuda")
        _fill(x[:, :, 0].view(pages, H, P, D), g)
        x[:, :, 1] = _randn(g, pages, H, P // BLOCK, BLOCK, D) * 0.3
        scales[l] = x.abs().amax((-1, -2)) / 127
        codes[l] = (x / scales[l][..., None, None]).round_().to(torch.int8).view(pages, H, 2, P, D)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    need = torch.tensor([_pages_of(n + r, P) for n, r in zip(lens, room)], device="cuda")
    j = torch.arange(width, device="cuda")
    used = j < need[:, None]
    table = torch.where(used, order[(used.flatten().cumsum(0) - 1).clamp(min=0).view(B, width)], -1)
    refs = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    refs[torch.where(used, table, pages).long().flatten()] = 1
    raw = (_randn(g, L, B, H, 2, BLOCK, D) * 0.5).to(dt)
    seq_len = torch.tensor(lens, dtype=torch.int32, device="cuda").expand(L, B).contiguous()
    return {"codes": codes, "scales": scales, "raw": raw, "table": table.contiguous(), "refs": refs[:pages].contiguous(), "seq_len": seq_len}


def _tree(case, seed):
    """Parents of every sequence's drafted nodes (-1: the sequence's newest token), wide at the top and narrow below."""
    rng = random.Random(1_000_003 * seed + 4)
    return [[max(-1, min(i - 1, int((i + 1) * rng.random() ** 1.5) - 1)) for i in range(case["new"])] for _ in range(case["batch"])]


def _branch(parents, most):
    """The nodes from the root to the deepest node, at most so many, in order."""
    depth = []
    for p in parents:
        depth.append(0 if p < 0 else depth[p] + 1)
    at, path = max(range(len(parents)), key=lambda i: (depth[i], -i)), []
    while at >= 0:
        path.append(at)
        at = parents[at]
    return path[::-1][:most]


def prepare(case, seed):
    g, kind, dt = _gen(seed), case["kind"], TYPES[case["dtype"]]
    H, Hq, B = case["kv_heads"], case["q_heads"], case["batch"]
    s = {"case": case, "kind": kind}
    if kind == "norm":
        n = case["new"]
        s["positions"], s["freq"] = _positions(B, n, case["start"]), _frequencies(case)
        for name, heads in (("q", Hq), ("k", H)):
            s[name] = _heads_in(case, (_randn(g, B, heads, n, D) * 3).to(dt))
            s[name + "_out"] = torch.empty_like(s[name])
            s[name + "_weight"] = _weight(g, dt)
            if case["grad"]:
                s[name + "_up"] = _heads_in(case, _randn(g, B, heads, n, D).to(dt))
                s[name + "_grad"] = torch.empty_like(s[name])
                s[name + "_weight_grad"] = torch.empty(D, device="cuda")
        return s
    L, P, lens = case["layers"], case["page"], _lens(case)
    if kind in ("window", "tree", "slide"):
        width = _pages_of(max(lens), P)
        s["cache"] = c = _store(case, g, sum(_pages_of(n, P) for n in lens) + 2, width, lens, [0] * B)
        if kind == "slide":
            s["dropped"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        else:
            n = case["new"]
            s["q"] = _randn(g, L, B, Hq, n, D).to(dt)
            s["out"] = torch.zeros(L, B, Hq, n, D, dtype=dt, device="cuda")
            s["q_len"] = torch.tensor(_news(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    elif kind == "stream":
        n = case["steps"]
        width = _pages_of(case["tokens"] + n, P)
        s["cache"] = c = _store(case, g, B * width + 2, width, lens, [n] * B)
        # (positions of every step in a tensor of its own, as a program that advances them has)
        s["positions"] = [_positions(B, 1, case["tokens"] + i) for i in range(n)]
        s["k"], s["q"] = (_randn(g, n, L, B, heads, 1, D).to(dt) for heads in (H, Hq))
        s["v"] = (_randn(g, n, L, B, H, 1, D) * 0.3).to(dt)
        s["out"] = torch.zeros(n, L, B, Hq, 1, D, dtype=dt, device="cuda")
    else:
        n, S, m = case["new"], B // 2, _accepted(case)
        width = _pages_of(max(lens) + n, P)
        s["cache"] = c = _store(case, g, 2 * S * (width + 2), width, lens, [0] * B)
        s["src"] = torch.arange(S, dtype=torch.int32, device="cuda")
        s["dst"] = s["src"] + S
        s["room"] = torch.tensor([0] * S + [a + n for a in lens[:S]], dtype=torch.int32, device="cuda")
        s["k"], s["q"] = (_randn(g, L, B, heads, n, D).to(dt) for heads in (H, Hq))
        s["v"] = (_randn(g, L, B, H, n, D) * 0.3).to(dt)
        s["out"] = torch.zeros(L, B, Hq, n, D, dtype=dt, device="cuda")
        s["q_len"] = torch.tensor(_news(case), dtype=torch.int32, device="cuda")
        s["start"] = torch.tensor(lens[:S], dtype=torch.int32, device="cuda").repeat(2)
        paths = [_branch(p, m) for p in _tree(case, seed)[S:]]
        s["path"] = torch.tensor([p + [0] * (m - len(p)) for p in paths], device="cuda").repeat(2, 1)
        s["taken"] = torch.tensor([len(p) for p in paths] + [0] * S, dtype=torch.int32, device="cuda")
        s["room_after"] = torch.tensor([a + len(p) for a, p in zip(lens, paths)] + [0] * S, dtype=torch.int32, device="cuda")
    if kind in ("tree", "speculate"):
        s["parents"] = torch.tensor(_tree(case, seed), dtype=torch.int32, device="cuda")
        s["seen"] = torch.zeros(B, case["new"], (case["new"] + 63) // 64, dtype=torch.int64, device="cuda")
        s["depth"] = torch.zeros(B, case["new"], dtype=torch.int32, device="cuda")
    if kind in ("stream", "speculate"):
        s["freq"] = _frequencies(case)
        s["q_weight"], s["k_weight"] = _weight(g, dt, L), _weight(g, dt, L)
        s["q_turned"], s["k_turned"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    if kind in ("slide", "stream", "speculate"):
        s["table0"], s["refs0"], s["len0"], s["raw0"] = (c[n].clone() for n in ("table", "refs", "seq_len", "raw"))
    return s


def _restore(s):
    """The state before the pass."""
    for name, kept in (("table", "table0"), ("refs", "refs0"), ("seq_len", "len0"), ("raw", "raw0")):
        s["cache"][name].copy_(s[kept])


# ------------------------------------------------------------------------------------------------ plain forms
def _axes(sections, interleaved):
    """Axis of every channel pair."""
    a, b, c = (int(x) for x in sections.split(","))
    if not interleaved:
        return [0] * a + [1] * b + [2] * c
    return [1 if i % 3 == 1 and i < 3 * b else 2 if i % 3 == 2 and i < 3 * c else 0 for i in range(a + b + c)]


def _turn_plain(y, positions, freq, sections, interleaved, inverse=False):
    """y [.., batch, heads, n, 128] fp32; angles in 64 bits, the products in 32."""
    if freq is None:
        return y
    half = freq.numel()
    axis = torch.tensor(_axes(sections, interleaved), device=y.device)
    angle = positions[axis].permute(1, 2, 0)[:, None].double() * freq        # [batch, 1, n, pairs]
    cos, sin = angle.cos().float(), angle.sin().float()
    if inverse:
        sin = -sin
    a, b, rest = y[..., :half], y[..., half:2 * half], y[..., 2 * half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _norm_plain(x, weight, *turn):
    y = x.float()
    y = y * (y.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.float()
    return _turn_plain(y, *turn).to(x.dtype)


def _norm_grad_plain(x, weight, up, *turn):
    u, y = _turn_plain(up.float(), *turn, True), x.float()
    r = (y.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = y * r
    wu = u * weight.float()
    grad = r * (wu - y * (y * wu).mean(-1, keepdim=True))
    return grad.to(x.dtype), (u * y).sum((0, 1, 2))


def _append_plain(c, layer, layers, k, v, new_len):
    """k, v [layers, batch, heads, n, 128]: the blocks that the new tokens touch, quantised from their raw tokens."""
    L, B, H, n, _ = k.shape
    P = c["codes"].shape[4]
    lens = c["seq_len"][layer:layer + layers].long()                          # [L, B]
    new = torch.full((B,), n, device=k.device) if new_len is None else new_len.long()
    r = lens % BLOCK
    nb = (BLOCK - 1 + n + BLOCK - 1) // BLOCK
    j = torch.arange(nb * BLOCK, device=k.device)
    src = torch.where(j < r[..., None], j, j - r[..., None] + BLOCK).clamp(max=BLOCK + n - 1)
    valid = j < (r + new)[..., None]                                          # [L, B, nb * 32]
    x = torch.cat([c["raw"][layer:layer + layers], torch.stack([k, v], 3)], 4)  # [L, B, H, 2, 32 + n, 128]
    x = x.gather(4, src[:, :, None, None, :, None].expand(L, B, H, 2, nb * BLOCK, D))
    f = (x.float() * valid[:, :, None, None, :, None]).view(L, B, H, 2, nb, BLOCK, D)
    scale = f.abs().amax((-1, -2)) / 127
    codes = torch.where(scale[..., None, None] > 0, f / scale[..., None, None], 0.0).round().clamp(-127, 127).to(torch.int8)
    at = lens - r                                                             # first token of the first block
    li, bi, ki = (valid.view(L, B, nb, BLOCK)[..., 0] & (new > 0)[:, None]).nonzero(as_tuple=True)
    pos = at[li, bi] + BLOCK * ki
    page, inside = c["table"][bi, pos // P].long(), pos % P // BLOCK
    c["codes"].view(*c["codes"].shape[:4], P // BLOCK, BLOCK, D)[li + layer, page, :, :, inside] = codes[li, bi, :, :, ki]
    c["scales"][li + layer, page, :, :, inside] = scale[li, bi, :, :, ki]
    last = (r + new) // BLOCK                                                 # the block that stays unfinished
    tail = torch.nn.functional.pad(x, (0, 0, 0, BLOCK)).view(L, B, H, 2, nb + 1, BLOCK, D)
    tail = tail.gather(4, last[:, :, None, None, None, None, None].expand(L, B, H, 2, 1, BLOCK, D))[:, :, :, :, 0]
    keep = torch.arange(BLOCK, device=k.device) < ((r + new) % BLOCK)[..., None]
    keep = keep & (new > 0)[None, :, None]
    c["raw"][layer:layer + layers] = torch.where(keep[:, :, None, None, :, None], tail, c["raw"][layer:layer + layers])
    c["seq_len"][layer:layer + layers] = (lens + new).int()


def _dense(c, layer, layers, width):
    """[layers, batch, heads, 2, width * page, 128] fp32: what the codes of the first `width` pages of every sequence stand for."""
    pages = c["table"][:, :width].clamp(min=0).long()
    codes, scales = c["codes"][layer:layer + layers, pages], c["scales"][layer:layer + layers, pages]  # [L, B, w, H, 2, ..]
    x = codes.unflatten(5, (-1, BLOCK)).float() * scales[..., None, None]
    L, B, w, H = x.shape[:4]
    return x.permute(0, 1, 3, 4, 2, 5, 6, 7).reshape(L, B, H, 2, -1, D)


def _mask_plain(c, layer, layers, n, q_len, T, window=None, sinks=0, seen=None):
    """[layers, batch, n, T]: tokens that a query sees, by a window or by the tree's bits."""
    lens = c["seq_len"][layer:layer + layers].long()[..., None, None]
    B, dev = lens.shape[1], lens.device
    nq = (torch.full((B,), n, device=dev) if q_len is None else q_len.long())[:, None, None]
    i, t = torch.arange(n, device=dev)[:, None], torch.arange(T, device=dev)
    base = lens - nq                                                          # token of the first query
    if seen is None:
        return (t <= base + i) & ((t < sinks) | (t > base + i - window)) & (i < nq)
    j = t - base                                                              # node of a token, [L, B, 1, T]
    node = j.clamp(0, n - 1).expand(lens.shape[0], B, n, T)
    bits = seen.expand(lens.shape[0], *seen.shape).gather(3, node >> 6) >> (node & 63) & 1
    return ((j < 0) | (bits == 1)) & (t < lens) & (i < nq)


def _attention_plain(c, layer, layers, q, q_len, tokens, **sight):
    L, B, Hq, n, _ = q.shape
    H, P = c["codes"].shape[2], c["codes"].shape[4]
    x = _dense(c, layer, layers, _pages_of(tokens, P))
    k, v = x[:, :, :, 0], x[:, :, :, 1]
    mask = _mask_plain(c, layer, layers, n, q_len, k.shape[-2], **sight)[:, :, None, None]
    s = q.float().view(L, B, H, Hq // H, n, D) @ k[:, :, :, None].transpose(-1, -2) * D ** -0.5
    s = s.masked_fill_(~mask, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    o = (p @ v[:, :, :, None]) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.view(L, B, Hq, n, D).to(q.dtype)


def _ancestors_plain(parents, q_len, words):
    """Bits and depths: a node has its parent's and its own."""
    B, n = parents.shape
    p = parents.long()
    up = torch.zeros(B, n, n, dtype=torch.bool, device=p.device)
    depth = torch.zeros(B, n, dtype=torch.int32, device=p.device)
    b = torch.arange(B, device=p.device)
    for i in range(n):
        a = p[:, i]
        up[:, i] = up[b, a.clamp(min=0)] & (a >= 0)[:, None]
        up[:, i, i] = True
        depth[:, i] = up[:, i].sum(-1) - 1
    there = torch.arange(n, device=p.device) < (n if q_len is None else q_len.long()[:, None])
    bits = torch.nn.functional.pad(up & there[..., None], (0, 64 * words - n)).view(B, n, words, 64).long()
    return (bits << torch.arange(64, device=p.device)).sum(-1), depth * there


def _slide_plain(c, window, sinks, dropped):
    P = c["codes"].shape[4]
    lens, width, pages = c["seq_len"].long().amin(0), c["table"].shape[1], c["refs"].numel()
    first = _pages_of(sinks, P)
    gone = ((lens - window + 1).clamp(min=0) // P - first).clamp(min=0)       # pages of each sequence
    j = torch.arange(width, device=lens.device)
    out = (j >= first) & (j < first + gone[:, None])
    rows = c["table"].long()
    left = torch.where(out & (rows >= 0), rows, pages).flatten()
    c["refs"] -= torch.bincount(left, minlength=pages + 1)[:pages].int()
    at = torch.where(j < first, j, j + gone[:, None])
    c["table"].copy_(torch.where(at < width, rows.gather(1, at.clamp(max=width - 1)), -1).int())
    c["seq_len"] -= (gone * P).int()
    dropped.copy_((gone * P).int())


def _fork_plain(c, src, dst):
    P, pages = c["codes"].shape[4], c["refs"].numel()
    src, dst = src.long(), dst.long()
    lens = c["seq_len"][:, src].long()
    full, used = lens.amin(0) // P, _pages_of(lens.amax(0), P)                # pages shared, pages holding anything
    j = torch.arange(c["table"].shape[1], device=src.device)
    shared, copied = j < full[:, None], (j >= full[:, None]) & (j < used[:, None])
    rows = c["table"][src].long()
    free = (c["refs"] == 0).nonzero().flatten()
    fresh = free[(copied.flatten().cumsum(0) - 1).clamp(min=0)].view_as(rows)
    c["table"][dst] = torch.where(shared, rows, torch.where(copied, fresh, -1)).int()
    c["refs"] += torch.bincount(torch.where(shared, rows, pages).flatten(), minlength=pages + 1)[:pages].int()
    a, b = rows[copied], fresh[copied]
    c["refs"][b] = 1
    for name in ("codes", "scales"):
        c[name][:, b] = c[name][:, a]
    c["raw"][:, dst] = c["raw"][:, src]
    c["seq_len"][:, dst] = c["seq_len"][:, src]


def _reserve_plain(c, cover):
    P = c["codes"].shape[4]
    j = torch.arange(c["table"].shape[1], device=cover.device)
    want = (j < ((cover.long() + P - 1) // P)[:, None]) & (c["table"] < 0)
    free = (c["refs"] == 0).nonzero().flatten()
    fresh = free[(want.flatten().cumsum(0) - 1).clamp(min=0)].view_as(c["table"])
    c["table"].copy_(torch.where(want, fresh.int(), c["table"]))
    c["refs"][fresh[want]] = 1


def _release_plain(c, ended):
    pages = c["refs"].numel()
    rows = c["table"][ended.long()].long()
    c["refs"] -= torch.bincount(torch.where(rows >= 0, rows, pages).flatten(), minlength=pages + 1)[:pages].int()
    c["table"][ended.long()] = -1
    c["seq_len"][:, ended.long()] = 0


# ------------------------------------------------------------------------------------------------ the library's calls
def _handle(s):
    """The cache as the library has it, over the state's buffers; made at a state's first pass, as a program makes it once."""
    from paper_2609_11582_b200 import binding as B
    if "handle" not in s:
        case = s["case"]
        s["handle"] = h = B.PagedCache(case["layers"], case["batch"], case["kv_heads"], case["q_heads"], page_tokens=case["page"],
                                       dtype=TYPES[case["dtype"]], buffers=s["cache"])
        s["workspace"] = torch.empty(B.paged_workspace_bytes(h, 1 if s["kind"] in ("stream", "speculate") else case["layers"], case.get("new", 1)),
                                     dtype=torch.uint8, device="cuda")
    return B, s["handle"]


def _rope_of(B, s, positions):
    if s["freq"] is None:
        return None
    sections = tuple(int(x) for x in _sections(s["case"]).split(","))
    return B.Rope(positions, s["freq"], sections, interleaved=s["case"].get("interleaved", True))


def _gather_path(k, path):
    """[layers, batch, heads, m, 128]: the accepted nodes' rows."""
    return k.gather(3, path[None, :, None, :, None].expand(k.shape[0], -1, k.shape[2], -1, D))


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case, kind = s["case"], s["kind"]
    if kind == "norm":
        turn = (s["positions"], s["freq"], case["sections"], case["interleaved"])
        if own:
            from paper_2609_11582_b200 import binding as B
            rope = _rope_of(B, s, s["positions"])
            B.norm_rope_apply(rope, s["q"], s["q_out"], s["q_weight"], s["k"], s["k_out"], s["k_weight"], eps=EPS)
            if not case["grad"]:
                return s["q_out"], s["k_out"]
            if "workspace" not in s:
                s["workspace"] = torch.empty(B.norm_rope_workspace_bytes(case["batch"], case["new"], case["q_heads"], case["kv_heads"]),
                                             dtype=torch.uint8, device="cuda")
            B.norm_rope_grad(rope, s["q"], s["q_up"], s["q_grad"], s["workspace"], s["q_weight"], s["q_weight_grad"],
                             s["k"], s["k_up"], s["k_grad"], s["k_weight"], s["k_weight_grad"], eps=EPS)
            return s["q_out"], s["k_out"], s["q_grad"], s["q_weight_grad"], s["k_grad"], s["k_weight_grad"]
        outs = [_norm_plain(s[n], s[n + "_weight"], *turn) for n in ("q", "k")]
        for n in ("q", "k") if case["grad"] else ():
            outs += _norm_grad_plain(s[n], s[n + "_weight"], s[n + "_up"], *turn)
        return tuple(outs)
    c = s["cache"]
    if kind == "window":
        if own:
            B, h = _handle(s)
            B.paged_attention_window(h, 0, case["layers"], s["q"], s["workspace"], s["out"], case["window"], case["sinks"], q_len=s["q_len"])
            return s["out"]
        return _attention_plain(c, 0, case["layers"], s["q"], s["q_len"], case["tokens"], window=case["window"], sinks=case["sinks"])
    if kind == "tree":
        if own:
            B, h = _handle(s)
            B.tree_ancestors(h, s["parents"], s["seen"], s["depth"], q_len=s["q_len"])
            B.paged_attention_tree(h, 0, case["layers"], s["q"], s["workspace"], s["out"], s["seen"], q_len=s["q_len"])
            return {"seen": s["seen"], "depth": s["depth"], "out": s["out"]}
        seen, depth = _ancestors_plain(s["parents"], s["q_len"], s["seen"].shape[2])
        return {"seen": seen, "depth": depth, "out": _attention_plain(c, 0, case["layers"], s["q"], s["q_len"], case["tokens"], seen=seen)}
    _restore(s)
    if kind == "slide":
        if own:
            B, h = _handle(s)
            B.pages_slide(h, case["window"], case["sinks"], s["dropped"])
        else:
            _slide_plain(c, case["window"], case["sinks"], s["dropped"])
        return {"table": c["table"], "refs": c["refs"], "seq_len": c["seq_len"], "dropped": s["dropped"]}
    L = case["layers"]
    if kind == "stream":
        window, sinks = case["window"], case["sinks"]
        if own:
            B, h = _handle(s)
            for i in range(case["steps"]):
                rope, k, v, q, out = _rope_of(B, s, s["positions"][i]), s["k"][i], s["v"][i], s["q"][i], s["out"][i]
                kt, qt = s["k_turned"][i], s["q_turned"][i]
                for l in range(L):
                    B.norm_rope_apply(rope, q[l], qt[l], s["q_weight"][l], k[l], kt[l], s["k_weight"][l], eps=EPS)
                    B.paged_append(h, l, 1, kt[l:l + 1], v[l:l + 1])
                    B.paged_attention_window(h, l, 1, qt[l:l + 1], s["workspace"], out[l:l + 1], window, sinks)
                B.pages_slide(h, window, sinks)
            return {"out": s["out"], "raw": c["raw"], "table": c["table"], "refs": c["refs"], "seq_len": c["seq_len"]}
        outs, dropped = [], torch.zeros(case["batch"], dtype=torch.int32, device="cuda")
        for i in range(case["steps"]):
            turn = (s["positions"][i], s["freq"], _sections(case), True)
            for l in range(L):
                q, k = (_norm_plain(s[n][i, l], s[n + "_weight"][l], *turn)[None] for n in ("q", "k"))
                _append_plain(c, l, 1, k, s["v"][i, l:l + 1], None)
                outs.append(_attention_plain(c, l, 1, q, None, c["table"].shape[1] * case["page"], window=window, sinks=sinks))
            _slide_plain(c, window, sinks, dropped)
        return {"out": torch.cat(outs).view_as(s["out"]), "raw": c["raw"], "table": c["table"], "refs": c["refs"], "seq_len": c["seq_len"]}
    S = case["batch"] // 2
    if own:
        B, h = _handle(s)
        B.pages_fork(h, s["src"], s["dst"], s["workspace"])
        B.pages_reserve(h, s["room"])
        B.tree_ancestors(h, s["parents"], s["seen"], s["depth"], q_len=s["q_len"])
        rope = _rope_of(B, s, (s["depth"] + s["start"][:, None])[None, S:].expand(3, S, case["new"]).contiguous())
        k, q, v, kt, qt = s["k"], s["q"], s["v"], s["k_turned"], s["q_turned"]
        for l in range(L):
            B.norm_rope_apply(rope, q[l, S:], qt[l, S:], s["q_weight"][l], k[l, S:], kt[l, S:], s["k_weight"][l], eps=EPS)
            B.paged_append(h, l, 1, kt[l:l + 1], v[l:l + 1], new_len=s["q_len"])
            B.paged_attention_tree(h, l, 1, qt[l:l + 1], s["workspace"], s["out"][l:l + 1], s["seen"], q_len=s["q_len"])
        B.pages_release(h, s["dst"])
        B.pages_reserve(h, s["room_after"])
        kt[:, :S].copy_(kt[:, S:])                       # (the accepted rows go to the first half, the originals)
        v = torch.cat([v[:, S:], v[:, S:]], 1)
        B.paged_append(h, 0, L, _gather_path(kt, s["path"]), _gather_path(v, s["path"]), new_len=s["taken"])
    else:
        _fork_plain(c, s["src"], s["dst"])
        _reserve_plain(c, s["room"])
        seen, depth = _ancestors_plain(s["parents"], s["q_len"], s["seen"].shape[2])
        s["seen"].copy_(seen)
        s["depth"].copy_(depth)
        turn = ((s["depth"] + s["start"][:, None])[None, S:].expand(3, S, case["new"]).contiguous(), s["freq"], _sections(case), True)
        keys, values = [], torch.cat([s["v"][:, S:], s["v"][:, S:]], 1)
        for l in range(L):
            q, k = (_norm_plain(s[n][l, S:], s[n + "_weight"][l], *turn).repeat(2, 1, 1, 1)[None] for n in ("q", "k"))
            keys.append(k)
            _append_plain(c, l, 1, k, values[l:l + 1], s["q_len"])
            out = _attention_plain(c, l, 1, q, s["q_len"], max(_lens(case)) + case["new"], seen=seen)
            s["out"][l, S:] = out[0, S:]
        _release_plain(c, s["dst"])
        _reserve_plain(c, s["room_after"])
        _append_plain(c, 0, L, _gather_path(torch.cat(keys), s["path"]), _gather_path(values, s["path"]), s["taken"])
    return {"out": s["out"], "seen": s["seen"], "depth": s["depth"], "raw": c["raw"][:, :S], "table": c["table"], "refs": c["refs"],
            "seq_len": c["seq_len"]}


# ------------------------------------------------------------------------------------------------ what it needs
def _seen_by_window(n, m, window, sinks):
    """(tokens that some query sees, pairs of a query and a token that it sees) of a sequence of n tokens and m queries"""
    pairs = 0
    for p in range(max(0, n - m), n):
        near = min(p + 1, window)
        pairs += near + min(sinks, p + 1 - near)
    if n <= 0 or m <= 0:
        return 0, 0
    first = max(0, max(0, n - m) - window + 1)
    return n - first + min(sinks, first), pairs


def work(case):
    kind, H, Hq, B = case["kind"], case["kv_heads"], case["q_heads"], case["batch"]
    size = 4 if case["dtype"] == "fp32" else 2
    if kind == "norm":
        rows = B * case["new"] * (H + Hq)
        return {"bytes": rows * (5.0 if case["grad"] else 2.0) * D * size + 12 * B * case["new"], "flops": rows * (22.0 if case["grad"] else 7.0) * D}
    L, P = case["layers"], case["page"]
    row = 2 * (D + 4 / BLOCK)                                 # codes and scales of a token of one head, both sides
    if kind in ("window", "tree"):
        lens, news = _lens(case), _news(case)
        if kind == "window":
            both = [_seen_by_window(n, m, case["window"], case["sinks"]) for n, m in zip(lens, news)]
        else:
            both = [(n if m else 0, m * (n - m) + m) for n, m in zip(lens, news)]   # (the sequence and the node itself: every tree's)
        return {"bytes": L * (H * row * sum(b[0] for b in both) + 4.0 * D * Hq * sum(news)), "flops": L * Hq * 4.0 * D * sum(b[1] for b in both)}
    if kind == "slide":
        width = _pages_of(max(_lens(case)), P)
        return {"bytes": 8.0 * B * width + 8.0 * L * B, "flops": 0.0}
    heads = Hq * 4.0 * D + H * (6.0 * D + row)                # queries there and back, keys there, back and in, values in, a token's codes
    if kind == "stream":
        rows = sum(_seen_by_window(case["tokens"] + i + 1, 1, case["window"], case["sinks"])[0] for i in range(case["steps"]))
        return {"bytes": L * B * (H * row * rows + case["steps"] * (heads + 4.0 * D * Hq)), "flops": L * B * Hq * 4.0 * D * rows}
    n, lens = case["new"], _lens(case)[:B // 2]
    pairs = sum(n * a + n for a in lens)
    return {"bytes": L * (H * row * sum(a + n for a in lens) + len(lens) * n * (heads + 4.0 * D * Hq)), "flops": L * Hq * 4.0 * D * pairs}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def _turn(x, positions, freq, sections, interleaved, sign):
    """Channels c and c + half as one complex number, times e^(i angle)."""
    if freq is None:
        return x
    a, b, c = (int(v) for v in sections.split(","))
    half = a + b + c
    angle = torch.empty(*positions.shape[1:], half, dtype=torch.float64, device=x.device)
    for i in range(half):
        axis = (0 if i < a else 1 if i < a + b else 2) if not interleaved else ((1 if i < 3 * b else 0) if i % 3 == 1 else (2 if i < 3 * c else 0) if i % 3 == 2 else 0)
        angle[..., i] = positions[axis].double() * freq[i]
    z = torch.complex(x[..., :half], x[..., half:2 * half]) * torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    return torch.cat([z.real, z.imag, x[..., 2 * half:]], -1)


def _normed(x, weight, *turn):
    x = x.double()
    return _turn(x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * weight.double(), *turn, 1)


def _normed_grad(x, weight, up, *turn):
    """By the norm's Jacobian: with s = mean(x^2) + eps, d(x_i s^-1/2)/dx_j = s^-1/2 (delta_ij - x_i x_j / (128 s))."""
    u, x = _turn(up.double(), *turn, -1), x.double()
    s = (x * x).sum(-1, keepdim=True) / D + EPS
    gw = (u * x / s.sqrt()).flatten(0, 2).sum(0)
    u = u * weight.double()
    return (u - x * ((x * u).sum(-1, keepdim=True) / (D * s))) / s.sqrt(), gw


def _exact_rows(old, new):
    """Values of a block sequence: `old` raw tokens of the unfinished block, then `new`; [rows, 128] in 64 bits, and the tail left raw."""
    x = torch.cat([old, new]).double()
    full = torch.zeros(_pages_of(x.shape[0], BLOCK) * BLOCK, D, dtype=torch.float64, device=x.device)
    full[:x.shape[0]] = x
    blocks = full.view(-1, BLOCK * D)
    step = blocks.abs().amax(1, keepdim=True) / 127
    # (the codes are those of the quotient by the stored step, which has 32 bits)
    codes = (blocks / torch.where(step > 0, step, 1.0).float().double()).round()
    return (codes * step).view(-1, D)[:x.shape[0]], x[x.shape[0] // BLOCK * BLOCK:]


def _exact_softmax(q, k, v, mask):
    """q [g, n, 128], k, v [T, 128] in 64 bits, mask [n, T]; rows that see nothing are zeros."""
    out = torch.zeros_like(q)
    for j in range(0, q.shape[1], 256):
        see = mask[j:j + 256]
        if not bool(see.any()):
            continue
        s = torch.einsum("gnd,td->gnt", q[:, j:j + 256], k) / math.sqrt(D)
        w = torch.softmax(s.masked_fill(~see, -math.inf), -1).nan_to_num(0.0)
        out[:, j:j + 256] = torch.einsum("gnt,td->gnd", w, v)
    return out


def _exact_values(c, l, row, h, n):
    """The first n tokens of a head, pages in `row`: [2, n, 128] in 64 bits."""
    P = c["codes"].shape[4]
    rows = [c["codes"][l, p, h].double() * c["scales"][l, p, h].double().repeat_interleave(BLOCK, -1)[..., None] for p in row[:_pages_of(n, P)]]
    return torch.cat(rows, 1)[:, :n] if rows else torch.zeros(2, 0, D, dtype=torch.float64, device="cuda")


def _exact_sight(n, m, window, sinks):
    """[m, n]: query i is token n - m + i"""
    t, p = torch.arange(n, device="cuda"), n - m + torch.arange(m, device="cuda")[:, None]
    return (t <= p) & ((p - t < window) | (t < sinks))


def _exact_tree(parents, n, m):
    """[m, n] from the parents of the first m nodes, the sequence's last m tokens."""
    see = torch.zeros(m, n, dtype=torch.bool)
    for i in range(m):
        if parents[i] >= 0:
            see[i] = see[parents[i]]
        see[i, :max(0, n - m)] = True
        see[i, n - m + i] = True
    return see.cuda()


def exact(case, seed):
    s = prepare(case, seed)
    kind, B, H, Hq = case["kind"], case["batch"], case["kv_heads"], case["q_heads"]
    G = Hq // H
    if kind == "norm":
        turn = (s["positions"], s["freq"], case["sections"], case["interleaved"])
        outs = [_normed(s[n], s[n + "_weight"], *turn) for n in ("q", "k")]
        for n in ("q", "k") if case["grad"] else ():
            outs += _normed_grad(s[n], s[n + "_weight"], s[n + "_up"], *turn)
        return tuple(outs)
    if kind == "slide":
        return None
    c, L, P, lens = s["cache"], case["layers"], case["page"], _lens(case)
    table = c["table"].tolist()
    if L * B * H > 1500:
        return None
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    if kind in ("window", "tree"):
        news = _news(case)
        if L * Hq * sum(a * b for a, b in zip(lens, news)) > 2e9:
            return None
        parents = _tree(case, seed) if kind == "tree" else None
        for b in range(B):
            m = news[b]
            if m == 0:
                continue
            see = _exact_tree(parents[b], lens[b], m) if parents else _exact_sight(lens[b], m, case["window"], case["sinks"])
            for l in range(L):
                for h in range(H):
                    k, v = _exact_values(c, l, table[b], h, lens[b])
                    out[l, b, h * G:h * G + G, :m] = _exact_softmax(s["q"][l, b, h * G:h * G + G, :m].double(), k, v, see)
        return {"seen": None, "depth": None, "out": out} if parents else out
    dt, raw = TYPES[case["dtype"]], s["raw0"].double()
    if kind == "stream":
        for l in range(L):
            q, k = ([_normed(s[n][i, l], s[n + "_weight"][l], s["positions"][i], s["freq"], _sections(case), True).to(dt) for i in range(case["steps"])] for n in ("q", "k"))
            for b in range(B):
                for h in range(H):
                    n, r = lens[b], lens[b] % BLOCK
                    kept = _exact_values(c, l, table[b], h, n)[:, :n - r]     # tokens of full blocks
                    tails = [s["raw0"][l, b, h, t, :r].clone() for t in (0, 1)]
                    for i in range(case["steps"]):
                        new = (k[i][b, h], s["v"][i, l, b, h])
                        tails = [torch.cat([tails[t], new[t]]) for t in (0, 1)]
                        now = [torch.cat([kept[t], _exact_rows(tails[t][:0], tails[t])[0]]) for t in (0, 1)]
                        n = now[0].shape[0]
                        out[i, l, b, h * G:h * G + G] = _exact_softmax(q[i][b, h * G:h * G + G].double(), *now, _exact_sight(n, 1, case["window"], case["sinks"]))
                        if tails[0].shape[0] == BLOCK:                        # (a full block leaves its slots as they were)
                            kept, tails = torch.stack(now), [x[:0] for x in tails]
                        for t in (0, 1):
                            raw[l, b, h, t, :tails[t].shape[0]] = tails[t].double()
                        first, last = _pages_of(case["sinks"], P), max(0, n - case["window"] + 1) // P
                        if last > first:
                            kept = torch.cat([kept[:, :first * P], kept[:, last * P:]], 1)
        return {"out": out, "raw": raw, "table": None, "refs": None, "seq_len": None}
    S, n = B // 2, case["new"]
    parents = _tree(case, seed)[S:]
    depths = []
    for p in parents:
        d = []
        for i in range(n):
            d.append(0 if p[i] < 0 else d[p[i]] + 1)
        depths.append(d)
    pos = (torch.tensor(depths, device="cuda") + torch.tensor(lens[:S], device="cuda")[:, None]).to(torch.int32)[None].expand(3, S, n)
    for l in range(L):
        q, k = (_normed(s[x][l, S:], s[x + "_weight"][l], pos, s["freq"], _sections(case), True).to(dt) for x in ("q", "k"))
        for b in range(S):
            a, r = lens[b], lens[b] % BLOCK
            see, path = _exact_tree(parents[b], a + n, n), _branch(parents[b], _accepted(case))
            whole = (r + len(path)) // BLOCK * BLOCK                         # tokens of the blocks that the branch fills
            for h in range(H):
                kept = _exact_values(c, l, table[b], h, a)
                sides = (k[b, h], s["v"][l, S + b, h])
                now = [torch.cat([kept[t][:a - r], _exact_rows(s["raw0"][l, b, h, t, :r], sides[t])[0]]) for t in (0, 1)]
                out[l, S + b, h * G:h * G + G] = _exact_softmax(q[b, h * G:h * G + G].double(), *now, see)
                for t in (0, 1):
                    tail = torch.cat([s["raw0"][l, b, h, t, :r], sides[t][path]])[whole:]
                    raw[l, b, h, t, :tail.shape[0]] = tail.double()
    return {"out": out, "seen": None, "depth": None, "raw": raw[:, :S], "table": None, "refs": None, "seq_len": None}
