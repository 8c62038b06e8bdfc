"""The operators of the 8-bit paged cache, as cases that can be timed and compared with their plain forms.

Every case is a dict of plain values; its "kind" names the part of a user's program it stands for:

  rope       rotary positions with three axes (time, height, width) on the queries and keys of a layer; with "grad" forwards and,
             for the gradients, backwards
  append     keys and values of new tokens into the cache (quantised in blocks of 32 tokens and one head), then read back
  attention  one call over a cache that is already full: one query per sequence, a few (drafted tokens), or a prompt's
  generate   a model's inner loop: per new token and layer the append (keys rotated on the way) and the attention (queries rotated
             on the way), from the same prompt each pass
  fork       a prompt shared by several sequences, room for their own tokens, and the end of some of them
  compact    the pages in use moved to the front of the pool

`run` computes them in elementary torch operations while `own` is false and with the library's calls where it is true.  Shapes are those of
the repository's workloads: 28 query and 4 key/value heads at 28 layers, 32 and 4 at 48; two-second chunks of 350 tokens.
"""
from __future__ import annotations

import math

import torch

own = False

D, BLOCK = 128, 32
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the smallest call: one new token of eight sequences, between a layer's projections and its attention
        {"name": "rope step", "kind": "rope", "dtype": "fp16", "batch": 8, "new": 1, "q_heads": 28, "kv_heads": 4,
         "sections": "16,24,24", "interleaved": False, "heads_inner": True, "grad": False, "start": 16384},
        # training on a long recording, odd length, far positions: forwards and backwards in fp32, interleaved axes
        {"name": "rope train", "kind": "rope", "dtype": "fp32", "batch": 1, "new": 8191, "q_heads": 32, "kv_heads": 4,
         "sections": "24,20,20", "interleaved": True, "heads_inner": True, "grad": True, "start": 1000003},
        # a prompt of 4097 tokens into all layers of an empty cache
        {"name": "append prompt", "kind": "append", "dtype": "fp16", "layers": 28, "batch": 1, "q_heads": 28, "kv_heads": 4,
         "held": 0, "new": 4097, "ragged": False, "page": 64, "rope": False},
        # pieces of different lengths appended to sequences of different lengths, keys rotated on the way
        {"name": "append ragged", "kind": "append", "dtype": "bf16", "layers": 1, "batch": 16, "q_heads": 28, "kv_heads": 4,
         "held": 1357, "new": 350, "ragged": True, "page": 32, "rope": True},
        # the smallest attention: one sequence, one key/value head with seven query heads, a context of a few seconds
        {"name": "attention tiny", "kind": "attention", "dtype": "fp16", "layers": 1, "batch": 1, "q_heads": 7, "kv_heads": 1,
         "tokens": 2048, "new": 1, "ragged": False, "page": 64},
        # one long recording
        {"name": "attention long", "kind": "attention", "dtype": "bf16", "layers": 1, "batch": 1, "q_heads": 28, "kv_heads": 4,
         "tokens": 131072, "new": 1, "ragged": False, "page": 64},
        # a layer of the largest decode shape: 16 sequences of 32k tokens
        {"name": "attention batch", "kind": "attention", "dtype": "fp16", "layers": 1, "batch": 16, "q_heads": 32, "kv_heads": 4,
         "tokens": 32768, "new": 1, "ragged": False, "page": 128},
        # drafted tokens checked: up to five queries per sequence, sequences of all lengths (one empty, one of a single token)
        {"name": "attention draft", "kind": "attention", "dtype": "fp16", "layers": 1, "batch": 16, "q_heads": 28, "kv_heads": 4,
         "tokens": 12345, "new": 5, "ragged": True, "page": 32},
        # a prompt's second piece: 2048 queries behind 6144 tokens that the cache holds already
        {"name": "attention prompt", "kind": "attention", "dtype": "bf16", "layers": 1, "batch": 1, "q_heads": 28, "kv_heads": 4,
         "tokens": 8192, "new": 2048, "ragged": False, "page": 64},
        # a model generating: append and attention layer by layer
        {"name": "generate", "kind": "generate", "dtype": "fp16", "layers": 28, "batch": 4, "q_heads": 28, "kv_heads": 4,
         "tokens": 4090, "steps": 4, "page": 64},
        # eight continuations of one prompt, three of them given up
        {"name": "pages fork", "kind": "fork", "dtype": "fp16", "layers": 28, "batch": 16, "q_heads": 28, "kv_heads": 4,
         "tokens": 8001, "copies": 8, "room": 512, "page": 64},
        # a pool after hours of serving, half of its pages free, made fit for handing back its end
        {"name": "pages compact", "kind": "compact", "dtype": "fp16", "layers": 28, "batch": 64, "q_heads": 28, "kv_heads": 4,
         "pages": 640, "page": 64},
    ]


MOST_ROPE = 36 * 8191 * 4            # elements / 128 x bytes of the largest listed case
MOST_APPEND = 28 * 4 * 4097          # token-heads
MOST_DECODE = 16 * 4 * 32768
MOST_SCORES = 28 * 2048 * 8192       # query heads x queries x keys
MOST_GENERATE = 28 * 4 * 4 * 4096
MOST_POOL = 28 * 4 * 64 * 640


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(lo * (max(hi, lo) / lo) ** rng.random()))))


def _heads(rng):
    kv, group = rng.choice([(1, 7), (2, 8), (4, 7), (4, 8), (4, 5), (8, 4), (8, 1), (3, 2)])
    return {"q_heads": kv * group, "kv_heads": kv}


def _half(rng):
    return {"dtype": rng.choice(["fp16", "bf16"]), "page": rng.choice([32, 64, 128, 256])}


def draw(rng):
    kind = rng.choice(["rope"] * 3 + ["append"] * 3 + ["attention"] * 7 + ["generate", "fork", "compact"])
    if kind == "rope":
        c = {"kind": kind, "dtype": rng.choice(["fp16", "bf16", "fp32"]), "batch": _log(rng, 1, 32), **_heads(rng)}
        top = MOST_ROPE // ((c["q_heads"] + c["kv_heads"]) * c["batch"] * 4)
        sections, interleaved = rng.choice([("16,24,24", False), ("24,20,20", True), ("64,0,0", False), ("16,8,8", False), ("12,10,10", True)])
        return {**c, "new": _log(rng, 1, top), "sections": sections, "interleaved": interleaved, "heads_inner": rng.random() < 0.5,
                "grad": rng.random() < 0.5, "start": _log(rng, 1, 2000000)}
    if kind == "append":
        c = {"kind": kind, "layers": rng.choice([1, 1, 28]), "batch": _log(rng, 1, 32), **_heads(rng), **_half(rng)}
        top = MOST_APPEND // (c["layers"] * c["batch"] * c["kv_heads"])
        new = _log(rng, 1, min(8192, top))
        return {**c, "held": _log(rng, 1, max(1, min(4096, top - new))) - 1, "new": new, "ragged": rng.random() < 0.5, "rope": rng.random() < 0.5}
    if kind == "attention":
        c = {"kind": kind, "layers": rng.choice([1, 1, 1, rng.randint(2, 28)]), "batch": _log(rng, 1, 64), **_heads(rng), **_half(rng)}
        form = rng.choice(["one", "one", "few", "prompt"])
        new = 1 if form == "one" else rng.randint(2, 16) if form == "few" else _log(rng, 17, 2048)
        top = MOST_DECODE // (c["layers"] * c["batch"] * c["kv_heads"])
        if new > 1:
            top = min(top, MOST_SCORES // (c["layers"] * c["batch"] * c["q_heads"] * new))
        tokens = _log(rng, 1, max(1, min(131072, top)))
        return {**c, "tokens": tokens, "new": min(new, tokens), "ragged": rng.random() < 0.4}
    if kind == "generate":
        c = {"kind": kind, "layers": rng.randint(1, 28), "batch": _log(rng, 1, 16), **_heads(rng), **_half(rng)}
        top = MOST_GENERATE // (c["layers"] * c["batch"] * c["kv_heads"])
        return {**c, "tokens": _log(rng, 1, max(1, min(16384, top - 4))), "steps": rng.randint(1, 4)}
    c = {"kind": kind, "layers": rng.choice([1, 28]), **_heads(rng), **_half(rng)}
    pages = MOST_POOL // (c["layers"] * c["kv_heads"] * c["page"])
    if kind == "fork":
        copies = rng.randint(1, 16)
        room = _log(rng, 1, 512)
        per = pages // 2 - 2 * (copies + 1) * (room // c["page"] + 2)
        return {**c, "batch": copies + rng.randint(1, 8), "tokens": _log(rng, 1, max(2, min(32768, per * c["page"]))), "copies": copies, "room": room}
    c["pages"] = _log(rng, 16, min(4096, max(17, pages)))
    return {**c, "batch": _log(rng, 2, min(64, c["pages"]))}


# ------------------------------------------------------------------------------------------------ sizes of a case
def _lens(case, top):
    """Tokens of each sequence: all alike, or of all lengths with an empty one and one of a single token among them."""
    if not case.get("ragged"):
        return [top] * case["batch"]
    return [top if b == 0 else 0 if b == 1 else min(1, top) if b == 2 else top * ((37 * b) % 64 + 1) // 64 for b in range(case["batch"])]


def _news(case):
    """New tokens or queries of each sequence."""
    if not case.get("ragged"):
        return [case["new"]] * case["batch"]
    return [case["new"] - (b * 29) % case["new"] if b != 3 else 0 for b in range(case["batch"])]


def _pages_of(tokens, page):
    return (tokens + page - 1) // page


def _fork_pages(case):
    """(pages of the pool, entries of a table row)"""
    width = _pages_of(case["tokens"] + case["room"], case["page"]) + 1
    return width * 2 + (case["copies"] + 1) * (case["room"] // case["page"] + 3), width


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + 20260911)
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


def _frequencies(case):
    """float64 [pairs]: theta^(-2 c / rotary channels)"""
    half = sum(int(x) for x in case.get("sections", "16,24,24").split(","))
    return 1000000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)


def _heads_in(case, x):
    """The same numbers as a projection [batch, token, head * 128] leaves them."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if case["heads_inner"] else x


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


def prepare(case, seed):
    g, kind, dt = _gen(seed), case["kind"], TYPES[case["dtype"]]
    H, Hq, B = case["kv_heads"], case["q_heads"], case["batch"]
    s = {"case": case, "kind": kind}
    if kind == "rope":
        n = case["new"]
        s["positions"], s["freq"] = _positions(B, n, case["start"]), _frequencies(case)
        for name, heads in (("q", Hq), ("k", H)):
            s[name] = _heads_in(case, _randn(g, B, heads, n, D).to(dt))
            s[name + "_out"] = torch.empty_like(s[name])
            if case["grad"]:
                s[name + "_up"] = _heads_in(case, _randn(g, B, heads, n, D).to(dt))
                s[name + "_grad"] = torch.empty_like(s[name])
        return s
    L, P = case["layers"], case["page"]
    if kind in ("append", "generate"):
        steps = case.get("steps", 0)
        lens = [case["tokens"]] * B if kind == "generate" else _lens(case, case["held"])
        news = [steps] * B if kind == "generate" else _news(case)
        width = max(_pages_of(a + b, P) for a, b in zip(lens, news)) + 1
        s["cache"] = c = _store(case, g, sum(_pages_of(a + b, P) for a, b in zip(lens, news)) + 2, width, lens, news)
        s["len0"], s["raw0"] = c["seq_len"].clone(), c["raw"].clone()
        n = steps if kind == "generate" else case["new"]
        s["freq"] = _frequencies(case)
        if kind == "append":
            s["positions"] = _positions(B, n, case["held"])
            s["k"] = _fill(torch.empty(L, B, H, n, D, device="cuda"), g).to(dt)
            s["v"] = (_randn(g, L, B, H, n, D) * 0.3).to(dt)
            s["new_len"] = torch.tensor(news, dtype=torch.int32, device="cuda") if case["ragged"] else None
            s["begin"] = min(lens) // BLOCK * BLOCK
            m = max(a + b for a, b in zip(lens, news)) - s["begin"]
        else:
            # (positions of every step in a tensor of its own, as a program that advances them has)
            s["positions"] = [_positions(B, 1, case["tokens"] + i) for i in range(n)]
            s["k"] = _randn(g, n, L, B, H, 1, D).to(dt)
            s["v"] = (_randn(g, n, L, B, H, 1, D) * 0.3).to(dt)
            s["q"] = _randn(g, n, L, B, Hq, 1, D).to(dt)
            s["out"] = torch.zeros(n, L, B, Hq, 1, D, dtype=dt, device="cuda")
            s["begin"] = case["tokens"] // BLOCK * BLOCK
            m = case["tokens"] + n - s["begin"]
        s["k_back"], s["v_back"] = (torch.zeros(L, B, H, m, D, dtype=dt, device="cuda") for _ in range(2))
    elif kind == "attention":
        lens = _lens(case, case["tokens"])
        s["cache"] = _store(case, g, sum(_pages_of(n, P) for n in lens) + 2, _pages_of(max(lens), P), lens, [0] * B)
        s["q"] = _randn(g, L, B, Hq, case["new"], D).to(dt)
        s["out"] = torch.zeros(L, B, Hq, case["new"], D, dtype=dt, device="cuda")
        s["q_len"] = torch.tensor(_news(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    elif kind == "fork":
        pages, width = _fork_pages(case)
        s["cache"] = c = _store(case, g, pages, width, [case["tokens"]] + [0] * (B - 1), [0] * B)
        s["src"] = torch.zeros(case["copies"], dtype=torch.int32, device="cuda")
        s["dst"] = torch.randperm(B - 1, generator=g, device="cuda")[:case["copies"]].to(torch.int32) + 1
        cover = torch.zeros(B, dtype=torch.int32, device="cuda")
        cover[s["dst"].long()] = case["tokens"] + case["room"]
        s["cover"] = cover
        s["ended"] = s["dst"][: (case["copies"] + 1) // 3].contiguous()
    else:
        # three quarters of the sequences of a full pool have ended
        pages = case["pages"]
        width = _pages_of(2 * pages, B)
        lens = [min(width * P, max(1, (pages // B) * P - (7 * b) % P)) for b in range(B)]
        s["cache"] = c = _store(case, g, pages, width, lens, [0] * B)
        gone = torch.rand(B, generator=g, device="cuda") < 0.5
        j = c["table"]
        ended = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
        ended[torch.where(gone[:, None] & (j >= 0), j, pages).long().flatten()] = True
        c["refs"][ended[:pages]] = 0
        c["table"][gone] = -1
        c["seq_len"][:, gone] = 0
        s["n_live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if kind in ("fork", "compact"):
        s["table0"], s["refs0"], s["len0"], s["raw0"] = (c[n].clone() for n in ("table", "refs", "seq_len", "raw"))
    return s


def _restore(s):
    """The prompt's state before the pass."""
    for name, kept in (("table", "table0"), ("refs", "refs0"), ("seq_len", "len0"), ("raw", "raw0")):
        if kept in s:
            s["cache"][name].copy_(s[kept])


# ------------------------------------------------------------------------------------------------ plain forms
def _axes(sections, interleaved):
    """Axis of every channel pair."""
    a, b, c = (int(x) for x in sections.split(","))
    if not interleaved:
        return [0] * a + [1] * b + [2] * c
    return [1 if i % 3 == 1 and i < 3 * b else 2 if i % 3 == 2 and i < 3 * c else 0 for i in range(a + b + c)]


def _rope_plain(x, positions, freq, sections="16,24,24", interleaved=False, inverse=False):
    """x [.., batch, heads, n, 128]; angles in 64 bits, the products in 32."""
    half = freq.numel()
    axis = torch.tensor(_axes(sections, interleaved), device=x.device)
    angle = positions[axis].permute(1, 2, 0)[:, None].double() * freq        # [batch, 1, n, pairs]
    cos, sin = angle.cos().float(), angle.sin().float()
    if inverse:
        sin = -sin
    a, b, rest = x[..., :half].float(), x[..., half:2 * half].float(), x[..., 2 * half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1).to(x.dtype)


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
    tail = x.view(L, B, H, 2, nb, BLOCK, D).gather(4, last.clamp(max=nb - 1)[:, :, None, None, None, None, None].expand(L, B, H, 2, 1, BLOCK, D))[:, :, :, :, 0]
    keep = torch.arange(BLOCK, device=k.device) < ((r + new) % BLOCK)[..., None]
    c["raw"][layer:layer + layers] = torch.where(keep[:, :, None, None, :, None], tail, c["raw"][layer:layer + layers])
    c["seq_len"][layer:layer + layers] = (lens + new).int()


def _dense(c, layer, layers, width):
    """[layers, batch, heads, 2, width * page, 128] fp32: what the codes of the first `width` pages of every sequence stand for."""
    pages = c["table"][:, :width].clamp(min=0).long()
    codes, scales = c["codes"][layer:layer + layers, pages], c["scales"][layer:layer + layers, pages]  # [L, B, w, H, 2, ..]
    x = codes.unflatten(5, (-1, BLOCK)).float() * scales[..., None, None]
    L, B, w, H = x.shape[:4]
    return x.permute(0, 1, 3, 4, 2, 5, 6, 7).reshape(L, B, H, 2, -1, D)


def _read_plain(c, begin, n, dtype):
    P = c["codes"].shape[4]
    first = begin // P
    x = _dense({**c, "table": c["table"][:, first:]}, 0, c["codes"].shape[0], _pages_of(begin + n, P) - first)
    x = x[..., begin - first * P:begin - first * P + n, :]
    held = begin + torch.arange(n, device=x.device) < c["seq_len"][..., None]
    x = (x * held[:, :, None, None, :, None]).to(dtype)
    return x[:, :, :, 0], x[:, :, :, 1]


def _attention_plain(c, layer, layers, q, q_len, tokens):
    L, B, Hq, n, _ = q.shape
    H, P = c["codes"].shape[2], c["codes"].shape[4]
    x = _dense(c, layer, layers, _pages_of(tokens, P))
    k, v = x[:, :, :, 0], x[:, :, :, 1]
    lens = c["seq_len"][layer:layer + layers].long()
    nq = torch.full((B,), n, device=q.device) if q_len is None else q_len.long()
    i = torch.arange(n, device=q.device)
    sees = lens[..., None] - nq[:, None] + i + 1                              # [L, B, n] keys that a query sees
    mask = torch.arange(k.shape[-2], device=q.device) < sees[..., None]
    mask = mask[:, :, None, None]
    s = q.float().view(L, B, H, Hq // H, n, D) @ k[:, :, :, None].transpose(-1, -2) * D ** -0.5
    s = s.masked_fill_(~mask, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    o = (p @ v[:, :, :, None]) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.view(L, B, Hq, n, D).to(q.dtype)
    return torch.where((i < nq[:, None])[None, :, None, :, None], o, torch.zeros_like(o))


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


def _compact_plain(c, n_live):
    live = c["refs"] > 0
    n = live.sum()
    i = torch.arange(live.numel(), device=live.device)
    holes, movers = (~live & (i < n)).nonzero().flatten(), (live & (i >= n)).nonzero().flatten()
    to = i.clone()
    to[movers] = holes
    for name in ("codes", "scales"):
        c[name][:, holes] = c[name][:, movers]
    c["refs"][holes] = c["refs"][movers]
    c["refs"][movers] = 0
    c["table"].copy_(torch.where(c["table"] >= 0, to[c["table"].clamp(min=0).long()].int(), -1))
    n_live.copy_(n.int())


# ------------------------------------------------------------------------------------------------ the library's calls
def _handle(s):
    """The cache as the library has it, over the state's buffers; made at a state's first pass, as a program makes it once."""
    from paper_2609_11582_b200 import binding as B
    if "handle" not in s:
        case = s["case"]
        s["handle"] = h = B.PagedCache(case["layers"], case["batch"], case["kv_heads"], case["q_heads"], page_tokens=case["page"],
                                       dtype=TYPES[case["dtype"]], buffers=s["cache"])
        s["workspace"] = torch.empty(B.paged_workspace_bytes(h, 1 if s["kind"] == "generate" else case["layers"], case.get("new", 1)),
                                     dtype=torch.uint8, device="cuda")
    return B, s["handle"]


def _rope_of(B, s, positions):
    case = s["case"]
    sections = tuple(int(x) for x in case.get("sections", "16,24,24").split(","))
    return B.Rope(positions, s["freq"], sections, interleaved=case.get("interleaved", False))


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case, kind = s["case"], s["kind"]
    if kind == "rope":
        how = {"sections": case["sections"], "interleaved": case["interleaved"]}
        if own:
            from paper_2609_11582_b200 import binding as B
            rope = _rope_of(B, s, s["positions"])
            B.rope_apply(rope, s["q"], s["q_out"], s["k"], s["k_out"])
            if not case["grad"]:
                return s["q_out"], s["k_out"]
            B.rope_apply(rope, s["q_up"], s["q_grad"], s["k_up"], s["k_grad"], inverse=True)
            return s["q_out"], s["k_out"], s["q_grad"], s["k_grad"]
        outs = [_rope_plain(s[n], s["positions"], s["freq"], **how) for n in ("q", "k")]
        if case["grad"]:
            outs += [_rope_plain(s[n], s["positions"], s["freq"], inverse=True, **how) for n in ("q_up", "k_up")]
        return tuple(outs)
    c = s["cache"]
    if kind == "append":
        _restore(s)
        if own:
            B, h = _handle(s)
            B.paged_append(h, 0, case["layers"], s["k"], s["v"], new_len=s["new_len"], rope=_rope_of(B, s, s["positions"]) if case["rope"] else None)
            B.paged_read(h, 0, case["layers"], s["begin"], s["k_back"], s["v_back"])
            return {"k": s["k_back"], "v": s["v_back"], "raw": c["raw"], "seq_len": c["seq_len"]}
        k = _rope_plain(s["k"], s["positions"], s["freq"]) if case["rope"] else s["k"]
        _append_plain(c, 0, case["layers"], k, s["v"], s["new_len"])
        k, v = _read_plain(c, s["begin"], s["k_back"].shape[3], s["k"].dtype)
        return {"k": k, "v": v, "raw": c["raw"], "seq_len": c["seq_len"]}
    if kind == "attention":
        if own:
            B, h = _handle(s)
            B.paged_attention(h, 0, case["layers"], s["q"], s["workspace"], s["out"], q_len=s["q_len"])
            return s["out"]
        return _attention_plain(c, 0, case["layers"], s["q"], s["q_len"], case["tokens"])
    if kind == "generate":
        _restore(s)
        if own:
            B, h = _handle(s)
            for i in range(case["steps"]):
                rope, k, v, q, out = _rope_of(B, s, s["positions"][i]), s["k"][i], s["v"][i], s["q"][i], s["out"][i]
                for l in range(case["layers"]):
                    B.paged_append(h, l, 1, k[l:l + 1], v[l:l + 1], rope=rope)
                    B.paged_attention(h, l, 1, q[l:l + 1], s["workspace"], out[l:l + 1], rope=rope)
            B.paged_read(h, 0, case["layers"], s["begin"], s["k_back"], s["v_back"])
            return {"out": s["out"], "k": s["k_back"], "v": s["v_back"], "raw": c["raw"], "seq_len": c["seq_len"]}
        outs = []
        for i in range(case["steps"]):
            k, q = (_rope_plain(s[n][i], s["positions"][i], s["freq"]) for n in ("k", "q"))
            for l in range(case["layers"]):
                _append_plain(c, l, 1, k[l:l + 1], s["v"][i, l:l + 1], None)
                outs.append(_attention_plain(c, l, 1, q[l:l + 1], None, case["tokens"] + i + 1))
        k, v = _read_plain(c, s["begin"], s["k_back"].shape[3], s["k"].dtype)
        return {"out": torch.cat(outs).view_as(s["out"]), "k": k, "v": v, "raw": c["raw"], "seq_len": c["seq_len"]}
    _restore(s)
    if kind == "fork":
        if own:
            B, h = _handle(s)
            B.pages_fork(h, s["src"], s["dst"], s["workspace"])
            B.pages_reserve(h, s["cover"])
            B.pages_release(h, s["ended"])
        else:
            _fork_plain(c, s["src"], s["dst"])
            _reserve_plain(c, s["cover"])
            _release_plain(c, s["ended"])
        return dict(c)
    if own:
        B, h = _handle(s)
        B.pages_compact(h, s["workspace"], s["n_live"])
    else:
        _compact_plain(c, s["n_live"])
    return {**c, "n_live": s["n_live"]}


# ------------------------------------------------------------------------------------------------ what it needs
def work(case):
    kind, H, Hq, B = case["kind"], case["kv_heads"], case["q_heads"], case["batch"]
    size = 4 if case["dtype"] == "fp32" else 2
    if kind == "rope":
        rows = B * case["new"] * (H + Hq) * (2 if case["grad"] else 1)
        half = sum(int(x) for x in case["sections"].split(","))
        return {"bytes": rows * 2.0 * D * size + 12 * B * case["new"], "flops": rows * 6.0 * half}
    L, P = case["layers"], case["page"]
    row = 2 * (D + 4 / BLOCK)                                 # codes and scales of a token of one head, both sides
    if kind == "append":
        lens, news = _lens(case, case["held"]), _news(case)
        begin = min(lens) // BLOCK * BLOCK
        new, back = sum(news), sum(max(0, a + b - begin) for a, b in zip(lens, news))
        return {"bytes": L * H * (new * (4 * D + row) + back * (row + 4 * D)), "flops": L * H * (new * 8.0 * D + back * 2 * D)}
    if kind == "attention":
        lens, news = _lens(case, case["tokens"]), _news(case)
        seen = sum(sum(max(0, n - m + i + 1) for i in range(m)) for n, m in zip(lens, news))
        return {"bytes": L * (H * row * sum(n for n, m in zip(lens, news) if m) + 4.0 * D * Hq * sum(news)), "flops": L * Hq * 4.0 * D * seen}
    if kind == "generate":
        rows = case["steps"] * case["tokens"] + case["steps"] * (case["steps"] + 1) // 2
        return {"bytes": L * B * (H * row * rows + case["steps"] * (4.0 * D * Hq + H * (4 * D + row))), "flops": L * B * Hq * 4.0 * D * rows}
    page = L * H * P * row
    if kind == "fork":
        moved = case["copies"] if case["tokens"] % P else 0
        return {"bytes": 2.0 * moved * page + 2.0 * case["copies"] * L * H * 2 * BLOCK * D * 2, "flops": 0.0}
    return {"bytes": 2.0 * page * max(1, case["pages"] // 4), "flops": 0.0}      # half of the pages live, half of those behind the front


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def _turn(x, positions, freq, sections, interleaved, sign):
    """Channels c and c + half as one complex number, times e^(i angle)."""
    a, b, c = (int(v) for v in sections.split(","))
    half = a + b + c
    angle = torch.empty(*positions.shape[1:], half, dtype=torch.float64, device=x.device)
    for i in range(half):
        axis = (0 if i < a else 1 if i < a + b else 2) if not interleaved else ((1 if i < 3 * b else 0) if i % 3 == 1 else (2 if i < 3 * c else 0) if i % 3 == 2 else 0)
        angle[..., i] = positions[axis].double() * freq[i]
    z = torch.complex(x[..., :half].double(), x[..., half:2 * half].double()) * torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    return torch.cat([z.real, z.imag, x[..., 2 * half:].double()], -1)


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


def _exact_softmax(q, k, v, first):
    """q [g, n, 128], k, v [T, 128] in 64 bits; query j sees the keys up to first + j."""
    out = torch.zeros_like(q)
    for j in range(0, q.shape[1], 256):
        n = min(256, q.shape[1] - j)
        seen = max(0, min(k.shape[0], first + j + n))
        if seen == 0:
            continue
        s = torch.einsum("gnd,td->gnt", q[:, j:j + n], k[:seen]) / math.sqrt(D)
        late = torch.arange(seen, device=q.device)[None, :] > first + j + torch.arange(n, device=q.device)[:, None]
        w = torch.softmax(s.masked_fill(late, -math.inf), -1).nan_to_num(0.0)
        out[:, j:j + n] = torch.einsum("gnt,td->gnd", w, v[:seen])
    return out


def _exact_values(c, l, b, h, n):
    """The first n tokens of a sequence and head: [2, n, 128] in 64 bits."""
    P = c["codes"].shape[4]
    pages = [int(p) for p in c["table"][b, :_pages_of(n, P)].tolist()]
    rows = [c["codes"][l, p, h].double() * c["scales"][l, p, h].double().repeat_interleave(BLOCK, -1)[..., None] for p in pages]
    return torch.cat(rows, 1)[:, :n] if rows else torch.zeros(2, 0, D, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    kind, B, H, Hq = case["kind"], case["batch"], case["kv_heads"], case["q_heads"]
    G = Hq // H
    how = (s.get("freq"), case.get("sections", "16,24,24"), case.get("interleaved", False))
    if kind == "rope":
        outs = [_turn(s[n], s["positions"], *how, 1) for n in ("q", "k")]
        return tuple(outs + [_turn(s[n], s["positions"], *how, -1) for n in ("q_up", "k_up")] if case["grad"] else outs)
    c, L, P = s["cache"], case["layers"], case["page"]
    if kind == "attention":
        news, lens = _news(case), _lens(case, case["tokens"])
        if L * B * H > 1500 or L * Hq * sum(a * b for a, b in zip(lens, news)) > 2e9:
            return None
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    k, v = _exact_values(c, l, b, h, lens[b])
                    m = news[b]
                    out[l, b, h * G:h * G + G, :m] = _exact_softmax(s["q"][l, b, h * G:h * G + G, :m].double(), k, v, lens[b] - m)
        return out
    if kind in ("append", "generate"):
        if L * B * H > 1500:
            return None
        news = [case["steps"]] * B if kind == "generate" else _news(case)
        lens = [case["tokens"]] * B if kind == "generate" else _lens(case, case["held"])
        dt, begin = TYPES[case["dtype"]], s["begin"]
        k_back, v_back = torch.zeros(s["k_back"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["v_back"].shape, dtype=torch.float64, device="cuda")
        raw, out = s["raw0"].double(), torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda") if kind == "generate" else None
        if kind == "generate":
            pos = torch.cat(s["positions"], 2)
            keys = s["k"].squeeze(-2).permute(1, 2, 3, 0, 4)                 # [L, B, H, n, 128]
            values, queries = s["v"].squeeze(-2).permute(1, 2, 3, 0, 4), s["q"].squeeze(-2).permute(1, 2, 3, 0, 4)
            keys, queries = (torch.stack([_turn(x[l], pos, *how, 1) for l in range(L)]).to(dt) for x in (keys, queries))
        else:
            keys, values = s["k"], s["v"]
            if case["rope"]:
                keys = torch.stack([_turn(keys[l], s["positions"], *how, 1) for l in range(L)]).to(dt)
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    n, m, r = lens[b], news[b], lens[b] % BLOCK
                    kept = _exact_values(c, l, b, h, n)
                    sides = [keys[l, b, h, :m], values[l, b, h, :m]]
                    for i in range(1, m + 1 if kind == "generate" else 1):   # the cache after each step
                        now = [torch.cat([kept[t][:n - r], _exact_rows(s["raw0"][l, b, h, t, :r], sides[t][:i])[0]]) for t in (0, 1)]
                        out[i - 1, l, b, h * G:h * G + G] = _exact_softmax(queries[l, b, h * G:h * G + G, i - 1:i].double(), *now, n + i - 1)
                        for t in (0, 1):                                     # raw tokens of the block unfinished at that step
                            tail = _exact_rows(s["raw0"][l, b, h, t, :r], sides[t][:i])[1]
                            raw[l, b, h, t, :tail.shape[0]] = tail
                    for t, back in ((0, k_back), (1, v_back)):
                        rows, tail = _exact_rows(s["raw0"][l, b, h, t, :r], sides[t])
                        whole = torch.cat([kept[t][:n - r], rows]) if m else kept[t]
                        back[l, b, h, :max(0, n + m - begin)] = whole[begin:]
                        if m:
                            raw[l, b, h, t, :tail.shape[0]] = tail
        got = {"k": k_back, "v": v_back, "raw": raw, "seq_len": None}
        return {**got, "out": out} if kind == "generate" else got
    # pages: the codes are moved as they are and compared as whole numbers; the floating outputs are the scales and the raw tokens
    table, refs, lens = s["table0"].tolist(), s["refs0"].tolist(), s["len0"][0].tolist()
    scales, raw = c["scales"].double(), s["raw0"].double()
    if kind == "fork":
        free = [p for p, n in enumerate(refs) if n == 0]
        n = lens[0]
        for d in s["dst"].tolist():
            raw[:, d] = raw[:, 0]
            if n % P:
                scales[:, free.pop(0)] = scales[:, table[0][n // P]]
    else:
        n = sum(r > 0 for r in refs)
        holes = [p for p in range(n) if refs[p] == 0]
        movers = [p for p in range(n, len(refs)) if refs[p] > 0]
        for a, b in zip(movers, holes):
            scales[:, b] = scales[:, a]
    got = {"codes": None, "scales": scales, "raw": raw, "table": None, "refs": None, "seq_len": None}
    return got if kind == "fork" else {**got, "n_live": None}
