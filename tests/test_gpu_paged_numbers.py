"""The 8-bit paged cache's attention where a number could lose its bits: values of very different sizes, tokens that take nearly all of the weight,
queries at the end of their type's range.  Against softmax attention in 64 bits, each kernel by its own bound.  Rotary positions near and
far, by a bound that goes with the angle.  Tokens taken back."""
import random

import numpy as np
import pytest
import torch

from oracle import okq_paged_oracle as O
from paper_2609_11582_b200 import binding as B
from tests.test_gpu_paged import BF16, BLOCK, D, F16, F32, SECTIONS, Model, f64, gen, randn

pytestmark = pytest.mark.gpu
TILE = 128


def kernel_bound(w, v, ref, amax, top, dtype, plan):
    """What rows of an output may be off by; w [.., rows, tokens] their weights, v [.., tokens, 128] the tokens' values, amax [.., tokens] the largest
    magnitude of a token's block (127 times its scale), top [.., rows] a row's largest |score|.
    Scores carry three roundings of fp32 and the exponent one more, in a numerator and in the sum: 8 * 2^-24 |s|; exponentials, factors and
    sums at most 32 * 2^-24.  Of that the weighted magnitudes sum w |v|.
    Decode kernel: a tile's numerators, weight times scale, are whole multiples of 2^-30 of the largest of its 128 or less; half of that
    times a code of 127 for each of 128 tokens: 2^-24 of the largest w * amax of the tile.
    Prompt kernel: fp16, half a step is 2^-12, and twice that with the sums that round towards it; below fp16's normal numbers half a step of
    2^-24, where the largest of a step's 64 numerators is 2^-6 at least: 64 * 2^-19 = 2^-13 of the largest w * amax of the step.  Numerators
    that lie 2^-68 below the row's largest, all of its tokens.  Blocks with a scale below 2^-112 count as zeros, values up to 127 * 2^-112."""
    mag = w @ v.abs()
    step, part = (TILE // 2, 2.0 ** -13) if plan == B.PLAN_PROMPT else (TILE, 2.0 ** -24)
    most = [x.amax(-1) for x in (w * amax[..., None, :]).split(step, -1)]
    most = sum(most) + (w.shape[-1] * 2.0 ** -68 / part * torch.stack(most).amax(0) if plan == B.PLAN_PROMPT else 0)
    err = (2.0 ** -24 * (8 * top[..., None] + 32) + (2.0 ** -11 if plan == B.PLAN_PROMPT else 0)) * mag + part * most[..., None]
    err = err + (127 * 2.0 ** -112 if plan == B.PLAN_PROMPT else 0)
    return err + torch.finfo(dtype).eps / 2 * (ref.abs() + err) + (2.0 ** -25 if dtype == F16 else 1e-38)


class Store:
    """A cache of one layer that holds given keys and values [batch, H, tokens, 128] (fp32, on the GPU), quantised here."""

    def __init__(self, k, v, Hq, wide, dtype=BF16, page=64, seed=0):
        batch, H, T, _ = k.shape
        self.T, self.H, self.Hq, self.dtype = T, H, Hq, dtype
        width = (T + page - 1) // page
        c = self.c = B.PagedCache(1, batch, H, Hq, batch * width + 2, (1 << 19) // page if wide else width, page, dtype)
        table = torch.randperm(batch * width + 2, generator=gen(seed))[:batch * width].view(batch, width).cuda()
        c.table[:, :width] = table.int()
        c.seq_len.fill_(T)
        x = torch.zeros(batch, H, 2, width * page, D, device="cuda")
        x[:, :, 0, :T], x[:, :, 1, :T] = k, v
        x = x.unflatten(3, (width, page // BLOCK, BLOCK))                       # [batch, H, 2, width, blocks, 32, 128]
        scales = x.abs().amax((-1, -2)) / 127
        codes = (x / torch.where(scales > 0, scales, 1.0)[..., None, None]).round().clamp(-127, 127)
        c.codes[0, table] = codes.permute(0, 3, 1, 2, 4, 5, 6).flatten(4, 5).to(torch.int8)
        c.scales[0, table] = scales.permute(0, 3, 1, 2, 4)
        self.held = (codes.double() * scales.double()[..., None, None]).flatten(3, 5)[..., :T, :]
        self.amax = (scales.double() * 127).repeat_interleave(BLOCK, -1).flatten(3, 4)[:, :, 1, :T]

    def attend(self, q, sm_scale=None):
        """One call, each row against its kernel's bound.  q [1, batch, Hq, n, 128]."""
        n, G, scale = q.shape[3], self.Hq // self.H, D ** -0.5 if sm_scale is None else sm_scale
        plan, q = B.paged_plan(self.c, 1, n), q.cuda()
        out = torch.full_like(q, 7.0)
        ws = torch.empty(B.paged_workspace_bytes(self.c, 1, n), dtype=torch.uint8, device="cuda")
        B.paged_attention(self.c, 0, 1, q, ws, out, sm_scale=sm_scale)
        late = torch.arange(self.T, device="cuda") > (self.T - n + torch.arange(n, device="cuda"))[:, None]
        for b in range(q.shape[1]):
            k, v = self.held[b, :, 0], self.held[b, :, 1]                       # [H, T, 128]
            s = torch.einsum("hgnd,htd->hgnt", q[0, b].double().unflatten(0, (self.H, G)), k) * scale
            top = s.masked_fill(late, 0.0).abs().amax(-1).flatten(1)
            w = torch.softmax(s.masked_fill(late, -torch.inf), -1).nan_to_num(0.0).flatten(1, 2)
            ref, got = w @ v, out[0, b].double().unflatten(0, (self.H, G)).flatten(1, 2)
            limit = kernel_bound(w, v, ref, self.amax[b], top, self.dtype, plan)
            assert ((got - ref).abs() <= limit).all(), (b, plan, ((got - ref).abs() / limit).max().item())
        assert self.c.device_status() == 0
        return plan


# (queries, batch, KV heads, query heads, tokens, wide table), so that a range of tiles has several: the prompt kernel with two streams of rows, with
# both streams on the same rows, and a few long items; the decode kernel's line, and its clusters
PROMPT = [(150, 6, 8, 16, 2500, True), (20, 12, 8, 16, 2500, True), (5, 1, 2, 16, 60000, True)]
LINE = [(1, 24, 8, 56, 2500, True), (3, 24, 8, 40, 2500, True)]
CLUSTER = [(1, 1, 3, 21, 8000, False), (8, 1, 1, 2, 8000, False)]
DECODE = LINE + CLUSTER
ALL = PROMPT + DECODE


def steered(n, batch, H, Hq, T, wide, seed=0, spread=1.0):
    """Queries whose first channel is 16 in all rows, keys whose first channel is 0: a key with x there scores 1.414 x more."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q, k, v = (torch.randn(*s, D, generator=g, device="cuda") for s in ((1, batch, Hq, n), (batch, H, T), (batch, H, T)))
    q *= spread
    q[..., 0], k[..., 0] = 16.0, 0.0
    return q.to(BF16), k, v * 0.3


def lift(natural):
    return natural / (16.0 * D ** -0.5)


def test_shapes_reach_their_kernels():
    for shapes, want in ((PROMPT, lambda p: p == B.PLAN_PROMPT), (LINE, lambda p: p == B.PLAN_LINE), (CLUSTER, lambda p: p > 0)):
        for n, batch, H, Hq, T, wide in shapes:
            assert want(B.paged_plan(B.PagedCache(1, batch, H, Hq, 8, (1 << 13) if wide else (T + 63) // 64), 1, n)), (n, batch, H, Hq, T, wide)


@pytest.mark.parametrize("size", [1e-4, 1e-6, 1e-9, 1e-20])
@pytest.mark.parametrize("zeros", [128, 300, 1000])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_small_values_behind_zeros(shape, zeros, size):
    """Tokens without any value first, as padding has it, then values far below 1."""
    q, k, v = steered(*shape, seed=1)
    v *= size
    v[..., :zeros, :] = 0
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("size", [1e4, 1e9])
@pytest.mark.parametrize("at", [0, 1280])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_large_values_without_weight(shape, at, size):
    """A tile of huge values whose tokens nobody looks at, first or in the middle."""
    q, k, v = steered(*shape, seed=2, spread=2.0)
    v[..., at:at + 128, :] *= size
    k[..., at:at + 128, 0] = lift(-90.0)
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("fall", [1, -1])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_values_of_all_sizes(shape, fall):
    """Values that fall, or rise, by 2^40 over the sequence, while the scores do the opposite."""
    q, k, v = steered(*shape, seed=9)
    t = torch.arange(shape[4], device="cuda") / shape[4]
    v *= torch.exp2(-40.0 * fall * t)[:, None]
    k[..., 0] = lift(40.0 * 0.6931) * fall * t
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("size", [2.0 ** -7, 2.0 ** -20])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_small_values_in_the_tiles_of_large_ones(shape, size):
    """Every other block of 32 tokens has values far below its neighbours', and all of the weight."""
    q, k, v = steered(*shape, seed=3, spread=2.0)
    large = torch.arange(shape[4], device="cuda") // BLOCK % 2 == 0
    v[..., ~large, :] *= size
    k[..., large, 0] = lift(-90.0)
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("above", [8.0, 16.0, 20.0, 26.0])
@pytest.mark.parametrize("at", [0, 700, 2200])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_sinks(shape, at, above):
    """A token far above the rest without any value, in a tile of small values: the others' numerators keep their bits."""
    q, k, v = steered(*shape, seed=4)
    first = at - at % TILE
    v[..., first:first + TILE, :] *= 2.0 ** -30
    v[..., at, :] = 0
    k[..., at, 0] = lift(above)
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("shape", ALL, ids=str)
def test_sinks_of_all_heights(shape):
    """Several of them, up and down: nothing overflows."""
    q, k, v = steered(*shape, seed=5)
    for at, above in ((0, 30.0), (300, 60.0), (640, 20.0), (900, 85.0), (1500, 10.0), (2000, 90.0)):
        k[..., at, 0] = lift(above)
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("size", [1e-8, 1e-20, 1e-30])
@pytest.mark.parametrize("above", [20.0, 40.0])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_small_values_behind_sinks(shape, above, size):
    """Both at once: sums that have grown large by the one, and are to be brought down by the other."""
    q, k, v = steered(*shape, seed=10)
    v *= size
    v[..., :TILE, :] = 0
    k[..., 5, 0] = lift(above)
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("rise", [0.0, 60.0, 110.0])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_scores_fall_without_end(shape, rise):
    """Scores that fall by 2^200 over the sequence, step by step, and values that rise: the first tokens have all of the weight, and the sums
    of the last ones overflow nothing."""
    q, k, v = steered(*shape, seed=11)
    t = torch.arange(shape[4], device="cuda") / shape[4]
    v *= torch.exp2(rise * t)[:, None]
    k[..., 0] = lift(200.0 * 0.6931) * (1 - t)
    Store(k, v, shape[3], shape[5]).attend(q)


@pytest.mark.parametrize("score", [1e3, 1e6, 2e7, 1e8, 1e9, 1e12])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_scores_of_all_sizes(shape, score):
    """One token whose score is so far above the others', which are 0, that the output is its value: scores beyond 2^24 have no digits behind the point.
    The rounding of the value alone is left: its code times its scale in fp32 (three roundings and those of a sum of one), 2^-20 relative, or
    the prompt kernel's numerator in fp16, 2^-11; then the output's."""
    n, batch, H, Hq, T, wide = shape
    q, k, v = steered(*shape, seed=12)
    q[..., 1:], k[..., 1:] = 0.0, 0.0
    at = T - n - 300
    k[..., at, 0] = score / (16.0 * D ** -0.5)
    v *= 0.01
    s = Store(k, v, Hq, wide)
    ws = torch.empty(B.paged_workspace_bytes(s.c, 1, n), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0)
    B.paged_attention(s.c, 0, 1, q, ws, out)
    want = s.held[:, :, 1, at].repeat_interleave(Hq // H, 1)[:, :, None]
    rel = 2.0 ** -11 if B.paged_plan(s.c, 1, n) == B.PLAN_PROMPT else 2.0 ** -20
    assert ((out[0].double() - want).abs() <= (rel + torch.finfo(BF16).eps / 2 * (1 + rel)) * want.abs()).all()


@pytest.mark.parametrize("fall", [4, 20, 60])
@pytest.mark.parametrize("n,batch,H,Hq", [(150, 6, 2, 14), (128, 20, 4, 4), (26, 40, 2, 2), (700, 2, 2, 4)])
def test_rows_that_see_small_values_only(n, batch, H, Hq, fall):
    """Prompts whose values grow from block to block: early rows see none of the large ones, which lie in the same tile."""
    q, k, v = steered(n, batch, H, Hq, n, True, seed=13)
    v *= torch.exp2(fall * (torch.arange(n, device="cuda") // BLOCK % 4 - 2.0))[:, None]
    Store(k, v, Hq, True).attend(q)


@pytest.mark.parametrize("lifts,zero", [((0, 20, 40, 0, 20), (1, 2, 4)), ((0, 0, 40, 0, 20), (1, 2, 4)), ((0, 30, 0, 0, 0), (1,)), ((40, 0, 0, 0, 40), (0, 4)),
                                        ((20, 20, 20, 0, 0), (0, 1, 2)), ((0, 20, 40, 0, 20), (2,))], ids=str)
@pytest.mark.parametrize("n,batch,H,Hq", [(150, 6, 2, 14), (150, 20, 2, 2), (26, 40, 2, 2)])
def test_blocks_without_value_and_all_of_the_weight(n, batch, H, Hq, lifts, zero):
    q, k, v = steered(n, batch, H, Hq, 150, True, seed=14, spread=3.0)
    block = torch.arange(150, device="cuda") // BLOCK
    k[..., 0] = torch.tensor(lifts, device="cuda")[block] * lift(1.0)
    for z in zero:
        v[..., block == z, :] = 0
    Store(k, v, Hq, True).attend(q)


@pytest.mark.parametrize("seed", range(12))
def test_mixtures(seed):
    """Forty calls each of random shapes: heads, groups, pages, queries, lengths, scores with a long tail, in steps, drifting or with a few dominant
    tokens, blocks of values up to 2^30 apart on either side (2^6 in fp16), blocks and dominant tokens without value."""
    rng = random.Random(seed)
    for _ in range(40):
        H, G, batch, n = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 5, 7, 8]), rng.choice([1, 1, 2, 6, 12]), rng.choice([1, 1, 2, 3, 5, 8, 20, 33, 70, 150, 300])
        T, dtype, wide = max(n, rng.choice([1, 31, 33, 100, 128, 129, 700, 2500, 2501])), rng.choice([F16, BF16]), rng.random() < 0.5
        q, k, v = steered(n, batch, H, H * G, T, wide, seed=rng.randrange(1 << 30), spread=rng.choice([0.3, 1.0, 3.0]))
        g = torch.Generator(device="cuda")
        g.manual_seed(rng.randrange(1 << 30))
        uniform = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
        above, kind = lift(rng.choice([5.0, 15.0, 30.0, 40.0])), rng.choice(["even", "tail", "steps", "drift", "few"])
        if kind == "tail":
            k[..., 0] = above * uniform(batch, H, T) ** 8
        elif kind == "steps":
            k[..., 0] = above * (torch.arange(T, device="cuda") // rng.choice([32, 64, 100, 500]) % 3) / 2
        elif kind == "drift":
            k[..., 0] = (above / 30 * (uniform(batch, H, T) - 0.5) * 3.5).cumsum(-1)
        elif kind == "few":
            k[..., 0] = above * (uniform(batch, H, T) > 1 - 3 / T)
        blocks = (T + BLOCK - 1) // BLOCK
        spread = rng.choice([0, 0, 2, 6] if dtype == F16 else [0, 2, 10, 30])
        by_token = lambda x: x.repeat_interleave(BLOCK, -1)[..., :T]  # noqa: E731
        v *= by_token(torch.exp2((uniform(batch, H, blocks) * 2 - 1) * spread))[..., None]
        if rng.random() < 0.3:
            v[by_token(uniform(batch, H, blocks) < 0.3)] = 0
        if rng.random() < 0.3:
            v[k[..., 0] > k[..., 0].amax() - lift(3.0)] = 0
        Store(k, v, H * G, wide, dtype, rng.choice([32, 64, 128, 256])).attend(q.to(dtype))


@pytest.mark.parametrize("largest", [5e37, 1e38, 3e38, float(torch.finfo(BF16).max)])
@pytest.mark.parametrize("shape", ALL, ids=str)
def test_queries_at_the_end_of_their_range(shape, largest):
    q, k, v = steered(*shape, seed=6)
    q = (q.float() / q.float().abs().amax(-1, keepdim=True) * largest).to(BF16)
    assert q.isfinite().all()
    Store(k * 2.0 ** -60, v, shape[3], shape[5]).attend(q, sm_scale=float(np.float32(2.0 ** 61 / largest)))


# Rows of several tiles of eight that the decode kernel takes (more than eight rows of a head, by its clusters or its line): here its own
# bound holds, not the prompt kernel's.
@pytest.mark.parametrize("H,Hq,n,tokens,wide", [(1, 1, 13, 2000, False), (1, 1, 13, 2000, True), (1, 7, 3, 900, False), (2, 8, 40, 500, False), (1, 8, 24, 900, False),
                                                (4, 28, 2, 1300, True), (1, 8, 2, 1700, True), (1, 1, 16, 1000, True), (1, 3, 8, 3000, False), (1, 8, 100, 130, False)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_many_rows_in_the_decode_kernel(H, Hq, n, tokens, wide, dtype):
    g = gen(7)
    k, v = randn(g, 1, H, tokens, D, dtype=F32).cuda(), randn(g, 1, H, tokens, D, dtype=F32).cuda()
    assert Store(k, v, Hq, wide, dtype).attend(randn(g, 1, 1, Hq, n, D, dtype=dtype)) != B.PLAN_PROMPT


# ------------------------------------------------------------------------------------------------ rotary positions
def turn_bound(x, ref, angle, half, dtype):
    """Cosine and sine are off by 2^-22 + |angle| 2^-51 at most: two units of fp32 of sincospi (2^-23), the angle's fraction of a turn rounded to
    fp32 (2^-25), its reduction in 64 bits (two roundings of 2^-53 and the constant's, relative to the angle).  The product and the sum
    round once each (2^-24 of |a| + |b|), the result to its type."""
    mag = np.abs(x)
    inner = np.zeros_like(mag)
    inner[..., :half] = inner[..., half:2 * half] = (mag[..., :half] + mag[..., half:2 * half]) * (2.0 ** -22 + 2.0 ** -23 + np.abs(angle) * 2.0 ** -51)
    tiny = {F16: 2.0 ** -25, BF16: 0.0, F32: 0.0}[dtype]
    return inner + (0 if dtype == F32 else torch.finfo(dtype).eps / 2 * (np.abs(ref) + inner)) + tiny


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("sections,interleaved", SECTIONS)
def test_rope_error_by_position(dtype, sections, interleaved):
    """From the nearest positions to the last ones, and where a sine is next to nothing (multiples of pi: 103993, 833719, 1146408)."""
    half = sum(sections)
    p = torch.tensor([0, 1, 2, 3, 22, 355, 710, 4095, 32767, 103993, 208341, 312689, 833719, 1146408, 16777217, 2 ** 30 + 1, 2 ** 31 - 1, -355, -2 ** 31 + 1])
    pos = p.int().expand(3, 1, -1).contiguous()
    x = randn(gen(8), 1, 4, len(p), D, dtype=dtype).cuda()
    for freq in (B.rope_frequencies(1e6, half, "cpu"), torch.ones(half, dtype=torch.float64)):
        out = torch.empty_like(x)
        B.rope_apply(B.Rope(pos.cuda(), freq.cuda(), sections, interleaved), x, out)
        ref = O.rope(f64(x), pos.numpy(), freq.numpy(), sections, interleaved)
        angle = p.double().numpy()[:, None] * freq.numpy()[None]
        assert (np.abs(f64(out) - ref) <= turn_bound(f64(x), ref, angle[None, None], half, dtype)).all()


# ------------------------------------------------------------------------------------------------ tokens taken back
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("held,draft,kept", [(62, 5, 1), (95, 7, 0), (31, 40, 3), (64, 5, 2), (50, 5, 4)])
def test_drafts_on_a_fork(dtype, held, draft, kept):
    """Drafted tokens across the end of a block, checked on a fork, given up with it, and the accepted ones appended to the original: the cache is
    as if the others had never been there."""
    m = Model(2, 3, 2, 6, max_pages=3, page=64, dtype=dtype, n_pages=12)
    m.c.table.fill_(-1)
    m.c.refs.zero_()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    ws = torch.empty(max(B.paged_workspace_bytes(m.c, 2, n) for n in (1, draft)), dtype=torch.uint8, device="cuda")
    B.pages_reserve(m.c, i32(held, 0, 20))
    m.append(held, [held, 0, 20])
    k, v = (randn(m.g, 2, 3, 2, draft, D, dtype=dtype) for _ in range(2))
    B.pages_fork(m.c, i32(0), i32(1), ws)
    for l in range(2):
        m.tok[l][1] = [list(t) for t in m.tok[l][0]]
    B.pages_reserve(m.c, i32(0, held + draft, 0))
    m.append(draft, [0, draft, 0], k=k, v=v)
    m.check()
    m.attend(draft, q_len=[0, draft, 0], workspace=ws)
    B.pages_release(m.c, i32(1))
    for l in range(2):
        m.tok[l][1] = [[torch.zeros(0, D, dtype=dtype)] * 2 for _ in range(2)]
    B.pages_reserve(m.c, i32(held + kept, 0, 0))
    k[:, 0], v[:, 0] = k[:, 1], v[:, 1]
    m.append(draft, [kept, 0, 0], k=k, v=v)
    m.check()
    m.attend(1, workspace=ws)
    assert m.c.device_status() == 0


def test_codes_after_a_take_back():
    """Tokens of the unfinished block given back: its codes keep the scale of all of them until the next append, which leaves what the remaining
    and the new ones alone would have."""
    m = Model(1, 1, 1, 1, max_pages=2, page=32, dtype=BF16, seed=9)
    k, v = randn(m.g, 1, 1, 1, 20, D, dtype=BF16), randn(m.g, 1, 1, 1, 20, D, dtype=BF16)
    k[:, :, :, 12:] *= 8
    m.append(20, k=k, v=v)
    before = m.c.codes.clone(), m.c.scales.clone()
    m.c.seq_len -= 8
    m.tok[0][0][0] = [t[:12] for t in m.tok[0][0][0]]
    B.paged_append(m.c, 0, 1, k[:, :, :, :1].cuda(), v[:, :, :, :1].cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert torch.equal(m.c.codes, before[0]) and torch.equal(m.c.scales, before[1])   # (no new token: nothing is written)
    m.append(1)
    m.check()
