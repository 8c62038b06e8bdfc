"""The 8-bit paged cache and the rotary positions on the GPU against the oracle in 64 bits."""
import threading

import numpy as np
import pytest
import torch

from oracle import okq_paged_oracle as O
from paper_2609_11582_b200 import binding as B

pytestmark = pytest.mark.gpu
D, BLOCK = 128, 32
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F16, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def f64(x):
    return x.detach().cpu().double().numpy()


# ------------------------------------------------------------------------------------------------ rotary positions
SECTIONS = [((16, 24, 24), False), ((24, 20, 20), True), ((64, 0, 0), False), ((8, 8, 8), False), ((12, 10, 10), True), ((0, 8, 0), False),
            ((8, 0, 0), True)]


def positions(g, batch, n, kind):
    p = torch.randint(0, 5000, (3, batch, n), generator=g, dtype=torch.int32)
    if kind == "far":
        p = p + 1_900_000_000
    elif kind == "negative":
        p = -p
    elif kind == "zero":
        p = p * 0
    return p


def rope_bound(x, ref, half, dtype):
    """Cos and sin to two units of fp32 (2^-22) and half a unit of their angle (2^-24), rounding of one product and of the sum (2^-24
    each): 6 * 2^-24 (|a| + |b|); the angle itself, 1e-6 for positions near 2^31 (2^-53 relative of up to 2e9 radians is 2e-7,
    twice); the result's own rounding."""
    mag = np.abs(x)
    pair = np.zeros_like(mag)
    pair[..., :half] = pair[..., half:2 * half] = mag[..., :half] + mag[..., half:2 * half]
    eps = torch.finfo(dtype).eps / 2
    tiny = {F16: 2.0 ** -25, BF16: 0.0, F32: 0.0}[dtype]
    inner = (6 * 2.0 ** -24 + 1e-6) * pair
    return inner + (0 if dtype == F32 else eps * (np.abs(ref) + inner)) + tiny


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("sections,interleaved", SECTIONS)
def test_rope_matches_the_formula(dtype, sections, interleaved):
    g = gen(1)
    half = sum(sections)
    freq = B.rope_frequencies(1e6, half, "cpu")
    for batch, hq, hk, n, kind, inner in ((1, 7, 1, 1, "near", True), (3, 4, 2, 37, "far", False), (2, 1, 0, 130, "negative", True), (2, 3, 3, 5, "zero", True)):
        pos = positions(g, batch, n, kind)
        rope = B.Rope(pos.cuda(), freq.cuda(), sections, interleaved)
        def tensor(h):
            x = randn(g, batch, n, h, D, dtype=dtype) if inner else randn(g, batch, h, n, D, dtype=dtype)
            return (x.cuda().transpose(1, 2) if inner else x.cuda())
        q, k = tensor(hq), tensor(hk) if hk else None
        for inverse in (False, True):
            qo, ko = torch.empty_like(q), None if k is None else torch.empty_like(k)
            B.rope_apply(rope, q, qo, k, ko, inverse=inverse)
            for x, y in ((q, qo), (k, ko)):
                if x is None:
                    continue
                x64 = f64(x)
                ref = O.rope(x64, pos.numpy(), freq.numpy(), sections, interleaved, inverse)
                assert (np.abs(f64(y) - ref) <= rope_bound(x64, ref, half, dtype)).all()
                assert torch.equal(y[..., 2 * half:], x[..., 2 * half:])
        if kind == "zero":
            assert torch.equal(qo, q)


def test_rope_in_place_and_strided():
    g = gen(2)
    freq = B.rope_frequencies(1e4, 64)
    pos = positions(g, 2, 19, "near").cuda()
    rope = B.Rope(pos, freq, (16, 24, 24))
    # q and k inside one projection [batch, n, (q heads | k heads | v heads) * 128]
    qkv = randn(g, 2, 19, 9, D, dtype=BF16).cuda()
    q, k = qkv[:, :, :5].transpose(1, 2), qkv[:, :, 5:7].transpose(1, 2)
    want_q, want_k, v = torch.empty_like(q), torch.empty_like(k), qkv[:, :, 7:].clone()
    B.rope_apply(rope, q, want_q, k, want_k)
    B.rope_apply(rope, q, q, k, k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(qkv[:, :, 7:], v)


def test_rope_rows_at_odd_multiples_of_16_bytes():
    g = gen(4)
    pos = positions(g, 2, 19, "near").cuda()
    rope = B.Rope(pos, B.rope_frequencies(1e4, 64), (16, 24, 24))
    for dtype, off in ((F32, 4), (BF16, 8), (F16, 8)):
        q, out = (randn(g, 2, 3, 19, D + off, dtype=dtype).cuda()[..., off:] for _ in range(2))
        want, behind = torch.empty_like(q.contiguous()), out._base[..., :off].clone()
        B.rope_apply(rope, q.contiguous(), want)
        B.rope_apply(rope, q, out)
        assert torch.equal(out, want) and torch.equal(out._base[..., :off], behind)


@pytest.mark.parametrize("sections,interleaved", SECTIONS[:2])
def test_rope_gradient(sections, interleaved):
    """The inverse is the gradient of the formula's 64-bit form, and agrees with differences of the call itself."""
    g = gen(3)
    freq = B.rope_frequencies(1e6, 64, "cpu")
    pos = positions(g, 2, 11, "near")
    rope = B.Rope(pos.cuda(), freq.cuda(), sections, interleaved)
    x, up, d = (randn(g, 2, 3, 11, D, dtype=F32).cuda() for _ in range(3))
    grad = torch.empty_like(x)
    B.rope_apply(rope, up, grad, inverse=True)
    xx = x.cpu().double().requires_grad_()
    axes = O.rope_axes(sections, interleaved)
    angle = torch.stack([pos[a].double() * freq[i] for i, a in enumerate(axes)], -1)[:, None]
    a, b = xx[..., :64], xx[..., 64:]
    y = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)
    y.backward(up.cpu().double())
    ref = xx.grad.numpy()
    assert (np.abs(f64(grad) - ref) <= rope_bound(f64(up), ref, 64, F32)).all()
    plus, minus = torch.empty_like(x), torch.empty_like(x)
    B.rope_apply(rope, x + 0.5 * d, plus)
    B.rope_apply(rope, x - 0.5 * d, minus)
    diff, inner = (f64(up) * (f64(plus) - f64(minus))).sum(), (f64(grad) * f64(d)).sum()
    # the map is linear: what is left are roundings of 2^-22 per number, of random signs
    assert abs(diff - inner) <= 2.0 ** -22 * np.abs(f64(up)).sum() * 4


# ------------------------------------------------------------------------------------------------ a cache and what it should hold
class Model:
    """A cache and every token appended to it, as the call was given it.  `wide`: the table has room for 2^19 tokens of each sequence, so
    that the rule of sizes does not take an item for a short one."""

    def __init__(self, L, batch, H, Hq, max_pages, page, dtype, n_pages=None, seed=0, wide=False):
        n_pages = n_pages or batch * max_pages + 3
        self.c = B.PagedCache(L, batch, H, Hq, n_pages, (1 << 19) // page if wide else max_pages, page, dtype)
        self.L, self.B, self.H, self.Hq, self.page, self.dtype = L, batch, H, Hq, page, dtype
        self.c.codes.random_(-127, 128)      # what is not written is not zero
        self.c.scales.normal_()
        self.c.raw.normal_()
        self.tok = [[[[torch.zeros(0, D, dtype=dtype)] * 2 for _ in range(H)] for _ in range(batch)] for _ in range(L)]
        self.g = gen(seed + 100)
        # pages in an order of their own
        order = torch.randperm(n_pages, generator=self.g).int()[:batch * max_pages]
        self.c.table[:, :max_pages] = order.view(batch, max_pages).cuda()
        self.c.refs[order.long()] = 1

    def lens(self, l=0):
        return [self.tok[l][b][0][0].shape[0] for b in range(self.B)]

    def append(self, n, new_len=None, layers=None, k=None, v=None, rope=None):
        l0, lc = layers or (0, self.L)
        k = randn(self.g, lc, self.B, self.H, n, D, dtype=self.dtype) if k is None else k
        v = randn(self.g, lc, self.B, self.H, n, D, dtype=self.dtype, scale=0.3) if v is None else v
        nl = None if new_len is None else torch.tensor(new_len, dtype=torch.int32).cuda()
        B.paged_append(self.c, l0, lc, k.cuda(), v.cuda(), nl, rope)
        kk = k
        if rope is not None:
            kk = torch.stack([k[i] for i in range(lc)]).cuda()
            for i in range(lc):
                B.rope_apply(rope, kk[i], kk[i])
            kk = kk.cpu()
        for i in range(lc):
            for b in range(self.B):
                m = n if new_len is None else max(0, min(n, new_len[b]))
                for h in range(self.H):
                    t = self.tok[l0 + i][b][h]
                    self.tok[l0 + i][b][h] = [torch.cat([t[0], kk[i, b, h, :m]]), torch.cat([t[1], v[i, b, h, :m]])]

    def values(self, l, b, h):
        """What the oracle has the cache stand for: (codes, scales) of keys and of values."""
        out = []
        for side in (0, 1):
            x = self.tok[l][b][h][side].float().numpy()
            parts = [O.quantise(x[i:i + BLOCK]) for i in range(0, len(x), BLOCK)]
            out.append((np.concatenate([p[0] for p in parts]) if parts else np.zeros((0, D), np.int8), np.array([p[1] for p in parts], np.float32)))
        return out

    def check(self):
        c, P = self.c, self.page
        codes, scales, table, lens = c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table.cpu().numpy(), c.seq_len.cpu().numpy()
        raw = c.raw.cpu()
        for l in range(self.L):
            for b in range(self.B):
                n = self.tok[l][b][0][0].shape[0]
                assert lens[l, b] == n
                for h in range(self.H):
                    for side, (want, ws) in enumerate(self.values(l, b, h)):
                        for i in range(0, n, BLOCK):
                            p = table[b, i // P]
                            rows = min(BLOCK, n - i)
                            assert scales[l, p, h, side, i % P // BLOCK] == ws[i // BLOCK] or np.isnan(ws[i // BLOCK])
                            assert np.isnan(scales[l, p, h, side, i % P // BLOCK]) == np.isnan(ws[i // BLOCK])
                            assert (codes[l, p, h, side, i % P:i % P + rows] == want[i:i + rows]).all(), (l, b, h, side, i)
                        t = self.tok[l][b][h][side][n - n % BLOCK:]
                        assert torch.equal(raw[l, b, h, side, :n % BLOCK], t)

    def attend(self, n, q_len=None, layers=None, sm_scale=None, q=None, rope=None, poison=7.0, workspace=None):
        """One call, checked against the oracle over the cache's own codes."""
        l0, lc = layers or (0, self.L)
        q = randn(self.g, lc, self.B, self.Hq, n, D, dtype=self.dtype) if q is None else q
        out = torch.full((lc, self.B, self.Hq, n, D), poison, dtype=self.dtype, device="cuda")
        ql = None if q_len is None else torch.tensor(q_len, dtype=torch.int32).cuda()
        ws = workspace if workspace is not None else torch.empty(B.paged_workspace_bytes(self.c, lc, n), dtype=torch.uint8, device="cuda")
        B.paged_attention(self.c, l0, lc, q.cuda(), ws, out, ql, rope, sm_scale)
        if rope is not None:
            q = q.cuda()
            for i in range(lc):
                B.rope_apply(rope, q[i], q[i])
            q = q.cpu()
        self.compare(out, q, n, q_len, l0, sm_scale, poison)
        return out

    def compare(self, out, q, n, q_len, l0, sm_scale, poison):
        got, G = f64(out), self.Hq // self.H
        scale = D ** -0.5 if sm_scale is None else sm_scale
        for i in range(got.shape[0]):
            for b in range(self.B):
                m = n if q_len is None else max(0, min(n, q_len[b]))
                assert (got[i, b, :, m:] == poison).all()
                for h in range(self.H):
                    (kc, ks), (vc, vs) = self.values(l0 + i, b, h)
                    k, v = O.dequantise(kc, ks), O.dequantise(vc, vs)
                    heads = slice(h * G, h * G + G)
                    seen = np.tile(len(k) - m + 1 + np.arange(m), G)
                    ref, mag, top = O.attention(f64(q[i, b, heads, :m]).reshape(-1, D), k, v, scale, seen)
                    y = got[i, b, heads, :m].reshape(-1, D)
                    assert (np.abs(y - ref) <= attention_bound(ref, mag, top, self.dtype, n * G)).all(), (
                        i, b, h, np.abs(y - ref).max(), (np.abs(y - ref) / attention_bound(ref, mag, top, self.dtype, n * G)).max())


def attention_bound(ref, mag, top, dtype, rows):
    """A score in units of log2 carries three roundings of fp32 (the dot product's integers, the two scales) and the softmax' exponent one
    more: 4 * 2^-24 * log2(e) |s|, that times ln 2 in a numerator and as much in the sum; the exponential, the 32-bit numerators and the
    sums add at most 32 * 2^-24; more than eight rows of a head meet in the prompt kernel, whose numerators have fp16's 11 bits; then
    the output's own rounding."""
    inner = 2.0 ** -24 * (8 * top[:, None] + 32) + (2.0 ** -11 if rows > 8 else 0)
    err = inner * mag
    return err + torch.finfo(dtype).eps / 2 * (np.abs(ref) + err) + (2.0 ** -25 if dtype == F16 else 1e-38)


# ------------------------------------------------------------------------------------------------ append, read
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_append_pieces(dtype, page):
    m = Model(2, 4, 2, 4, max_pages=max(2, 512 // page), page=page, dtype=dtype)
    for n, new_len in ((1, None), (30, None), (1, None), (1, [1, 0, 1, -3]), (70, [70, 3, 64, 0]), (5, [9, 5, 0, 1]), (32, None), (129, [129, 1, 128, 31])):
        m.append(n, new_len)
        m.check()
    assert m.c.device_status() == 0


def test_append_is_independent_of_the_pieces():
    """One call with all tokens and one call per token leave the same bytes."""
    a, b = (Model(1, 2, 2, 2, max_pages=3, page=64, dtype=F16, seed=5) for _ in range(2))
    k, v = randn(gen(6), 1, 2, 2, 101, D), randn(gen(7), 1, 2, 2, 101, D)
    a.append(101, k=k, v=v)
    for i in range(101):
        b.append(1, k=k[:, :, :, i:i + 1], v=v[:, :, :, i:i + 1])
    a.check()
    b.check()
    assert a.c.device_status() == b.c.device_status() == 0


def test_append_strides_layers_and_taking_back():
    m = Model(3, 2, 4, 8, max_pages=2, page=64, dtype=BF16)
    x = randn(m.g, 2, 45, 12, D, dtype=BF16)                       # a projection [batch, n, (.. | k heads | v heads) * 128]
    k, v = x[:, :, 4:8].transpose(1, 2)[None], x[:, :, 8:].transpose(1, 2)[None]
    xd = x.cuda()
    B.paged_append(m.c, 1, 1, xd[:, :, 4:8].transpose(1, 2)[None], xd[:, :, 8:].transpose(1, 2)[None])
    for b in range(2):
        for h in range(4):
            m.tok[1][b][h] = [k[0, b, h], v[0, b, h]]
    m.check()
    # the same keys for every layer: stride 0
    k3 = k[:, :, :, :7].contiguous().expand(3, 2, 4, 7, D)
    m.append(7, k=k3, v=k3)
    m.check()
    # tokens of the unfinished block given back, others appended in their place
    m.c.seq_len[1] -= 9
    for b in range(2):
        for h in range(4):
            m.tok[1][b][h] = [t[:-9] for t in m.tok[1][b][h]]
    m.append(3)
    m.check()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_append_extreme_blocks(dtype):
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    m = Model(1, 8, 1, 1, max_pages=2, page=32, dtype=dtype)
    k = torch.zeros(1, 8, 1, 33, D, dtype=dtype)
    k[0, 1, 0, 3, 5] = big
    k[0, 2, 0] = torch.arange(33 * D).reshape(33, D) % 77 * (small / 64)   # subnormal
    k[0, 3, 0, 31, 127] = float("nan")
    k[0, 4, 0, 0, 0] = float("inf")
    k[0, 5, 0, 2, 0] = -float("inf")
    k[0, 6, 0] = -3.0
    k[0, 7, 0, :, 0] = torch.arange(33) / 8
    m.append(33, k=k, v=k.flip(-1))
    m.check()
    back = [torch.full((1, 8, 1, 33, D), 5.0, dtype=dtype, device="cuda") for _ in range(2)]
    B.paged_read(m.c, 0, 1, 0, *back)
    assert torch.isnan(back[0][0, 3:6, 0, :32]).all() and not torch.isnan(back[0][0, 3:6, 0, 32]).any()
    assert (back[0][0, 0] == 0).all() and back[0][0, 1, 0, 3, 5] == big
    assert (back[0][0, 6, 0, :32] == -3.0).all()


def test_append_with_rope_is_rope_then_append():
    for dtype, sections, inter in ((F16, (16, 24, 24), False), (BF16, (24, 20, 20), True), (F16, (8, 8, 0), False)):
        a, b = (Model(2, 3, 2, 2, max_pages=3, page=64, dtype=dtype, seed=9) for _ in range(2))
        for n in (1, 40, 66):
            pos = positions(a.g, 3, n, "near").cuda()
            rope = B.Rope(pos, B.rope_frequencies(1e6, sum(sections)), sections, inter)
            k, v = randn(gen(n), 2, 3, 2, n, D, dtype=dtype), randn(gen(n + 1), 2, 3, 2, n, D, dtype=dtype)
            a.append(n, k=k, v=v, rope=rope)
            a.check()


def test_append_refused_sequences_stay():
    """A missing page, a bad one, a row without room: status, and the others go on."""
    m = Model(1, 4, 1, 1, max_pages=2, page=32, dtype=F16)
    m.append(20)
    m.c.table[1, 1] = -1
    m.c.table[2, 1] = m.c.n_pages
    before = m.c.codes.clone(), m.c.raw.clone(), m.c.scales.clone()
    k, v = randn(m.g, 1, 4, 1, 45, D), randn(m.g, 1, 4, 1, 45, D)
    B.paged_append(m.c, 0, 1, k.cuda(), v.cuda(), torch.tensor([13, 13, 13, 45], dtype=torch.int32).cuda())
    assert m.c.device_status() == B.ERR_CAPACITY
    assert m.c.seq_len[0].tolist() == [33, 20, 20, 20]
    changed = (m.c.codes != before[0]).flatten(1).any(1)
    own = set(m.c.table[0].tolist())
    assert {p for p in range(m.c.n_pages) if (m.c.codes[0, p] != before[0][0, p]).any()} <= own and changed.any()
    assert torch.equal(m.c.raw[0, 1:], before[1][0, 1:])
    for b in range(4):
        m.tok[0][b][0] = [torch.cat([m.tok[0][b][0][0], k[0, b, 0, :13]]), torch.cat([m.tok[0][b][0][1], v[0, b, 0, :13]])] if b == 0 else m.tok[0][b][0]
    m.c.table[1, 1], m.c.table[2, 1] = 0, 0     # (not looked at: behind the lengths)
    m.check()


@pytest.mark.parametrize("dtype,page", [(F16, 32), (BF16, 256)])
def test_read(dtype, page):
    m = Model(2, 3, 2, 2, max_pages=4, page=page, dtype=dtype)
    m.append(100, [100, 0, 33])
    for begin, n in ((0, 100), (31, 5), (32, 1), (90, 200), (5, 0)):
        out = [torch.full((2, 3, 2, n, D), 9.0, dtype=dtype, device="cuda") for _ in range(2)]
        B.paged_read(m.c, 0, 2, begin, *out)
        for l in range(2):
            for b in range(3):
                held = max(0, min(n, m.lens()[b] - begin))
                for h in range(2):
                    for side, (codes, scales) in enumerate(m.values(l, b, h)):
                        ref = O.dequantise(codes, scales)[begin:begin + held]
                        y = f64(out[side][l, b, h])
                        assert (np.abs(y[:held] - ref) <= 2.0 ** -24 * np.abs(ref) + torch.finfo(dtype).eps / 2 * np.abs(ref) * (1 + 2.0 ** -20) + 2.0 ** -25).all()
                        assert (y[held:] == 9.0).all()
    assert m.c.device_status() == 0


# ------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,Hq,page", [(1, 7, 64), (2, 16, 32), (4, 4, 128), (3, 15, 256), (2, 4, 64), (1, 1, 32)])
def test_attention_single_tokens(dtype, H, Hq, page):
    m = Model(2, 5, H, Hq, max_pages=max(2, 768 // page), page=page, dtype=dtype)
    m.append(1, [1, 1, 1, 0, 1])
    m.attend(1)
    m.append(700, [700, 0, 31, 0, 128])
    m.attend(1)
    m.append(33, [1, 2, 32, 0, 0])
    m.attend(1)
    m.attend(1, q_len=[1, 0, 1, 1, 5])
    m.attend(1, layers=(1, 1))
    assert m.c.device_status() == 0


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("H,Hq,page,n", [(1, 7, 64, 2), (2, 16, 32, 5), (4, 4, 128, 3), (3, 15, 256, 40), (2, 4, 64, 130), (1, 8, 32, 17), (1, 1, 32, 200)])
def test_attention_several_queries(dtype, H, Hq, page, n, wide):
    m = Model(1, 5, H, Hq, max_pages=max(2, 1024 // page), page=page, dtype=dtype, wide=wide)
    assert not wide or n * Hq // H <= 16 or B.paged_plan(m.c, 1, n) == B.PLAN_PROMPT
    m.append(n, [n, max(1, n // 2), 1, 0, n - 1])
    m.attend(n)                                            # more queries than tokens: rows that see nothing
    m.append(420, [420, 7, 160, 0, 33])
    m.attend(n)
    m.attend(n, q_len=[n, 0, 1, 2, n - 1])
    assert m.c.device_status() == 0


@pytest.mark.parametrize("n", [1, 3, 33])
def test_attention_long_context(n):
    m = Model(1, 2, 1, 7, max_pages=80, page=256, dtype=F16)
    m.append(20000, [20000, 6001])
    m.attend(n)


@pytest.mark.parametrize("n,wide", [(1, False), (40, False), (1, True), (40, True)])
def test_attention_scales_and_sinks(n, wide):
    """Softmax scales of either sign and zero; one token that takes nearly all of the mass with next to no value; large scores."""
    m = Model(1, 2, 2, 8, max_pages=8, page=64, dtype=F16, wide=wide)
    k, v = randn(m.g, 1, 2, 2, 400, D), randn(m.g, 1, 2, 2, 400, D)
    k[:, 1, :, 0] = 0.5
    v[:, 1, :, 0] = 0
    m.append(400, k=k, v=v)
    for scale in (-0.1, 0.0, 0.3):
        m.attend(n, sm_scale=scale)
    q = randn(m.g, 1, 2, 8, n, D)
    q[:, 1] = q[:, 1] * 0.05 + 2.0        # the first token's score is 128 / sqrt(128) above the rest
    m.attend(n, q=q)
    q[0, 0, 0] = 0
    q[0, 0, 1] *= 30
    m.attend(n, q=q)


def test_attention_infinite_and_lost_things():
    for n, wide in ((1, False), (20, False), (1, True), (20, True)):
        m = Model(1, 4, 1, 2, max_pages=4, page=32, dtype=F16, wide=wide)
        k, v = randn(m.g, 1, 4, 1, 100, D), randn(m.g, 1, 4, 1, 100, D)
        k[0, 1, 0, 40, 3] = float("inf")         # second block of sequence 1
        v[0, 2, 0, 99, 3] = float("nan")         # last block of sequence 2
        m.append(100, k=k, v=v)
        m.c.table[3, 1] = -1
        q = randn(m.g, 1, 4, 2, n, D)
        q[0, 0, 1] = float("nan")
        out = torch.zeros(1, 4, 2, n, D, dtype=F16, device="cuda")
        ws = torch.empty(B.paged_workspace_bytes(m.c, 1, n), dtype=torch.uint8, device="cuda")
        B.paged_attention(m.c, 0, 1, q.cuda(), ws, out)
        assert torch.isfinite(out[0, 0, 0]).all() and torch.isnan(out[0, 0, 1]).all()
        assert torch.isnan(out[0, 1]).all() and torch.isnan(out[0, 3]).all()
        sees = 100 - n + 1 + np.arange(n) > 96       # queries that see a token of the last block, and those that do not
        assert torch.isnan(out[0, 2][:, sees]).all() and torch.isfinite(out[0, 2][:, ~sees]).all()
        assert m.c.device_status() == B.ERR_INVALID_ARG


def test_attention_rope_strides_and_streams():
    m = Model(2, 3, 2, 6, max_pages=4, page=64, dtype=BF16)
    m.append(200, [200, 64, 3])
    for n in (1, 4, 50):
        pos = positions(m.g, 3, n, "near").cuda()
        m.attend(n, rope=B.Rope(pos, B.rope_frequencies(1e6, 64), (24, 20, 20), True))
        # [batch, n, heads * 128] in and out, another stream
        x = randn(m.g, 2, 3, n, 6, D, dtype=BF16)
        xd, od = x.cuda(), torch.full((2, 3, n, 6, D), 7.0, dtype=BF16, device="cuda")
        ws = torch.empty(B.paged_workspace_bytes(m.c, 2, n), dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        B.paged_attention(m.c, 0, 2, xd.transpose(2, 3), ws, od.transpose(2, 3), stream=s)
        s.synchronize()
        m.compare(od.transpose(2, 3), x.transpose(2, 3), n, None, 0, None, 7.0)


@pytest.mark.parametrize("n", [1, 3, 64])
def test_attention_graphs_share_a_workspace(n):
    """Two captured graphs with one workspace, replayed after the cache has grown; results equal eager calls bit for bit."""
    m = Model(2, 3, 2, 14, max_pages=6, page=64, dtype=F16)
    m.append(100, [100, 64, 0])
    qs = [randn(m.g, 1, 3, 14, n, D).cuda() for _ in range(2)]
    outs = [torch.zeros_like(q) for q in qs]
    ws = torch.empty(B.paged_workspace_bytes(m.c, 1, n), dtype=torch.uint8, device="cuda")
    for i in (0, 1):
        B.paged_attention(m.c, i, 1, qs[i], ws, outs[i])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i in (0, 1):
        with torch.cuda.graph(graphs[i]):
            B.paged_attention(m.c, i, 1, qs[i], ws, outs[i])
    m.append(150, [150, 150, 1])
    for i in (1, 0):
        ws.fill_(0xff)
        graphs[i].replay()
    got = [o.clone() for o in outs]
    for i in (0, 1):
        m.compare(got[i], qs[i].cpu(), n, None, i, None, 0.0)
        B.paged_attention(m.c, i, 1, qs[i], ws, outs[i])
        assert torch.equal(outs[i], got[i])


@pytest.mark.parametrize("n", [1, 64])
def test_a_threads_first_call_may_be_a_captured_one(n):
    """What the library asks the device about once per thread is asked in a capture here."""
    m = Model(1, 2, 2, 14, max_pages=6, page=64, dtype=F16)
    m.append(200, [200, 64])
    q = randn(m.g, 1, 2, 14, n, D).cuda()
    want, got = torch.zeros_like(q), torch.zeros_like(q)
    ws = torch.empty(B.paged_workspace_bytes(m.c, 1, n), dtype=torch.uint8, device="cuda")
    graph, failed = torch.cuda.CUDAGraph(), []

    def capture():
        try:
            with torch.cuda.graph(graph):
                B.paged_attention(m.c, 0, 1, q, ws, got)
        except BaseException as e:   # noqa: BLE001
            failed.append(e)
    t = threading.Thread(target=capture)
    t.start()
    t.join()
    assert not failed
    graph.replay()
    B.paged_attention(m.c, 0, 1, q, ws, want)
    assert torch.equal(got, want)
    m.compare(got, q.cpu(), n, None, 0, None, 0.0)


def random_cache(g, L, batch, H, Hq, page, dtype, lens):
    """A cache filled with numbers rather than through appends: lens[b] tokens, pages in an order of their own."""
    width = max(1, max((n + page - 1) // page for n in lens))
    n_pages = sum((n + page - 1) // page for n in lens) + 2
    c = B.PagedCache(L, batch, H, Hq, n_pages, width, page, dtype)
    c.codes.copy_(torch.randint(-127, 128, c.codes.shape, generator=g, dtype=torch.int8))
    c.scales.copy_(torch.rand(c.scales.shape, generator=g) * 0.02 + 0.002)
    order, k = torch.randperm(n_pages, generator=g).tolist(), 0
    table = torch.full((batch, width), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        for j in range((n + page - 1) // page):
            table[b, j] = order[k]
            k += 1
    c.table.copy_(table)
    c.seq_len.copy_(torch.tensor(lens, dtype=torch.int32).expand(L, batch))
    return c


def check_random(c, q, out, q_len, poison):
    """Against softmax attention in 64 bits (torch, on the GPU), sequence by sequence."""
    G, n, P = c.n_q_heads // c.n_kv_heads, q.shape[3], c.page_tokens
    lens = c.seq_len[0].tolist()
    for b, T in enumerate(lens):
        m = n if q_len is None else max(0, min(n, q_len[b]))
        assert (out[:, b, :, m:] == poison).all()
        if m == 0:
            continue
        pages = c.table[b, :(T + P - 1) // P].long()
        x = (c.codes[:, pages].double().unflatten(5 - 1, (-1, BLOCK)) * c.scales[:, pages].double()[..., None, None]).flatten(4, 5)   # [L, w, H, 2, P, 128]
        x = x.permute(0, 2, 3, 1, 4, 5).flatten(3, 4)[:, :, :, :T]
        k, v = x[:, :, 0], x[:, :, 1]
        s = torch.einsum("lhgnd,lhtd->lhgnt", q[:, b, :, :m].double().unflatten(1, (-1, G)), k) * D ** -0.5
        seen = T - m + 1 + torch.arange(m, device="cuda")
        late = torch.arange(T, device="cuda")[None] >= seen[:, None]
        top = s.masked_fill(late, 0).abs().amax(-1) if T else torch.zeros(s.shape[:-1], device="cuda", dtype=torch.float64)
        w = torch.softmax(s.masked_fill(late, -float("inf")), -1).nan_to_num(0.0)
        ref, mag = w @ v[:, :, None], w @ v[:, :, None].abs()
        got = out[:, b, :, :m].double().unflatten(1, (-1, G))
        # attention_bound, here as tensors
        inner = 2.0 ** -24 * (8 * top[..., None] + 32) + (2.0 ** -11 if n * G > 8 else 0)
        err = inner * mag
        bound = err + torch.finfo(q.dtype).eps / 2 * (ref.abs() + err) + (2.0 ** -25 if q.dtype == F16 else 1e-38)
        assert ((got - ref).abs() <= bound).all(), (b, T, m, ((got - ref).abs() / bound).max().item())


# (layers, batch, KV heads, group, page, queries, longest): more items than ranges, items of one tile, row tiles of every kind (eight rows
# and fewer; 256, up to 128 and between) behind one another in a range, ranges that end inside items, sequences that are empty
SCHEDULES = [(3, 64, 8, 4, 32, 1, 300), (1, 300, 4, 2, 64, 1, 130), (2, 1, 1, 8, 32, 1, 9000), (28, 9, 4, 7, 64, 1, 700), (1, 2, 8, 1, 256, 8, 40000),
             (1, 40, 4, 7, 32, 5, 400), (2, 33, 8, 4, 64, 40, 300), (1, 5, 2, 7, 128, 700, 1500), (1, 1, 1, 8, 64, 1000, 1000), (3, 17, 3, 5, 32, 130, 140),
             (1, 200, 2, 8, 32, 20, 90), (1, 2, 1, 1, 64, 3000, 3500), (1, 3, 4, 8, 256, 33, 30000), (4, 50, 4, 1, 64, 300, 310),
             (1, 40, 4, 7, 32, 2, 400), (2, 9, 3, 5, 64, 4, 2000), (1, 1, 2, 1, 64, 13, 5000), (1, 2, 2, 7, 32, 9, 500), (1, 1, 4, 8, 64, 24, 900),
             (28, 2, 4, 7, 64, 3, 700), (1, 1, 1, 3, 256, 8, 33000)]


@pytest.mark.parametrize("shape", SCHEDULES, ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_schedules(shape, dtype):
    L, batch, H, G, page, n, longest = shape
    g = gen(sum(shape))
    for ragged in (False, True):
        lens = [longest] * batch if not ragged else [int(longest * x ** 2) for x in torch.rand(batch, generator=g).tolist()]
        if ragged:
            lens[-1] = 0
        q_len = None if not ragged else torch.randint(-1, n + 2, (batch,), generator=g).tolist()
        c = random_cache(g, L, batch, H, H * G, page, dtype, lens)
        q = randn(g, L, batch, H * G, n, D, dtype=dtype).cuda()
        out = torch.full_like(q, 5.0)
        ws = torch.full((B.paged_workspace_bytes(c, L, n),), 0xff, dtype=torch.uint8, device="cuda")
        ql = None if q_len is None else torch.tensor(q_len, dtype=torch.int32).cuda()
        B.paged_attention(c, 0, L, q, ws, out, ql)
        assert c.device_status() == 0
        check_random(c, q, out, q_len, 5.0)
        again = torch.full_like(q, 5.0)
        B.paged_attention(c, 0, L, q, ws, again, ql)
        assert torch.equal(out, again)


def test_attention_plans():
    """The rule of sizes: a cluster for few short items of eight rows; even ranges for many or long ones, up to 16 rows, and 24 where not
    all is read from memory again; the prompt kernel else."""
    def plan(L, batch, H, Hq, tokens, n):
        c = B.PagedCache(L, batch, H, Hq, 4, (tokens + 63) // 64, 64)
        return B.paged_plan(c, L, n)
    assert plan(1, 1, 1, 7, 2048, 1) == 8 and plan(1, 4, 4, 28, 4096, 1) in (4, 5, 6) and plan(1, 30, 4, 4, 130, 1) in (1, 2)
    assert plan(1, 1, 4, 28, 131072, 1) == plan(1, 16, 4, 32, 32768, 1) == plan(28, 8, 4, 28, 512, 1) == B.PLAN_LINE
    assert plan(1, 1, 1, 7, 2048, 2) == plan(1, 1, 1, 8, 64, 2) == plan(1, 1, 1, 1, 2048, 8) == 8 and plan(1, 1, 4, 32, 1000, 24) in (1, 2)
    assert plan(1, 16, 4, 32, 32768, 2) == plan(1, 1, 4, 32, 131072, 3) == B.PLAN_LINE
    assert plan(1, 16, 4, 32, 32768, 3) == plan(1, 1, 4, 32, 131072, 4) == plan(1, 1, 4, 28, 8192, 2048) == plan(1, 16, 4, 28, 12345, 5) == B.PLAN_PROMPT


@pytest.mark.parametrize("batch,H,n,tokens", [(1, 1, 1, 2000), (30, 8, 1, 1500), (1, 2, 40, 2000), (2, 2, 300, 700)])
def test_attention_waits_are_bounded(batch, H, n, tokens):
    """With nothing delivered every role's wait runs out: NaN, the status word, and a device that goes on."""
    g = gen(11)
    c = random_cache(g, 1, batch, H, 7 * H, 64, F16, [tokens] * batch)
    q = randn(g, 1, batch, 7 * H, n, D).cuda()
    out, ws = torch.zeros_like(q), torch.empty(B.paged_workspace_bytes(c, 1, n), dtype=torch.uint8, device="cuda")
    B.debug_paged_timeout(c, 0, 1, q, ws, out, limit_clocks=2_000_000)
    torch.cuda.synchronize()
    assert c.device_status() == B.ERR_TIMEOUT and torch.isnan(out).all()
    c.status.zero_()
    out.fill_(5.0)
    B.paged_attention(c, 0, 1, q, ws, out)
    check_random(c, q, out, None, 5.0)
    assert c.device_status() == 0


def test_offsets_beyond_32_bits():
    """A pool of 5 GB whose last pages are the ones in use."""
    m = Model(1, 2, 4, 8, max_pages=2, page=256, dtype=F16, n_pages=20000)
    ids = torch.tensor([[19999, 19997], [1, 19990]], dtype=torch.int32)
    m.c.table.copy_(ids)
    m.c.refs.zero_()
    m.c.refs[ids.flatten().long()] = 1
    m.append(300)
    m.attend(1)
    m.attend(20)
    out = [torch.zeros(1, 2, 4, 300, D, dtype=F16, device="cuda") for _ in range(2)]
    B.paged_read(m.c, 0, 1, 0, *out)
    assert torch.equal(out[1][0, 0, 1, 299].cpu(), torch.from_numpy(O.dequantise(*m.values(0, 0, 1)[1])[299]).half())
    B.pages_copy(m.c, torch.tensor([19999], dtype=torch.int32).cuda(), torch.tensor([19998], dtype=torch.int32).cuda())
    assert torch.equal(m.c.codes[0, 19998], m.c.codes[0, 19999]) and torch.equal(m.c.scales[0, 19998], m.c.scales[0, 19999])


# ------------------------------------------------------------------------------------------------ pages
@pytest.mark.parametrize("seed,batch,max_pages,n_pages,page", [(0, 6, 9, 40, 32), (1, 12, 33, 300, 64), (2, 3, 700, 5000, 32), (3, 40, 130, 9001, 32)])
def test_pages_against_lists(seed, batch, max_pages, n_pages, page):
    """Random sequences of calls; tables, counts and what the pages hold follow the oracle's lists."""
    rng = np.random.RandomState(seed)
    c = B.PagedCache(2, batch, 1, 1, n_pages, max_pages, page, F16)
    c.codes.random_(-127, 128)
    c.scales.normal_()
    c.raw.normal_()
    P = O.Pages(batch, max_pages, n_pages, page)
    P.content = list(range(n_pages))
    first = c.codes.clone(), c.scales.clone()
    ws = torch.empty(B.paged_workspace_bytes(c, 1, 1), dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    status = 0
    for step in range(60):
        c.status.zero_()
        what = rng.choice(["reserve", "reserve", "fork", "release", "compact", "fill"])
        if what == "reserve":
            t = [int(x) for x in rng.randint(-2, max_pages * page // (2 if step % 3 else 4), batch)]
            if step % 11 == 5:
                t[0] = max_pages * page + 1
            ok = P.reserve(t)
            B.pages_reserve(c, i32(t))
            assert (c.device_status() == 0) == ok
        elif what == "fill":
            for b in range(batch):   # lengths up to the pages that are there
                have = 0
                while have < max_pages and P.table[b][have] >= 0:
                    have += 1
                P.lens[b] = int(rng.randint(0, have * page + 1))
            c.seq_len.copy_(i32(P.lens).expand(2, batch))
        elif what == "fork":
            pairs = [(int(rng.randint(0, batch)), int(rng.randint(0, batch))) for _ in range(rng.randint(1, 5))]
            ok = P.fork(*zip(*pairs))
            B.pages_fork(c, i32([a for a, _ in pairs]), i32([d for _, d in pairs]), ws)
            assert (c.device_status() == 0) == ok
        elif what == "release":
            s = [int(x) for x in rng.randint(0, batch, rng.randint(1, 4))]
            P.release(s)
            B.pages_release(c, i32(s + s[:1]))
            assert c.device_status() == 0
        else:
            n = torch.zeros(1, dtype=torch.int32, device="cuda")
            want = P.compact()
            B.pages_compact(c, ws, n)
            assert int(n) == want
        assert c.table.cpu().tolist() == P.table and c.refs.cpu().tolist() == P.refs, (step, what)
        assert c.seq_len.cpu().tolist() == [P.lens] * 2
        used = [p for p in range(n_pages) if P.refs[p] > 0]
        if used:
            at, of = torch.tensor(used).cuda(), torch.tensor([P.content[p] for p in used]).cuda()
            assert torch.equal(c.codes[:, at], first[0][:, of]) and torch.equal(c.scales[:, at], first[1][:, of]), (step, what)
        free = P.free()
        if free:                     # pages that came free hold their first content again
            f = torch.tensor(free).cuda()
            c.codes[:, f] = first[0][:, f]
            c.scales[:, f] = first[1][:, f]
            for p in free:
                P.content[p] = p


def test_pages_fork_chain_and_bad_indices():
    m = Model(2, 6, 2, 2, max_pages=3, page=64, dtype=F16, n_pages=40)
    m.c.table.fill_(-1)
    m.c.refs.zero_()
    B.pages_reserve(m.c, torch.tensor([128, 0, 0, 0, 0, 0], dtype=torch.int32).cuda())
    m.append(100, [100, 0, 0, 0, 0, 0])
    ws = torch.empty(B.paged_workspace_bytes(m.c, 1, 1), dtype=torch.uint8, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    # 0 -> 1 -> 2 in one call (2 comes from a page that the same call fills), a pair out of range, an occupied destination
    B.pages_fork(m.c, i32(0, 1, 7, 2, 0), i32(1, 2, 3, 0, 9), ws)
    assert m.c.device_status() == B.ERR_INVALID_ARG
    m.c.status.zero_()
    assert m.c.seq_len.tolist() == [[100, 100, 100, 0, 0, 0]] * 2
    assert m.c.table[:3, 0].unique().numel() == 1 and m.c.table[:3, 1].unique().numel() == 3
    for l in range(2):
        for b in (1, 2):
            m.tok[l][b] = [list(t) for t in m.tok[l][0]]
    m.check()
    # each goes on alone
    B.pages_reserve(m.c, torch.tensor([192, 192, 192, 0, 0, 0], dtype=torch.int32).cuda())
    m.append(50, [50, 13, 28, 0, 0, 0])
    m.check()
    m.attend(1)
    B.pages_release(m.c, i32(0, -1, 6, 0))
    assert m.c.device_status() == B.ERR_INVALID_ARG
    for l in range(2):
        m.tok[l][0] = [[torch.zeros(0, D, dtype=F16)] * 2 for _ in range(2)]
    m.check()
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pages_compact(m.c, ws, n)
    assert int(n) == 5 and int(m.c.table.max()) == 4
    m.check()
    m.attend(1)


def test_pages_copy_refuses_conflicts():
    c = B.PagedCache(2, 1, 2, 2, 9, 4, 32, BF16)
    c.codes.random_(-127, 128)
    c.scales.normal_()
    before = c.codes.clone(), c.scales.clone()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    B.pages_copy(c, i32(0, 0, 5), i32(1, 2, 5))
    assert c.device_status() == 0
    for p in (1, 2):
        assert torch.equal(c.codes[:, p], before[0][:, 0]) and torch.equal(c.scales[:, p], before[1][:, 0])
    keep = c.codes.clone()
    # 3 named twice as destination, 6 as source and destination, indices out of range
    B.pages_copy(c, i32(0, 5, 6, 5, -1, 0), i32(3, 3, 7, 6, 8, 9))
    assert c.device_status() == B.ERR_INVALID_ARG
    keep[:, 7] = keep[:, 6]
    assert torch.equal(c.codes, keep)


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_serving_run(dtype):
    """A prompt with positions, continuations of it, single tokens and drafts, an end, a compaction."""
    m = Model(2, 5, 2, 14, max_pages=6, page=64, dtype=dtype, n_pages=30)
    m.c.table.fill_(-1)
    m.c.refs.zero_()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    ws = torch.empty(max(B.paged_workspace_bytes(m.c, 2, n) for n in (1, 4, 150)), dtype=torch.uint8, device="cuda")
    freq = B.rope_frequencies(1e6, 64)

    def rope(n, start):
        p = (torch.arange(n)[None] + torch.tensor(start)[:, None])[None].expand(3, 5, n).contiguous().int().cuda()
        return B.Rope(p, freq, (16, 24, 24))

    B.pages_reserve(m.c, i32(150, 0, 0, 0, 0))
    r = rope(150, [0] * 5)
    m.append(150, [150, 0, 0, 0, 0], rope=r)
    m.attend(150, q_len=[150, 0, 0, 0, 0], rope=r, workspace=ws)
    B.pages_fork(m.c, i32(0, 0), i32(3, 1), ws)
    for l in range(2):
        for b in (1, 3):
            m.tok[l][b] = [list(t) for t in m.tok[l][0]]
    B.pages_reserve(m.c, i32(200, 200, 0, 200, 0))
    for step in range(3):
        lens = m.lens()
        r = rope(1, lens)
        m.append(1, [1, 1, 0, 1, 0], rope=r)
        m.attend(1, q_len=[1, 1, 0, 1, 0], rope=r, workspace=ws)
    r = rope(4, m.lens())
    m.append(4, [4, 2, 0, 3, 0], rope=r)
    m.attend(4, q_len=[4, 2, 0, 3, 0], workspace=ws)
    B.pages_release(m.c, i32(0))
    for l in range(2):
        m.tok[l][0] = [[torch.zeros(0, D, dtype=dtype)] * 2 for _ in range(2)]
    B.pages_compact(m.c, ws)
    m.check()
    m.attend(1, workspace=ws)
    assert m.c.device_status() == 0
