"""Normed heads with rotary positions, and their gradients, on the GPU against the oracle in 64 bits."""
import threading

import numpy as np
import pytest
import torch

from oracle import okq_norm_oracle as N
from paper_2609_11582_b200 import binding as B
from tests.test_gpu_paged import BF16, D, F16, F32, SECTIONS, f64, gen, positions, randn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = {F16: 2.0 ** -25, BF16: 0.0, F32: 2.0 ** -149}


def pairs(mag, turn):
    """Magnitudes that a rotation mixes: the sum of a pair's."""
    if turn is None:
        return mag
    half, out = sum(turn[2]), mag.copy()
    out[..., :half] = out[..., half:2 * half] = mag[..., :half] + mag[..., half:2 * half]
    return out


def turn_error(turn):
    """Cosine and sine to two units (2^-22), half a unit of their angle, roundings of product and sum: 6 * 2^-24; 1e-6 of angles near 2^31."""
    return 0.0 if turn is None else 6 * U + 1e-6


def rounded(ref, err, dtype):
    return err + (torch.finfo(dtype).eps / 2 * (np.abs(ref) + err) if dtype != F32 else 0) + TINY[dtype]


def apply_bound(ref, y, dtype, turn):
    """The sum of squares takes 16 steps and three exchanges, all of one sign: 19 * 2^-24 of it, half of that in its root, the sum with eps, the
    root's own rounding, and the two products: 13 * 2^-24 of a normed number; then the rotation, and the result's rounding."""
    return rounded(ref, (13 * U + turn_error(turn)) * pairs(np.abs(y), turn), dtype)


def grad_bounds(x, w, g, u, dx, dtype, eps, turn, chain):
    """x r to 12 * 2^-24, u by the rotation, w u one rounding more; the mean of w u x r 16 steps, three exchanges and a product; then a
    product, a difference and a product, each to 2^-24 of what enters.  The weights' sums: `chain` additions one after another at most."""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, du = np.abs(x * r), turn_error(turn) * pairs(np.abs(g), turn)
    aw, wu = np.abs(w), np.abs(w * u)
    dot = (wu * xh).mean(-1, keepdims=True)
    d_dot = (aw * du * xh + (12 + 1 + 20) * U * wu * xh).mean(-1, keepdims=True)
    err = r * (aw * du + 16 * U * (wu + xh * dot) + xh * d_dot)
    err_w = (du * xh + (13 + chain) * U * np.abs(u) * xh).reshape(-1, D).sum(0)
    return rounded(dx, err, dtype), err_w


def weight(g, dtype, big=4.0):
    w = 1 + 0.3 * torch.randn(D, generator=g)
    w[:4] *= big
    return w.to(dtype).cuda()


def tensor(g, batch, heads, n, dtype, inner, scale=3.0):
    x = randn(g, batch, n, heads, D, dtype=dtype, scale=scale) if inner else randn(g, batch, heads, n, D, dtype=dtype, scale=scale)
    return x.cuda().transpose(1, 2) if inner else x.cuda()


CASES = [(1, 7, 1, 1, "near", True), (3, 4, 2, 37, "far", False), (2, 1, 0, 130, "negative", True), (2, 32, 4, 17, "near", True), (1, 9, 16, 5, "zero", False)]


def check(dtype, wdtype, sections, interleaved, shape, eps, seed=1):
    g = gen(seed)
    batch, hq, hk, n, kind, inner = shape
    rope, turn = None, None
    if sections:
        pos, freq = positions(g, batch, n, kind), B.rope_frequencies(1e6, sum(sections), "cpu")
        rope, turn = B.Rope(pos.cuda(), freq.cuda(), sections, interleaved), (pos.numpy(), freq.numpy(), sections, interleaved)
    q, k = tensor(g, batch, hq, n, dtype, inner), tensor(g, batch, hk, n, dtype, inner) if hk else None
    q_up, k_up = tensor(g, batch, hq, n, dtype, not inner, 1.0), tensor(g, batch, hk, n, dtype, inner, 1.0) if hk else None
    wq, wk = weight(g, wdtype), weight(g, F32) if hk % 2 == 0 else None
    outs = [None if x is None else torch.full_like(x, float("nan")) for x in (q, k, q_up, k_up)]
    sums = [torch.full((D,), float("nan"), device="cuda") for _ in range(2)]
    B.norm_rope_apply(rope, q, outs[0], wq, k, outs[1], wk, eps=eps)
    ws = torch.empty(B.norm_rope_workspace_bytes(batch, n, hq, hk), dtype=torch.uint8, device="cuda")
    B.norm_rope_grad(rope, q, q_up, outs[2], ws, wq, sums[0], k, k_up, outs[3], wk, sums[1] if hk else None, eps=eps)
    for x, up, out, dx, w, dw in ((q, q_up, outs[0], outs[2], wq, sums[0]), (k, k_up, outs[1], outs[3], wk, sums[1])):
        if x is None:
            continue
        x64, w64, up64 = f64(x), np.ones(D) if w is None else f64(w), f64(up)
        ref, y = N.norm_rope(x64, w64, np.float64(np.float32(eps)), turn)
        assert (np.abs(f64(out) - ref) <= apply_bound(ref, y, dtype, turn)).all()
        gx, gw, u = N.norm_rope_grad(x64, w64, up64, np.float64(np.float32(eps)), turn)
        bx, bw = grad_bounds(x64, w64, up64, u, gx, dtype, eps, turn, 64)
        assert (np.abs(f64(dx) - gx) <= bx).all()
        assert (np.abs(f64(dw) - gw) <= bw).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("sections,interleaved", SECTIONS + [(None, False)])
def test_norm_and_gradient_match_the_formula(dtype, sections, interleaved):
    for shape in CASES:
        check(dtype, dtype, sections, interleaved, shape, 1e-6)


@pytest.mark.parametrize("dtype,wdtype", [(F16, F32), (F32, BF16), (BF16, F16)])
def test_weights_of_another_type(dtype, wdtype):
    check(dtype, wdtype, (24, 20, 20), True, CASES[1], 1e-5)


def test_many_rows():
    """More units of work than blocks: 5003 tokens, 13 heads; a thread adds up 8 heads of 1 or 2 tokens, 64 additions with the rest."""
    check(F32, F32, (24, 20, 20), True, (1, 9, 4, 5003, "near", True), 1e-6)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_in_place_and_strided(dtype):
    """q and k inside one projection [batch, n, (q heads | k heads | v heads) * 128]; the gradients in the place of the results'."""
    g = gen(2)
    rope = B.Rope(positions(g, 2, 19, "near").cuda(), B.rope_frequencies(1e4, 64), (16, 24, 24))
    qkv, up = (randn(g, 2, 19, 9, D, dtype=dtype).cuda() for _ in range(2))
    part = lambda x: (x[:, :, :5].transpose(1, 2), x[:, :, 5:7].transpose(1, 2))  # noqa: E731
    (q, k), (qu, ku) = part(qkv), part(up)
    wq, wk = weight(g, dtype), weight(g, dtype)
    ws = torch.empty(B.norm_rope_workspace_bytes(2, 19, 5, 2), dtype=torch.uint8, device="cuda")
    want = [torch.empty_like(x) for x in (q, k, q, k)]
    sums = [torch.empty(D, device="cuda") for _ in range(4)]
    B.norm_rope_apply(rope, q, want[0], wq, k, want[1], wk)
    B.norm_rope_grad(rope, q, qu, want[2], ws, wq, sums[0], k, ku, want[3], wk, sums[1])
    v, vu = qkv[:, :, 7:].clone(), up[:, :, 7:].clone()
    B.norm_rope_grad(rope, q, qu, qu, ws, wq, sums[2], k, ku, ku, wk, sums[3])
    B.norm_rope_apply(rope, q, q, wq, k, k, wk)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, 7:], v)
    assert torch.equal(qu, want[2]) and torch.equal(ku, want[3]) and torch.equal(up[:, :, 7:], vu)
    assert torch.equal(sums[0], sums[2]) and torch.equal(sums[1], sums[3])
    # one row for all heads and tokens
    one = randn(g, 1, 1, 1, D, dtype=dtype).cuda()
    out = torch.empty(2, 5, 19, D, dtype=dtype, device="cuda")
    B.norm_rope_apply(rope, one.expand(2, 5, 19, D), out, wq)
    full = torch.empty_like(out)
    B.norm_rope_apply(rope, one.expand(2, 5, 19, D).contiguous(), full, wq)
    assert torch.equal(out, full)


def test_same_numbers_as_the_norm_alone_and_the_rotation():
    """Without a turn at position 0, and, in fp32, the rotation of the normed numbers bit for bit."""
    g = gen(3)
    q, w = tensor(g, 2, 3, 41, F32, True), weight(g, F32)
    pos = positions(g, 2, 41, "near").cuda()
    freq = B.rope_frequencies(1e6, 64)
    normed, both, turned = (torch.empty_like(q) for _ in range(3))
    B.norm_rope_apply(None, q, normed, w)
    B.norm_rope_apply(B.Rope(pos * 0, freq, (16, 24, 24)), q, both, w)
    assert torch.equal(normed, both)
    rope = B.Rope(pos, freq, (16, 24, 24))
    B.norm_rope_apply(rope, q, both, w)
    B.rope_apply(rope, normed, turned)
    assert torch.equal(turned, both)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_rows_at_the_ends_of_the_range(dtype):
    """Zeros, the largest numbers of the type, numbers whose squares are zeros or infinite in fp32, infinities and NaN; other rows do not
    notice."""
    g = gen(4)
    x = randn(g, 1, 1, 12, D, dtype=F32)
    top = torch.finfo(dtype).max
    x[0, 0, 1] = 0
    x[0, 0, 2] = top * torch.sign(x[0, 0, 2])
    x[0, 0, 3] *= 1e-24
    x[0, 0, 4, 1:] = 0
    x[0, 0, 4, 0] = top
    x[0, 0, 5] *= 6e4 if dtype == F16 else 1e19
    x[0, 0, 6] *= 3e4 if dtype == F16 else 4e36
    x[0, 0, 7, 5] = float("inf")
    x[0, 0, 8, 100] = float("nan")
    x = x.clamp(-top, top).masked_fill(x == float("inf"), float("inf")).to(dtype)
    up, w, eps = randn(g, 1, 1, 12, D, dtype=dtype), weight(g, F32, 1.0), 1e-6
    out, dx, dw = torch.empty_like(x).cuda(), torch.empty_like(x).cuda(), torch.empty(D, device="cuda")
    ws = torch.empty(B.norm_rope_workspace_bytes(1, 12, 1), dtype=torch.uint8, device="cuda")
    B.norm_rope_apply(None, x.cuda(), out, w, eps=eps)
    B.norm_rope_grad(None, x.cuda(), up.cuda(), dx, ws, w, dw, eps=eps)
    fine = [i for i in range(12) if i not in (7, 8)]
    x64, w64, up64 = f64(x)[:, :, fine], f64(w), f64(up)[:, :, fine]
    ref, y = N.norm_rope(x64, w64, np.float64(np.float32(eps)))
    assert (np.abs(f64(out)[:, :, fine] - ref) <= apply_bound(ref, y, dtype, None)).all()
    gx, _, u = N.norm_rope_grad(x64, w64, up64, np.float64(np.float32(eps)))
    bx, _ = grad_bounds(x64, w64, up64, u, gx, dtype, eps, None, 64)
    got = f64(dx)[:, :, fine]
    # (a row of zeros has gradients of w g / sqrt(eps), 1000 times g: within every type's range; numbers below 2^-126 may be flushed)
    assert (np.abs(got - gx) <= bx + 2.0 ** -126).all()
    # 0 / inf in the other channels, inf * 0 in that one
    row = out[0, 0, 7].float()
    assert torch.isnan(row[5]) and (row[:5] == 0).all() and (row[6:] == 0).all() and torch.isnan(out[0, 0, 8]).all() and torch.isnan(dw).any()


def test_an_eps_beside_large_rows():
    """Rows whose squares have no sum in fp32, and an eps of their size."""
    g = gen(9)
    x, up = randn(g, 1, 1, 5, D, dtype=F32) * 2e18, randn(g, 1, 1, 5, D, dtype=F32)
    w, eps = weight(g, F32, 1.0), 1e37
    out, dx = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    B.norm_rope_apply(None, x.cuda(), out, w, eps=eps)
    B.norm_rope_grad(None, x.cuda(), up.cuda(), dx, None, w, eps=eps)
    ref, y = N.norm_rope(f64(x), f64(w), np.float64(np.float32(eps)))
    assert (np.abs(f64(out) - ref) <= apply_bound(ref, y, F32, None)).all()
    gx, _, u = N.norm_rope_grad(f64(x), f64(w), f64(up), np.float64(np.float32(eps)))
    assert (np.abs(f64(dx) - gx) <= grad_bounds(f64(x), f64(w), f64(up), u, gx, F32, eps, None, 64)[0]).all()


def test_gradient_agrees_with_differences():
    """The call's gradients against central differences of the formula in 64 bits (h = 1e-5: 1e-8 of the sum).  Roundings of fp32, 2^-18 of the
    products' magnitudes at most by the bound of the numbers."""
    g = gen(5)
    pos, freq = positions(g, 1, 23, "near"), B.rope_frequencies(1e4, 64, "cpu")
    turn = (pos.numpy(), freq.numpy(), (24, 20, 20), True)
    x, up, d = (tensor(g, 1, 3, 23, F32, False, 1.0) for _ in range(3))
    w, dw = weight(g, F32, 1.0), torch.randn(D, generator=g).cuda()
    dx, sums = torch.empty_like(x), torch.empty(D, device="cuda")
    ws = torch.empty(B.norm_rope_workspace_bytes(1, 23, 3), dtype=torch.uint8, device="cuda")
    B.norm_rope_grad(B.Rope(pos.cuda(), freq.cuda(), (24, 20, 20), True), x, up, dx, ws, w, sums)
    h, eps = 1e-5, np.float64(np.float32(1e-6))
    f = lambda a, b: (N.norm_rope(f64(x) + a * f64(d), f64(w) + b * f64(dw), eps, turn)[0] * f64(up)).sum()  # noqa: E731
    scale = np.abs(f64(up)).sum() * 4
    assert abs((f(h, 0) - f(-h, 0)) / (2 * h) - (f64(dx) * f64(d)).sum()) <= 2.0 ** -18 * scale
    assert abs((f(0, h) - f(0, -h)) / (2 * h) - (f64(sums) * f64(dw)).sum()) <= 2.0 ** -18 * scale


def test_no_rows_and_no_workspace():
    q = torch.empty(2, 3, 0, D, dtype=F16, device="cuda")
    sums = torch.full((D,), 7.0, device="cuda")
    B.norm_rope_apply(None, q, q)
    B.norm_rope_grad(None, q, q, q, None, None, sums)
    assert (sums == 0).all()
    # gradients of the inputs alone
    g = gen(6)
    x, up = (randn(g, 1, 2, 9, D, dtype=BF16).cuda() for _ in range(2))
    a, b = torch.empty_like(x), torch.empty_like(x)
    B.norm_rope_grad(None, x, up, a, None, weight(g, BF16))
    g = gen(6)
    [randn(g, 1, 2, 9, D, dtype=BF16) for _ in range(2)]
    ws = torch.empty(B.norm_rope_workspace_bytes(1, 9, 2), dtype=torch.uint8, device="cuda")
    B.norm_rope_grad(None, x, up, b, ws, weight(g, BF16), sums)
    assert torch.equal(a, b) and (sums != 0).any()


def test_other_stream_and_graph():
    """Calls on a stream of their own, captured and replayed with other inputs, give the same numbers each time."""
    g = gen(7)
    rope = B.Rope(positions(g, 3, 65, "near").cuda(), B.rope_frequencies(1e6, 64), (24, 20, 20), True)
    q, k, qu, ku = (tensor(g, 3, h, 65, BF16, True) for h in (8, 2, 8, 2))
    wq, wk = weight(g, BF16), weight(g, BF16)
    ws = torch.empty(B.norm_rope_workspace_bytes(3, 65, 8, 2), dtype=torch.uint8, device="cuda")
    make = lambda: [torch.empty_like(x) for x in (q, k, qu, ku)] + [torch.empty(D, device="cuda") for _ in range(2)]  # noqa: E731
    def both(o, stream=None):
        B.norm_rope_apply(rope, q, o[0], wq, k, o[1], wk, stream=stream)
        B.norm_rope_grad(rope, q, qu, o[2], ws, wq, o[4], k, ku, o[3], wk, o[5], stream=stream)
    want, got = make(), make()
    both(want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    both(got, s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph, out = torch.cuda.CUDAGraph(), make()
    with torch.cuda.graph(graph):
        both(out)
    for i in range(2):
        q.mul_(0.5)
        both(want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_keys_alone_and_queries_alone(dtype):
    """A side without heads; its weight's gradient is zeros.  The other side's numbers are those of a call with both."""
    g = gen(8)
    rope = B.Rope(positions(g, 2, 21, "near").cuda(), B.rope_frequencies(1e6, 64), (24, 20, 20), True)
    q, k, qu, ku = (tensor(g, 2, h, 21, dtype, True) for h in (5, 3, 5, 3))
    wq, wk = weight(g, dtype), weight(g, dtype)
    ws = torch.empty(B.norm_rope_workspace_bytes(2, 21, 5, 3), dtype=torch.uint8, device="cuda")
    both, alone = [torch.empty_like(x) for x in (q, k, q, k)], [torch.empty_like(x) for x in (q, k, q, k)]
    none = torch.empty(2, 0, 21, D, dtype=dtype, device="cuda")
    sums = torch.full((2, D), 7.0, device="cuda")
    B.norm_rope_apply(rope, q, both[0], wq, k, both[1], wk)
    B.norm_rope_grad(rope, q, qu, both[2], ws, wq, sums[0], k, ku, both[3], wk, sums[1])
    B.norm_rope_apply(rope, none, none, wq, k, alone[1], wk)
    B.norm_rope_apply(rope, q, alone[0], wq)
    sums[0] = 7.0
    B.norm_rope_grad(rope, none, none, none, ws, wq, sums[0], k, ku, alone[3], wk)
    assert (sums[0] == 0).all()
    B.norm_rope_grad(rope, q, qu, alone[2], ws, wq)
    assert all(torch.equal(a, b) for a, b in zip(both, alone))


def test_a_threads_first_call_may_be_a_captured_one():
    """What the library asks the device about once per thread is asked in a capture here; two graphs share a workspace."""
    g = gen(10)
    q, up = tensor(g, 2, 6, 33, BF16, True), tensor(g, 2, 6, 33, BF16, True)
    w, ws = weight(g, BF16), torch.empty(B.norm_rope_workspace_bytes(2, 33, 6), dtype=torch.uint8, device="cuda")
    make = lambda: [torch.empty_like(q), torch.empty_like(q), torch.empty(D, device="cuda")]  # noqa: E731
    want, got, graphs, failed = make(), [make(), make()], [torch.cuda.CUDAGraph() for _ in range(2)], []

    def both(o):
        B.norm_rope_apply(None, q, o[0], w)
        B.norm_rope_grad(None, q, up, o[1], ws, w, o[2])

    def capture():
        try:
            for o, graph in zip(got, graphs):
                with torch.cuda.graph(graph):
                    both(o)
        except BaseException as e:   # noqa: BLE001
            failed.append(e)
    t = threading.Thread(target=capture)
    t.start()
    t.join()
    assert not failed
    for graph in graphs:
        ws.fill_(0xff)
        graph.replay()
    both(want)
    assert all(torch.equal(a, b) for o in got for a, b in zip(o, want))
