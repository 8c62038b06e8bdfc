"""Attention with a window and for trees of drafted tokens over the 8-bit paged cache, and sliding pages, on the GPU against the oracle in
64 bits."""
import random
import threading

import numpy as np
import pytest
import torch

from oracle import okq_norm_oracle as N
from oracle import okq_paged_oracle as O
from oracle import okq_sight_oracle as S
from paper_2609_11582_b200 import binding as B
from tests.test_gpu_norm import apply_bound
from tests.test_gpu_paged import BF16, BLOCK, D, F16, Model, f64, gen, positions, randn, random_cache
from tests.test_gpu_paged_numbers import Store, kernel_bound, lift, steered

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731


def scratch(c, layers, n, fill=0xff):
    return torch.full((B.paged_workspace_bytes(c, layers, n),), fill, dtype=torch.uint8, device="cuda")


def held(c, l, b, T):
    """[H, 2, T, 128] what the codes stand for and [H, T] the largest magnitude of a token's values' block, 64 bits; pages that are missing
    hold zeros."""
    P = c.page_tokens
    pages = c.table[b, :(T + P - 1) // P].long()
    scales = c.scales[l, pages.clamp(min=0)].double() * (pages >= 0)[:, None, None, None]
    x = c.codes[l, pages.clamp(min=0)].double().unflatten(3, (-1, BLOCK)) * scales[..., None, None]
    x = torch.where(scales[..., None, None] == 0, 0.0, x)
    return x.flatten(3, 4).permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :T], (scales * 127).repeat_interleave(BLOCK, -1).permute(1, 2, 0, 3).flatten(2, 3)[:, 1, :T]


def check(c, q, out, q_len, poison, plan, mask_of, layer=0, sm_scale=None):
    """mask_of(b, T, m): bool [m, T]"""
    G, n, scale = c.n_q_heads // c.n_kv_heads, q.shape[3], D ** -0.5 if sm_scale is None else sm_scale
    for l in range(q.shape[0]):
        lens = c.seq_len[layer + l].tolist()
        for b, T in enumerate(lens):
            m = n if q_len is None else max(0, min(n, q_len[b]))
            assert (out[l, b, :, m:] == poison).all()
            if m == 0:
                continue
            see = torch.as_tensor(mask_of(b, T, m)).cuda()
            if T == 0 or not see.any():
                assert (out[l, b, :, :m] == 0).all()
                continue
            x, amax = held(c, layer + l, b, T)
            s = torch.einsum("hgnd,htd->hgnt", q[l, b, :, :m].double().unflatten(0, (-1, G)), x[:, 0]) * scale
            top = s.masked_fill(~see, 0.0).abs().amax(-1).flatten(1)
            w = torch.softmax(s.masked_fill(~see, -torch.inf), -1).nan_to_num(0.0).flatten(1, 2)
            ref, got = w @ x[:, 1], out[l, b, :, :m].double().unflatten(0, (-1, G)).flatten(1, 2)
            limit = kernel_bound(w, x[:, 1], ref, amax, top, q.dtype, plan)
            assert ((got - ref).abs() <= limit).all(), (l, b, T, m, plan, ((got - ref).abs() / limit).max().item())


def lengths(g, batch, longest, ragged):
    lens = [longest] * batch
    if ragged:
        lens = [int(longest * x ** 2) for x in torch.rand(batch, generator=g).tolist()]
        lens[-1] = 0
        lens[0] = min(longest, 1 + lens[0])
    return lens


# ------------------------------------------------------------------------------------------------ windows
# (layers, batch, KV heads, group, page, queries, longest, windows with sinks)
WINDOWS = [(1, 1, 1, 7, 64, 1, 2048, [(350, 4), (1, 0), (127, 1), (128, 128), (2047, 0)]), (1, 5, 2, 8, 32, 1, 700, [(33, 0), (200, 33), (1, 300)]),
           (2, 30, 4, 7, 64, 1, 3000, [(1000, 4), (129, 0), (512, 513)]), (28, 9, 4, 7, 32, 1, 700, [(100, 1), (400, 64)]),
           (1, 16, 4, 8, 128, 2, 9000, [(4096, 4), (31, 0)]), (1, 3, 2, 4, 256, 5, 1500, [(64, 5), (700, 0), (1, 1)]), (1, 40, 4, 7, 32, 3, 2500, [(300, 40)]),
           (1, 16, 4, 7, 64, 5, 5000, [(511, 1), (64, 0), (3000, 1)]), (1, 5, 3, 5, 32, 40, 1000, [(1, 0), (16, 3), (333, 129)]),
           (1, 2, 2, 7, 64, 300, 2500, [(64, 4), (1000, 0), (2048, 65), (5, 2000)]), (1, 3, 1, 8, 128, 1000, 1100, [(100, 4), (901, 0)]),
           (3, 2, 2, 1, 64, 130, 4000, [(1000, 1), (17, 64)]), (1, 1, 4, 8, 64, 2048, 2048, [(257, 4), (1, 0)])]


@pytest.mark.parametrize("shape", WINDOWS, ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_window(shape, dtype):
    L, batch, H, G, page, n, longest, sights = shape
    g = gen(longest + n)
    for ragged in (False, True):
        lens = lengths(g, batch, longest, ragged)
        q_len = None if not ragged else torch.randint(-1, n + 2, (batch,), generator=g).tolist()
        c = random_cache(g, L, batch, H, H * G, page, dtype, lens)
        q, ql, ws = randn(g, L, batch, H * G, n, D, dtype=dtype).cuda(), None if q_len is None else i32(q_len), scratch(c, L, n)
        for window, sinks in sights:
            out, again = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
            B.paged_attention_window(c, 0, L, q, ws, out, window, sinks, ql)
            B.paged_attention_window(c, 0, L, q, ws, again, window, sinks, ql)
            assert c.device_status() == 0 and torch.equal(out, again)
            check(c, q, out, q_len, 5.0, B.paged_plan_window(c, L, n, window, sinks), lambda b, T, m: S.window_mask(T, m, window, sinks))


def test_windows_reach_their_kernels():
    """A short window makes short items of long rows: a cluster to each, where the whole row would go to the line; few rows of prompts too."""
    def plans(L, batch, H, Hq, tokens, n, window, sinks=4):
        c = B.PagedCache(L, batch, H, Hq, 4, (tokens + 63) // 64, 64)
        return B.paged_plan(c, L, n), B.paged_plan_window(c, L, n, window, sinks)
    assert plans(1, 1, 1, 7, 2048, 1, 350) == (8, 8) and plans(1, 1, 4, 28, 131072, 1, 1000)[0] == B.PLAN_LINE < 0 < plans(1, 1, 4, 28, 131072, 1, 1000)[1]
    assert plans(28, 8, 4, 28, 4096, 1, 1000)[1] == B.PLAN_LINE and plans(1, 16, 4, 28, 12345, 5, 511)[1] == B.PLAN_PROMPT
    assert plans(1, 1, 4, 28, 8192, 2048, 1400)[1] == B.PLAN_PROMPT


@pytest.mark.parametrize("n", [1, 3, 40])
def test_window_of_the_whole_row_is_none(n):
    g = gen(3)
    c = random_cache(g, 1, 3, 2, 14, 64, BF16, [900, 500, 1])
    q, ws = randn(g, 1, 3, 14, n, D, dtype=BF16).cuda(), scratch(c, 1, n)
    want = torch.zeros_like(q)
    B.paged_attention(c, 0, 1, q, ws, want)
    room = c.max_pages * 64
    for window, sinks in ((room, 0), (0x7fffffff, 5), (1, room), (7, 0x7fffffff)):
        out = torch.zeros_like(q)
        B.paged_attention_window(c, 0, 1, q, ws, out, window, sinks)
        assert torch.equal(out, want)


@pytest.mark.parametrize("n", [1, 4, 60])
@pytest.mark.parametrize("page", [32, 128])
def test_pages_out_of_sight_need_not_be_there(page, n):
    """Missing pages, and blocks whose scales are NaN, where no query sees them; then where one does."""
    g = gen(n)
    T, window, sinks = 2000, 300, 40
    for batch in (2, 40):                                                       # clusters and the line
        c = random_cache(g, 1, batch, 2, 10, page, F16, [T] * batch)
        q, ws = randn(g, 1, batch, 10, n, D).cuda(), scratch(c, 1, n)
        want, out = torch.zeros_like(q), torch.zeros_like(q)
        B.paged_attention_window(c, 0, 1, q, ws, want, window, sinks)
        first, last = -(-sinks // page), (T - n - window + 1) // page           # whole pages that nobody sees
        c.table[1, first:last] = -1
        mine = c.table[0, first:last].long()
        c.scales[0, mine] = float("nan")
        # the part of the first page behind the sinks, by blocks
        blocks = -(-sinks // BLOCK)
        c.scales[0, c.table[0, sinks // page].long(), :, :, blocks % (page // BLOCK) if blocks % (page // BLOCK) else page // BLOCK:] = float("nan")
        B.paged_attention_window(c, 0, 1, q, ws, out, window, sinks)
        assert torch.equal(out, want) and c.device_status() == 0
        c.scales[0, c.table[0, (T - window) // page].long()] = float("nan")     # the newest query sees one of these
        c.table[1, (T - 1) // page] = -1
        B.paged_attention_window(c, 0, 1, q, ws, out, window, sinks)
        assert torch.isnan(out[0, 0, :, n - 1]).all() and torch.isnan(out[0, 1, :, n - 1]).all() and c.device_status() == B.ERR_INVALID_ARG


@pytest.mark.parametrize("n", [1, 40])
def test_lost_blocks_reach_the_rows_that_see_them(n):
    """A NaN scale of values: rows whose window has left it, and rows that see it as a sink."""
    g = gen(7)
    T, window = 700, 200
    c = random_cache(g, 1, 2, 1, 8, 64, BF16, [T, T])
    at = T - window - 10                                                        # its block ends before the newest query's window begins
    p, blk = c.table[0, at // 64].long(), at % 64 // BLOCK
    c.scales[0, p, :, 1, blk] = float("nan")
    q, ws = randn(g, 1, 2, 8, n, D, dtype=BF16).cuda(), scratch(c, 1, n)
    for sinks in (0, at + 1):
        out = torch.zeros_like(q)
        B.paged_attention_window(c, 0, 1, q, ws, out, window, sinks)
        see = S.window_mask(T, n, window, sinks)[:, at // BLOCK * BLOCK:at // BLOCK * BLOCK + BLOCK].any(1)
        assert torch.isnan(out[0, 0][:, see]).all() and torch.isfinite(out[0, 0][:, ~see]).all() and torch.isfinite(out[0, 1]).all()


def test_window_rope_strides_scale_and_stream():
    m = Model(2, 3, 2, 6, max_pages=4, page=64, dtype=BF16)
    m.append(200, [200, 64, 3])
    for n in (1, 4, 50):
        rope = B.Rope(positions(m.g, 3, n, "near").cuda(), B.rope_frequencies(1e6, 64), (24, 20, 20), True)
        x = randn(m.g, 2, 3, n, 6, D, dtype=BF16).cuda()                        # [batch, n, heads * 128] in and out
        turned = x.transpose(2, 3).clone()
        for l in range(2):
            B.rope_apply(rope, turned[l], turned[l])
        out, ws, s = torch.full_like(x, 7.0), scratch(m.c, 2, n), torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        B.paged_attention_window(m.c, 0, 2, x.transpose(2, 3), ws, out.transpose(2, 3), 50, 3, rope=rope, sm_scale=-0.07, stream=s)
        s.synchronize()
        check(m.c, turned, out.transpose(2, 3), None, 7.0, B.paged_plan_window(m.c, 2, n, 50, 3), lambda b, T, k: S.window_mask(T, k, 50, 3), sm_scale=-0.07)


# ------------------------------------------------------------------------------------------------ trees
def random_tree(rng, n):
    return [max(-1, min(i - 1, int((i + 1) * rng.random() ** 1.5) - 1)) for i in range(n)]


def to_words(seen, n):
    """Python's whole numbers as int64 words"""
    words = (n + 63) // 64
    return [[(s >> 64 * w & (1 << 64) - 1) - (1 << 64 if s >> 64 * w + 63 & 1 else 0) for w in range(words)] for s in seen]


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 200, 4096])
def test_ancestors(n):
    rng = random.Random(n)
    trees = [random_tree(rng, n), list(range(-1, n - 1)), [-1] * n, random_tree(rng, n)]
    q_len = [n, n, n, n // 2]
    c = B.PagedCache(1, 4, 1, 1, 2, 2)
    seen = torch.full((4, n, (n + 63) // 64), 77, dtype=torch.int64, device="cuda")
    depth = torch.full((4, n), 77, dtype=torch.int32, device="cuda")
    B.tree_ancestors(c, i32(trees), seen, depth, q_len=i32(q_len))
    for b in range(4):
        want, d, _ = S.ancestors(trees[b])
        assert seen[b, :q_len[b]].tolist() == to_words(want, n)[:q_len[b]] and depth[b, :q_len[b]].tolist() == d[:q_len[b]]
        assert (seen[b, q_len[b]:] == 77).all() and (depth[b, q_len[b]:] == 77).all()
    assert c.device_status() == 0


def test_ancestors_of_bad_parents():
    c = B.PagedCache(1, 5, 1, 1, 2, 2)
    trees = [[-1, 0, 1], [-1, 1, 0], [0, 0, 0], [-1, -2, 1], [-1, 0, 2]]
    seen = torch.zeros(5, 3, 1, dtype=torch.int64, device="cuda")
    B.tree_ancestors(c, i32(trees), seen, q_len=i32([3, 0, 0, 0, 2]))           # those with wrong ones are not looked at
    assert c.device_status() == 0 and seen[:, :, 0].tolist() == [[1, 3, 7], [0, 0, 0], [0, 0, 0], [0, 0, 0], [1, 3, 0]]
    B.tree_ancestors(c, i32(trees), seen)
    assert c.device_status() == B.ERR_INVALID_ARG
    assert seen[:, :, 0].tolist() == [S.ancestors(t)[0] for t in trees]


# (layers, batch, KV heads, group, page, nodes, longest)
TREES = [(1, 1, 1, 7, 64, 1, 500), (1, 1, 1, 7, 64, 2, 2048), (1, 5, 2, 4, 32, 4, 700), (1, 40, 4, 7, 32, 2, 2500), (28, 9, 2, 5, 64, 3, 300), (1, 1, 4, 8, 64, 3, 900),
         (1, 2, 1, 1, 32, 16, 130), (1, 8, 4, 7, 64, 16, 4000), (1, 3, 2, 7, 128, 64, 1000), (2, 2, 1, 8, 32, 65, 333), (1, 2, 2, 3, 64, 128, 1500), (1, 1, 1, 8, 256, 200, 5000),
         (1, 3, 3, 1, 64, 129, 700), (1, 1, 1, 1, 32, 700, 900), (1, 60, 8, 8, 32, 7, 200)]


@pytest.mark.parametrize("shape", TREES, ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_tree(shape, dtype):
    L, batch, H, G, page, n, longest = shape
    g, rng = gen(longest + n), random.Random(longest + n)
    for ragged in (False, True):
        lens = lengths(g, batch, longest, ragged)                               # (ragged: some have fewer tokens than nodes)
        q_len = None if not ragged else torch.randint(-1, n + 2, (batch,), generator=g).tolist()
        c = random_cache(g, L, batch, H, H * G, page, dtype, lens)
        q, ql, ws = randn(g, L, batch, H * G, n, D, dtype=dtype).cuda(), None if q_len is None else i32(q_len), scratch(c, L, n)
        trees = [random_tree(rng, n) for _ in range(batch)]
        sets = [S.ancestors(t)[0] for t in trees]
        seen = torch.zeros(batch, n, (n + 63) // 64, dtype=torch.int64, device="cuda")
        B.tree_ancestors(c, i32(trees), seen)
        for anything in (False, True):
            if anything:                                                        # any bits, in any order, some rows without one
                sets = [[rng.getrandbits(64 * ((n + 63) // 64)) if rng.random() < 0.8 else 0 for _ in range(n)] for _ in range(batch)]
                seen.copy_(torch.tensor([to_words(s, n) for s in sets]))
            out, again = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
            B.paged_attention_tree(c, 0, L, q, ws, out, seen, ql)
            B.paged_attention_tree(c, 0, L, q, ws, again, seen, ql)
            assert c.device_status() == 0 and torch.equal(out, again)
            check(c, q, out, q_len, 5.0, B.paged_plan(c, L, n), lambda b, T, m: S.tree_mask(T, m, sets[b]))


def test_trees_reach_their_kernels():
    plans = set()
    for L, batch, H, G, page, n, longest in TREES:
        p = B.paged_plan(B.PagedCache(L, batch, H, H * G, 4, (longest + page - 1) // page, page), L, n)
        plans.add("cluster" if p > 0 else p)
    assert plans == {"cluster", B.PLAN_LINE, B.PLAN_PROMPT}


def test_masked_nodes_with_lost_scales():
    """A node's block whose values are NaN: only rows that see a token of it notice; a block of nodes alone."""
    g = gen(5)
    n, T = 40, 96 + 40                                                          # the nodes' first block begins with node 0
    for G, batch in ((1, 1), (8, 3)):
        c = random_cache(g, 1, batch, 1, G, 32, F16, [T] * batch)
        c.scales[0, c.table[0, 4].long(), :, 1] = float("nan")                  # nodes 32 .. 39
        sets = [(1 << i) | (1 << 39 if i % 3 == 0 else 0) for i in range(n)]
        seen = torch.tensor([to_words(sets, n)] * batch).cuda()
        q, ws = randn(g, 1, batch, G, n, D).cuda(), scratch(c, 1, n)
        out = torch.zeros_like(q)
        B.paged_attention_tree(c, 0, 1, q, ws, out, seen)
        lost = torch.tensor([s >> 32 != 0 for s in sets])
        assert torch.isnan(out[0, 0][:, lost]).all() and torch.isfinite(out[0, 0][:, ~lost]).all() and torch.isfinite(out[0, 1:]).all()


# ------------------------------------------------------------------------------------------------ graphs
@pytest.mark.parametrize("n", [1, 3, 64])
def test_graphs_share_a_workspace(n):
    """A window's and a tree's call, captured with one workspace, replayed after the cache has grown and slid; equal to eager calls bit for bit."""
    m = Model(2, 3, 2, 14, max_pages=8, page=64, dtype=F16)
    m.append(300, [300, 64, 0])
    rng = random.Random(n)
    q = randn(m.g, 2, 3, 14, n, D).cuda()
    outs, ws = [torch.zeros_like(q[:1]) for _ in range(2)], scratch(m.c, 1, n)
    seen, parents = torch.zeros(3, n, (n + 63) // 64, dtype=torch.int64, device="cuda"), i32([random_tree(rng, n) for _ in range(3)])

    def call(i):
        if i == 0:
            B.paged_attention_window(m.c, 0, 1, q[:1], ws, outs[0], 100, 5)
        else:
            B.tree_ancestors(m.c, parents, seen)
            B.paged_attention_tree(m.c, 1, 1, q[1:], ws, outs[1], seen)
    call(0), call(1)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(3)]
    for i in (0, 1):
        with torch.cuda.graph(graphs[i]):
            call(i)
    with torch.cuda.graph(graphs[2]):
        B.pages_slide(m.c, 100, 5)
    m.append(150, [150, 150, 1])
    for _ in range(2):
        parents.copy_(i32([random_tree(rng, n) for _ in range(3)]))
        for i in (1, 0):
            ws.fill_(0xff)
            graphs[i].replay()
        got = [o.clone() for o in outs]
        for i in (0, 1):
            call(i)
            assert torch.equal(outs[i], got[i])
        graphs[2].replay()
    assert m.c.seq_len[0].tolist() == [T - 64 * S.slide(T, 64, 100, 5)[1] for T in (450, 214, 1)] == [450 - 64 * 4, 214, 1] and m.c.device_status() == 0


@pytest.mark.parametrize("n", [1, 5, 64])
def test_a_threads_first_call_may_be_a_captured_one(n):
    m = Model(1, 2, 2, 14, max_pages=6, page=64, dtype=F16)
    m.append(200, [200, 64])
    q, ws = randn(m.g, 1, 2, 14, n, D).cuda(), scratch(m.c, 1, n)
    seen = torch.tensor([to_words([1 << i for i in range(n)], n)] * 2).cuda()
    want, got, graph, failed = [torch.zeros_like(q) for _ in range(2)], [torch.zeros_like(q) for _ in range(2)], torch.cuda.CUDAGraph(), []

    def both(o):
        B.paged_attention_window(m.c, 0, 1, q, ws, o[0], 70, 2)
        B.paged_attention_tree(m.c, 0, 1, q, ws, o[1], seen)

    def capture():
        try:
            with torch.cuda.graph(graph):
                both(got)
        except BaseException as e:   # noqa: BLE001
            failed.append(e)
    t = threading.Thread(target=capture)
    t.start()
    t.join()
    assert not failed
    graph.replay()
    both(want)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_calls_at_once_on_two_streams():
    """Two sequences' worth of calls next to one another, each with its own workspace, give what they give alone."""
    g = gen(31)
    jobs = []
    for n, window in ((1, 300), (5, 200), (70, 450), (3, None), (40, None)):
        c = random_cache(g, 1, 3, 2, 14, 64, BF16, [2000, 900, 64])
        q = randn(g, 1, 3, 14, n, D, dtype=BF16).cuda()
        seen = torch.tensor([to_words([1 << i | i for i in range(n)], n)] * 3).cuda()
        jobs.append((c, q, n, window, seen, [scratch(c, 1, n) for _ in range(2)], [torch.zeros_like(q) for _ in range(3)]))

    def call(job, which, out, stream=None):
        c, q, n, window, seen, ws, outs = job
        if window:
            B.paged_attention_window(c, 0, 1, q, ws[which], outs[out], window, 4, stream=stream)
        else:
            B.paged_attention_tree(c, 0, 1, q, ws[which], outs[out], seen, stream=stream)
    for job in jobs:
        call(job, 0, 0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for k in range(len(jobs)):
            call(jobs[k], 0, 1, streams[0])
            call(jobs[-1 - k], 1, 2, streams[1])
    torch.cuda.synchronize()
    for job in jobs:
        assert torch.equal(job[6][0], job[6][1]) and torch.equal(job[6][0], job[6][2]) and job[0].device_status() == 0


# ------------------------------------------------------------------------------------------------ values of very different sizes
@pytest.mark.parametrize("seed", range(6))
def test_numbers_behind_masks(seed):
    """Windows and any bits over keys and values with zeros, values from 1e-20 to 1e9 and tokens that take all of the weight, in stretches that
    masks cut: each row by its kernel's own bound."""
    rng = random.Random(seed)
    for shape in ((150, 2, 4, 8, 2500, True), (16, 2, 2, 16, 3000 + seed, True), (1, 24, 8, 56, 2500, True), (3, 24, 8, 40, 2500, True), (8, 1, 1, 2, 8000, False)):
        n, batch, H, Hq, T, wide = shape
        q, k, v = steered(*shape, seed=seed, spread=rng.choice([0.5, 1.0, 3.0, 8.0]))
        for _ in range(rng.randint(1, 4)):
            a = rng.randrange(T)
            b = min(T, a + rng.choice([1, 32, 128, 300, 1000]))
            what = rng.choice(["size", "zeros", "lift", "sink"])
            if what == "size":
                v[..., a:b, :] *= 10.0 ** rng.choice([-20, -9, -6, -4, 4, 9])
            elif what == "zeros":
                v[..., a:b, :] = 0
            elif what == "lift":
                k[..., a:b, 0] = lift(rng.choice([-90.0, -30.0, 20.0, 60.0, 300.0]))
            else:
                k[..., a, 0] = lift(rng.choice([30.0, 100.0]))
                v[..., a, :] = 0
        c = Store(k, v, Hq, wide, seed=seed).c
        q, ws = q.cuda(), scratch(c, 1, n)
        window, sinks = max(1, int(T ** rng.random())), rng.choice([0, 1, 4, 100, 700])
        sets = [[rng.getrandbits(64 * ((n + 63) // 64)) for _ in range(n)] for _ in range(batch)]
        out = torch.full_like(q, 5.0)
        B.paged_attention_window(c, 0, 1, q, ws, out, window, sinks)
        check(c, q, out, None, 5.0, B.paged_plan_window(c, 1, n, window, sinks), lambda b, T, m: S.window_mask(T, m, window, sinks))
        B.paged_attention_tree(c, 0, 1, q, ws, out, torch.tensor([to_words(x, n) for x in sets]).cuda())
        check(c, q, out, None, 5.0, B.paged_plan(c, 1, n), lambda b, T, m: S.tree_mask(T, m, sets[b]))
        assert c.device_status() == 0


# ------------------------------------------------------------------------------------------------ few rows in the prompt kernel
# (layers, batch, KV heads, group, queries, longest): up to 128 rows to a head; items of one tile, and such that are cut
NARROW = [(1, 40, 4, 7, 5, 400), (18, 28, 8, 4, 9, 12), (1, 3, 2, 8, 16, 9000), (1, 1, 1, 8, 4, 60000), (2, 33, 4, 7, 18, 1500)]


@pytest.mark.parametrize("shape", NARROW, ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_up_to_128_rows(shape, dtype):
    L, batch, H, G, n, longest = shape
    g = gen(longest + n)
    for ragged in (False, True):
        lens = lengths(g, batch, longest, ragged)
        q_len = None if not ragged else torch.randint(-1, n + 2, (batch,), generator=g).tolist()
        c = random_cache(g, L, batch, H, H * G, 64, dtype, lens)
        q, ws = randn(g, L, batch, H * G, n, D, dtype=dtype).cuda(), scratch(c, L, n)
        plan = B.paged_plan(c, L, n)
        assert ragged or plan == B.PLAN_PROMPT
        out = torch.full_like(q, 5.0)
        B.paged_attention(c, 0, L, q, ws, out, None if q_len is None else i32(q_len))
        assert c.device_status() == 0
        check(c, q, out, q_len, 5.0, plan, lambda b, T, m: S.window_mask(T, m, 1 << 30, 0))


@pytest.mark.parametrize("batch,H,n,tokens", [(40, 4, 5, 1000), (3, 2, 16, 9000)])
def test_waits_are_bounded_with_few_rows(batch, H, n, tokens):
    """As for the other kernels: with nothing delivered every role's wait runs out, and the device goes on."""
    g = gen(11)
    c = random_cache(g, 1, batch, H, 7 * H, 64, F16, [tokens] * batch)
    assert B.paged_plan(c, 1, n) == B.PLAN_PROMPT
    q = randn(g, 1, batch, 7 * H, n, D).cuda()
    out, ws = torch.zeros_like(q), scratch(c, 1, n)
    B.debug_paged_timeout(c, 0, 1, q, ws, out, limit_clocks=2_000_000)
    torch.cuda.synchronize()
    assert c.device_status() == B.ERR_TIMEOUT and torch.isnan(out).all()
    c.status.zero_()
    out.fill_(5.0)
    B.paged_attention(c, 0, 1, q, ws, out)
    check(c, q, out, None, 5.0, B.PLAN_PROMPT, lambda b, T, m: S.window_mask(T, m, 1 << 30, 0))
    assert c.device_status() == 0


# ------------------------------------------------------------------------------------------------ pages that slide
@pytest.mark.parametrize("page,max_pages,batch", [(32, 9, 40), (64, 40, 7), (32, 3001, 5), (256, 3, 300)])
def test_slide_against_lists(page, max_pages, batch):
    """Tables, counts and lengths after calls in a row, with pages that sequences share."""
    rng = random.Random(page)
    c = B.PagedCache(2, batch, 1, 1, batch * max_pages, max_pages, page)
    table, lens, refs = [], [], [0] * (batch * max_pages)
    order = list(range(batch * max_pages))
    rng.shuffle(order)
    for b in range(batch):
        n = rng.choice([0, 1, max_pages * page, rng.randint(0, max_pages * page)])
        ahead = rng.randint(0, 2)                                               # pages reserved beyond the length
        row = [order[b * max_pages + j] if j < min(max_pages, -(-n // page) + ahead) else -1 for j in range(max_pages)]
        if b % 3 == 2:                                                          # some of the row before
            k = rng.randint(0, max_pages)
            row = [p if p >= 0 and j < k and row[j] >= 0 else row[j] for j, p in enumerate(table[b - 1])]
        table.append(row)
        lens.append([n, max(0, n - rng.choice([0, 0, 1, page]))])
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    c.table.copy_(i32(table)), c.refs.copy_(i32(refs)), c.seq_len.copy_(i32(lens).t())
    for window, sinks in ((max_pages * page, 0), (7 * page + 3, page), (3 * page, 2 * page - 1), (page, 1), (1, 4), (1, 0), (1, 0x7fffffff), (0x7fffffff, 0), (1, 0)):
        dropped = torch.full((batch,), 99, dtype=torch.int32, device="cuda")
        B.pages_slide(c, window, sinks, dropped if sinks != 1 else None)
        lost = []
        for b in range(batch):
            first, gone = S.slide(min(lens[b]), page, window, sinks)
            for p in table[b][first:first + gone]:
                if p >= 0:
                    refs[p] -= 1
            if gone:
                table[b] = table[b][:first] + table[b][first + gone:] + [-1] * gone
            lens[b] = [n - gone * page for n in lens[b]]
            lost.append(gone * page)
        assert c.table.tolist() == table and c.refs.tolist() == refs and c.seq_len.t().tolist() == lens
        assert sinks == 1 or dropped.tolist() == lost
    assert c.device_status() == 0


def test_slide_with_counts_that_do_not_match():
    c = B.PagedCache(1, 3, 1, 1, 8, 4, 32)
    c.table.copy_(i32([[0, 1, 2, 3], [8, 4, 5, -1], [-1, 6, 7, -1]]))
    c.refs.copy_(i32([0, 1, 1, 1, 1, 1, 1, 1]))
    c.seq_len.fill_(96)
    B.pages_slide(c, 32, 0)                                                     # page 0 is counted nowhere, page 8 is none
    assert c.device_status() == B.ERR_INVALID_ARG and c.refs.tolist() == [0, 0, 1, 1, 0, 1, 0, 1]
    assert c.table.tolist() == [[2, 3, -1, -1], [5, -1, -1, -1], [7, -1, -1, -1]] and c.seq_len.tolist() == [[32, 32, 32]]


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,page", [(F16, 32), (BF16, 64)])
def test_streaming_run(dtype, page):
    """A model with normed heads, positions and a window: a prompt in two pieces, then tokens one by one; after each the pages slide.  What is
    attended to is checked against the sequence as it would be without any page given up."""
    L, batch, H, G, window, sinks = 2, 3, 2, 7, 100, 3
    # a full copy that never slides, and the cache with room for a window only
    full = B.PagedCache(L, batch, H, H * G, 3 * 20, 20, page, dtype)
    c = B.PagedCache(L, batch, H, H * G, 3 * 9, 9, page, dtype)
    B.pages_reserve(full, i32([20 * page] * 3))
    g, freq, total, lost = gen(21), B.rope_frequencies(1e6, 64), [0] * 3, [0] * 3
    w = [(1 + 0.3 * torch.randn(2, D, generator=g)).to(dtype).cuda() for _ in range(L)]
    for n, news in ((110, [110, 60, 0]), (90, [90, 90, 33]), *[(1, [1, 1, 1])] * 80, (4, [4, 2, 1])):
        start = torch.tensor(total)
        rope = B.Rope((torch.arange(n) + start[:, None]).int().expand(3, batch, n).contiguous().cuda(), freq, (24, 20, 20), True)
        B.pages_reserve(c, i32([t - d + k for t, d, k in zip(total, lost, news)]))
        outs = []
        for l in range(L):
            x, k = (randn(g, batch, h, n, D, dtype=dtype, scale=3.0).cuda() for h in (H * G, H))
            v = randn(g, 1, batch, H, n, D, dtype=dtype, scale=0.3).cuda()
            q = torch.empty_like(x)
            x64 = f64(x)
            B.norm_rope_apply(rope, x, q, w[l][0], k, k, w[l][1])
            turn = (rope.positions.cpu().numpy(), freq.cpu().numpy(), (24, 20, 20), True)
            ref, y = N.norm_rope(x64, f64(w[l][0]), np.float64(np.float32(1e-6)), turn)
            assert (np.abs(f64(q) - ref) <= apply_bound(ref, y, dtype, turn)).all()
            for to in (c, full):
                B.paged_append(to, l, 1, k[None], v, i32(news))
            out = torch.zeros(1, batch, H * G, n, D, dtype=dtype, device="cuda")
            B.paged_attention_window(c, l, 1, q[None], scratch(c, 1, n), out, window, sinks, q_len=i32(news))
            outs.append((l, q[None], out))
        total = [a + b for a, b in zip(total, news)]
        if n > 1 or total[0] % 16 == 0:
            for l, q, out in outs:
                check(full, q, out, news, 0.0, B.paged_plan_window(c, 1, n, window, sinks), lambda b, T, m: S.window_mask(T, m, window, sinks), layer=l)
        dropped = torch.zeros(3, dtype=torch.int32, device="cuda")
        B.pages_slide(c, window, sinks, dropped)
        lost = [a + b for a, b in zip(lost, dropped.tolist())]
        assert c.seq_len[0].tolist() == [t - d for t, d in zip(total, lost)]
    assert c.device_status() == full.device_status() == 0 and lost == [page * S.slide(T, page, window, sinks)[1] for T in total]
    assert max(lost) > 0 and (c.refs > 0).sum().item() <= 3 * (2 + -(-(window + page) // page))


def branch(parents, node):
    path = []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


@pytest.mark.parametrize("dtype,n", [(F16, 3), (BF16, 16)])
def test_speculative_run(dtype, n):
    """Trees on forks, the accepted branch on the original, twice; the cache holds in the end what appending the branches alone gives, bit
    for bit, and a node's output is that of its branch as a sequence of its own."""
    L, S2, H, G, page = 2, 2, 2, 7, 64
    rng, m = random.Random(n), Model(L, 3 * S2, H, H * G, max_pages=5, page=page, dtype=dtype)
    c = m.c
    c.table.fill_(-1), c.refs.zero_()
    B.pages_reserve(c, i32([90, 61, 0, 0, 0, 0]))
    m.append(90, [90, 61, 0, 0, 0, 0])
    ws, freq = scratch(c, L, n + 90), B.rope_frequencies(1e6, 64)
    for step in range(2):
        lens = m.lens()[:S2]
        trees = [random_tree(rng, n) for _ in range(3 * S2)]
        nodes = [0, 0, n, n, 0, 0]
        B.pages_fork(c, i32([0, 1]), i32([2, 3]), ws)
        B.pages_reserve(c, i32([0, 0, lens[0] + n, lens[1] + n, 0, 0]))
        seen = torch.zeros(6, n, 1, dtype=torch.int64, device="cuda")
        depth = torch.zeros(6, n, dtype=torch.int32, device="cuda")
        B.tree_ancestors(c, i32(trees), seen, depth, q_len=i32(nodes))
        start = i32([0, 0, *lens, 0, 0])[:, None]
        rope = B.Rope((depth + start).expand(3, 6, n).contiguous(), freq, (16, 24, 24))
        k, v, q = (randn(m.g, L, 6, h, n, D, dtype=dtype).cuda() for h in (H, H, H * G))
        out = torch.zeros_like(q)
        B.paged_append(c, 0, L, k, v, i32(nodes), rope)
        B.paged_attention_tree(c, 0, L, q, ws, out, seen, i32(nodes), rope)
        turned, kt = q.clone(), k.clone()
        for l in range(L):
            B.rope_apply(rope, turned[l], turned[l], kt[l], kt[l])
        sets = [S.ancestors(t)[0] for t in trees]
        check(c, turned, out, nodes, 0.0, B.paged_plan(c, L, n), lambda b, T, x: S.tree_mask(T, x, sets[b]))
        B.pages_release(c, i32([2, 3]))
        # the accepted branches
        paths = [branch(trees[2 + b], n - 1 - step) for b in range(S2)]
        news = [len(p) for p in paths] + [0] * 4
        most = max(news)
        rows = torch.tensor([p + [0] * (most - len(p)) for p in paths]).cuda()
        take = lambda x: torch.cat([x[:, 2 + b:3 + b, :, rows[b]] for b in range(S2)] + [x[:, 2:, :, :1].expand(-1, -1, -1, most, -1)], 1).contiguous()  # noqa: E731
        B.pages_reserve(c, i32([a + k for a, k in zip(lens, news)] + [0] * 4))
        m.append(most, news, k=take(kt).cpu(), v=take(v).cpu())
        m.check()
        m.attend(1, q_len=[1, 1, 0, 0, 0, 0])
    assert c.device_status() == 0 and (c.refs > 0).sum().item() == sum(-(-x // page) for x in m.lens()[:S2])
