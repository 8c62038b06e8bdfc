"""Attention with a window and for trees over the 8-bit paged cache: more pairs of layer and sequence than threads of a block, waits that run out
in each of the kernels, scales and queries at their ends.  On the GPU against the oracle in 64 bits."""
import random

import pytest
import torch

from oracle import okq_sight_oracle as S
from paper_2609_11582_b200 import binding as B
from tests.test_gpu_paged import BF16, D, F16, gen, randn, random_cache
from tests.test_gpu_sight import check, i32, lengths, random_tree, scratch, to_words

pytestmark = pytest.mark.gpu


# (layers, batch, KV heads, group, page, queries, longest, window, sinks)
@pytest.mark.parametrize("shape", [(18, 28, 8, 4, 64, 9, 300, 200, 5), (25, 20, 1, 8, 32, 20, 500, 65, 0)], ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_more_pairs_than_threads(shape, dtype):
    """A thread has two pairs: equal lengths (whole items to a range), ragged ones with empty sequences, some queries of each."""
    L, batch, H, G, page, n, longest, window, sinks = shape
    g, rng = gen(longest), random.Random(longest)
    for ragged in (False, True):
        lens = lengths(g, batch, longest, ragged)
        q_len = None if not ragged else torch.randint(-1, n + 2, (batch,), generator=g).tolist()
        c = random_cache(g, L, batch, H, H * G, page, dtype, lens)
        q, ql, ws = randn(g, L, batch, H * G, n, D, dtype=dtype).cuda(), None if q_len is None else i32(q_len), scratch(c, L, n)
        assert B.paged_plan(c, L, n) == B.paged_plan_window(c, L, n, window, sinks) == B.PLAN_PROMPT and L * batch > 480
        out = torch.full_like(q, 5.0)
        B.paged_attention_window(c, 0, L, q, ws, out, window, sinks, ql)
        check(c, q, out, q_len, 5.0, B.PLAN_PROMPT, lambda b, T, m: S.window_mask(T, m, window, sinks))
        sets = [S.ancestors(random_tree(rng, n))[0] for _ in range(batch)]
        out.fill_(5.0)
        B.paged_attention_tree(c, 0, L, q, ws, out, torch.tensor([to_words(s, n) for s in sets]).cuda(), ql)
        check(c, q, out, q_len, 5.0, B.PLAN_PROMPT, lambda b, T, m: S.tree_mask(T, m, sets[b]))
        assert c.device_status() == 0


# clusters, the line, few rows and many in the prompt kernel, whole items to a range (more items than ranges, all alike)
@pytest.mark.parametrize("batch,H,G,n,tokens,window", [(1, 2, 7, 1, 2000, 700), (30, 4, 7, 1, 3000, 1000), (40, 4, 7, 5, 1000, 300), (2, 4, 7, 300, 2500, 900),
                                                       (111, 4, 8, 9, 700, 250)])
def test_waits_are_bounded_with_a_window_and_for_a_tree(batch, H, G, n, tokens, window):
    """With nothing delivered every role's wait runs out, the device goes on, and the next call with the same scratch is right."""
    g, rng = gen(13), random.Random(13)
    c = random_cache(g, 1, batch, H, G * H, 64, F16, [tokens] * batch)
    q = randn(g, 1, batch, G * H, n, D).cuda()
    ws = scratch(c, 1, n)
    sets = [S.ancestors(random_tree(rng, n))[0] for _ in range(batch)]
    seen = torch.tensor([to_words(s, n) for s in sets]).cuda()
    for kw in (dict(window=window, sinks=4), dict(seen=seen)):
        out = torch.zeros_like(q)
        B.debug_paged_timeout_sight(c, 0, 1, q, ws, out, limit_clocks=2_000_000, **kw)
        torch.cuda.synchronize()
        assert c.device_status() == B.ERR_TIMEOUT and torch.isnan(out).all()
        c.status.zero_()
        out.fill_(5.0)
        if "seen" in kw:
            B.paged_attention_tree(c, 0, 1, q, ws, out, seen)
            check(c, q, out, None, 5.0, B.paged_plan(c, 1, n), lambda b, T, m: S.tree_mask(T, m, sets[b]))
        else:
            B.paged_attention_window(c, 0, 1, q, ws, out, window, 4)
            check(c, q, out, None, 5.0, B.paged_plan_window(c, 1, n, window, 4), lambda b, T, m: S.window_mask(T, m, window, 4))
        assert c.device_status() == 0


@pytest.mark.parametrize("n", [1, 4, 60])
@pytest.mark.parametrize("batch", [2, 40])
def test_no_scale_and_queries_without_a_number(batch, n):
    """A softmax scale of zero is the mean of what is seen; queries with an infinity or NaN give NaN where they see a token, zeros where none."""
    g, T, window = gen(n), 900, 130
    c = random_cache(g, 1, batch, 2, 10, 64, F16, [T] * batch)
    q, ws = randn(g, 1, batch, 10, n, D).cuda(), scratch(c, 1, n)
    out = torch.full_like(q, 5.0)
    B.paged_attention_window(c, 0, 1, q, ws, out, window, 40, sm_scale=0.0)
    check(c, q, out, None, 5.0, B.paged_plan_window(c, 1, n, window, 40), lambda b, t, m: S.window_mask(t, m, window, 40), sm_scale=0.0)
    sets = [0 if i % 2 else 1 << i for i in range(n)]
    seen = torch.tensor([to_words(sets, n)] * batch).cuda()
    B.paged_attention_tree(c, 0, 1, q, ws, out, seen, sm_scale=0.0)
    check(c, q, out, None, 5.0, B.paged_plan(c, 1, n), lambda b, t, m: S.tree_mask(t, m, sets), sm_scale=0.0)
    q[0, 0, 3, :, 5], q[0, 1, 4, :, 127] = float("inf"), float("nan")
    B.paged_attention_window(c, 0, 1, q, ws, out, window, 40)
    assert torch.isnan(out[0, 0, 3]).all() and torch.isnan(out[0, 1, 4]).all() and torch.isfinite(out[0, 0, :3]).all() and torch.isfinite(out[0, 1, 5:]).all()
    c.seq_len.fill_(n)                                                          # nodes alone: the odd ones see nothing
    B.paged_attention_tree(c, 0, 1, q, ws, out, seen)
    for i in range(n):
        if i % 2:
            assert (out[0, :, :, i] == 0).all()
        else:
            assert torch.isnan(out[0, 0, 3, i]).all() and torch.isnan(out[0, 1, 4, i]).all() and torch.isfinite(out[0, 0, :3, i]).all()
    assert c.device_status() == 0


def test_gradients_of_keys_that_are_not_there_are_refused():
    q, sums = torch.ones(1, 2, 3, D, dtype=F16, device="cuda"), torch.zeros(D, device="cuda")
    ws = torch.empty(B.norm_rope_workspace_bytes(1, 3, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(AssertionError):
        B.norm_rope_grad(None, q, q, torch.empty_like(q), ws, None, None, k_weight_grad=sums)
