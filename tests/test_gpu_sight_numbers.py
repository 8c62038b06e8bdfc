"""Attention with a window and for trees of drafted tokens over the 8-bit paged cache where a number could lose its bits: the numerators of many
rows, small weights behind tokens without value.  On the GPU against softmax attention in 64 bits."""
import random

import pytest
import torch

from oracle import okq_sight_oracle as S
from paper_2609_11582_b200 import binding as B
from tests.test_gpu_paged import D, F16, gen, randn, random_cache
from tests import test_gpu_sight as sight
from tests.test_gpu_paged_numbers import PROMPT, Store, kernel_bound, lift, steered
from tests.test_gpu_sight import held, scratch, to_words

pytestmark = pytest.mark.gpu


def reference(c, q, b, see, layer=0):
    """(weights [H, rows, T], values [H, T, 128], what the output should be, largest magnitudes of the tokens' blocks, largest |score| of a row)"""
    G, T = c.n_q_heads // c.n_kv_heads, int(c.seq_len[layer, b])
    x, amax = held(c, layer, b, T)
    s = torch.einsum("hgnd,htd->hgnt", q[layer, b].double().unflatten(0, (-1, G)), x[:, 0]) * D ** -0.5
    see = torch.as_tensor(see).cuda()
    top = s.masked_fill(~see, 0.0).abs().amax(-1).flatten(1)
    w = torch.softmax(s.masked_fill(~see, -torch.inf), -1).nan_to_num(0.0).flatten(1, 2)
    return w, x[:, 1], w @ x[:, 1], amax, top


def both_calls(c, q, window, sinks, sets):
    """(output, mask of a sequence) of the call with a window and of the one for a tree"""
    n, T = q.shape[3], int(c.seq_len[0, 0])
    ws, out = scratch(c, 1, n), torch.zeros_like(q)
    B.paged_attention_window(c, 0, 1, q, ws, out, window, sinks)
    yield out.clone(), lambda b: S.window_mask(T, n, window, sinks)
    B.paged_attention_tree(c, 0, 1, q, ws, out, torch.tensor([to_words(x, n) for x in sets]).cuda())
    yield out, lambda b: S.tree_mask(T, n, sets[b])


@pytest.mark.parametrize("n,G", [(40, 4), (24, 2), (70, 4)])
@pytest.mark.parametrize("spread", [1.0, 4.0])
def test_numerators_of_many_rows_keep_their_bits(n, G, spread):
    """The prompt kernel's numerators with a window and for a tree have 22 bits.  Scores as in the other kernels: 2^-24 (8 |s| + 32) of the weighted
    magnitudes.  A numerator as two fp16 numbers: 2^-22 of it, and half a step of 2^-24 where the largest of the row is 2^8 or more (its
    reference lies 6 below 2^14 at most): 2^-33 of the row's largest weight times block, for each token.  The sums: 16 tokens at a time, twice,
    17 numbers each of which may lose 2^-24 of the largest: T / 8 * 17 * 2^-24.  A single fp16 number's 2^-12 of a few large weights is far
    above all that where the output itself is small."""
    g, rng, T, batch, H = gen(n), random.Random(n), 230, 40, 4
    c = random_cache(g, 1, batch, H, H * G, 64, F16, [T] * batch)
    q = (randn(g, 1, batch, H * G, n, D) * spread).cuda()
    assert B.paged_plan(c, 1, n) == B.paged_plan_window(c, 1, n, 150, 5) == B.PLAN_PROMPT
    sets = [[rng.getrandbits(64 * ((n + 63) // 64)) for _ in range(n)] for _ in range(batch)]
    for out, mask in both_calls(c, q, 150, 5, sets):
        for b in range(batch):
            w, v, ref, amax, top = reference(c, q, b, mask(b))
            err = (2.0 ** -24 * (8 * top[..., None] + 32 + T / 8 * 17) + 2.0 ** -22) * (w @ v.abs()) + T * 2.0 ** -33 * (w * amax[:, None]).amax(-1, True)
            limit = err + 2.0 ** -11 * (ref.abs() + err) + 2.0 ** -25
            got = out[0, b].double().unflatten(0, (-1, G)).flatten(1, 2)
            assert ((got - ref).abs() <= limit).all(), (b, ((got - ref).abs() / limit).max().item())


@pytest.mark.parametrize("shape", PROMPT, ids=str)
@pytest.mark.parametrize("main", [35.0, 45.0])
def test_weights_behind_tokens_without_value(shape, main):
    """A token without value that takes all of the weight, tokens e^(main - 95) of it, and others far below these: what the second ones bring
    is the output, whatever reference the parts of a row end with.  The kernel's bound with all tokens of that size."""
    n, batch, H, Hq, T, wide = shape
    q, k, v = steered(*shape, seed=4)
    k[..., 10::256, 0] = lift(main)
    v[..., 600:1000, :] = 0
    k[..., 700, 0] = lift(95.0)
    store, rng = Store(k, v, Hq, wide, seed=4), random.Random(n)
    assert store.attend(q) == B.PLAN_PROMPT
    c, q = store.c, q.cuda()
    sets = [[rng.getrandbits(64 * ((n + 63) // 64)) for _ in range(n)] for _ in range(batch)]
    for out, mask in both_calls(c, q, T - 300, 800, sets):
        for b in range(batch):
            w, x, ref, amax, top = reference(c, q, b, mask(b))
            got = out[0, b].double().unflatten(0, (-1, Hq // H)).flatten(1, 2)
            limit = kernel_bound(w, x, ref, amax, top, q.dtype, B.PLAN_PROMPT)
            assert (ref.abs().amax(-1) > 100 * limit.amin(-1)).all()            # (it says something)
            assert ((got - ref).abs() <= limit).all(), (b, ((got - ref).abs() / limit).max().item())
    assert c.device_status() == 0


@pytest.mark.parametrize("seed", [65, 100])
def test_numbers_behind_masks_of_other_seeds(seed):
    sight.test_numbers_behind_masks(seed)
