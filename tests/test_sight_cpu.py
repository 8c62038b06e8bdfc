"""Windows, trees and sliding pages of the 8-bit paged cache without a GPU: what the calls refuse before they launch anything, how they are
planned, and pins of the oracle."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

from oracle import okq_sight_oracle as S
from paper_2609_11582_b200 import binding as B
from paper_2609_11582_b200 import build as build_mod
from tests.test_paged_cpu import P16, POINTERS, S4, SHAPES, cache, rope


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return B.lib()


def window(L, c, layer=0, count=1, k=P16, n=2, q_len=P16, rp=None, window=5, sinks=1, ws=P16, ws_bytes=1 << 30, out=P16, s=S4):
    return L.okq_paged_attention_window(c, layer, count, k, s, n, q_len, rp, 0.1, window, sinks, ws, ws_bytes, out, s, None)


def tree(L, c, layer=0, count=1, k=P16, n=2, q_len=P16, rp=None, seen=P16, ws=P16, ws_bytes=1 << 30, out=P16, s=S4):
    return L.okq_paged_attention_tree(c, layer, count, k, s, n, q_len, rp, 0.1, seen, ws, ws_bytes, out, s, None)


@pytest.mark.parametrize("bad,want", SHAPES + POINTERS)
def test_bad_caches_are_refused(L, bad, want):
    c = cache(**bad)
    got = {window(L, c), tree(L, c), L.okq_tree_ancestors(c, P16, 2, None, P16, None, None), L.okq_pages_slide(c, 5, 1, None, None)}
    assert got == {want}


@pytest.mark.parametrize("kw,want", [
    (dict(layer=-1), B.ERR_INVALID_ARG), (dict(count=3), B.ERR_INVALID_ARG), (dict(layer=0x7fffffff, count=0x7fffffff), B.ERR_INVALID_ARG),
    (dict(k=0), B.ERR_INVALID_ARG), (dict(k=P16 + 8), B.ERR_ALIGNMENT), (dict(n=-1), B.ERR_INVALID_ARG), (dict(q_len=P16 + 2), B.ERR_ALIGNMENT),
    (dict(s=None), B.ERR_INVALID_ARG), (dict(s=(C.c_int64 * 4)(8, 8, 8, 4)), B.ERR_ALIGNMENT), (dict(rp=rope((16, 24, 25))), B.ERR_UNSUPPORTED),
    (dict(ws=0), B.ERR_WORKSPACE), (dict(ws_bytes=100), B.ERR_WORKSPACE), (dict(ws=P16 + 4), B.ERR_ALIGNMENT), (dict(out=0), B.ERR_INVALID_ARG),
    (dict(out=P16 + 4), B.ERR_ALIGNMENT),
])
def test_bad_calls_are_refused(L, kw, want):
    assert window(L, cache(), **kw) == tree(L, cache(), **kw) == want


def test_other_refusals(L):
    c = cache()
    for bad in (dict(window=0), dict(window=-1), dict(window=-(1 << 31)), dict(sinks=-1)):
        assert window(L, c, **bad) == B.ERR_INVALID_ARG
        w, s = bad.get("window", 5), bad.get("sinks", 1)
        assert L.okq_pages_slide(c, w, s, None, None) == B.ERR_INVALID_ARG and L.okq_debug_paged_plan_window(c, 1, 1, w, s) == 0
    assert L.okq_paged_attention_window(None, 0, 1, P16, S4, 1, None, None, 0.1, 5, 1, P16, 1 << 30, P16, S4, None) == B.ERR_INVALID_ARG
    assert L.okq_pages_slide(c, 5, 1, P16 + 2, None) == B.ERR_ALIGNMENT and L.okq_pages_slide(None, 5, 1, None, None) == B.ERR_INVALID_ARG
    assert tree(L, c, seen=0) == B.ERR_INVALID_ARG and tree(L, c, seen=P16 + 4) == B.ERR_ALIGNMENT
    go = lambda p=P16, n=2, q_len=None, seen=P16, depth=None: L.okq_tree_ancestors(c, p, n, q_len, seen, depth, None)  # noqa: E731
    assert go(p=0) == go(seen=0) == go(n=-1) == B.ERR_INVALID_ARG and go(n=4097) == B.ERR_UNSUPPORTED
    assert go(p=P16 + 2) == go(q_len=P16 + 2) == go(seen=P16 + 4) == go(depth=P16 + 2) == B.ERR_ALIGNMENT


def test_nothing_to_do_is_fine(L):
    assert window(L, cache(), n=0, k=0) == tree(L, cache(), n=0, k=0, seen=0) == L.okq_tree_ancestors(cache(), None, 0, None, None, None, None) == B.OK


def test_plans_of_windows(L):
    """A window as long as the row is none; a short one never needs more scratch than none, whatever kernel it takes."""
    for shape in (dict(), dict(batch=8, max_pages=512, n_pages=4096), dict(n_layers=28, batch=64, n_kv_heads=8, n_q_heads=64, max_pages=1000)):
        c = cache(**shape)
        room = 64 * shape.get("max_pages", 5)
        for n in (1, 2, 3, 5, 40, 700):
            plain = L.okq_debug_paged_plan(c, 1, n)
            for w in (room, room + 1, 0x7fffffff):
                assert L.okq_debug_paged_plan_window(c, 1, n, w, 0) == plain
            assert L.okq_debug_paged_plan_window(c, 1, n, 1, 0x7fffffff) == plain
            for w in (1, 100, room // 2 + 1):
                assert L.okq_debug_paged_plan_window(c, 1, n, w, 4) != 0


def test_tensors_that_do_not_fit_are_refused():
    c = B.PagedCache(1, 2, 1, 1, 4, 2, device="cpu")
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        B.tree_ancestors(c, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 2, dtype=torch.int64))
    with pytest.raises(AssertionError):
        B._seen(c, torch.zeros(2, 65, 1, dtype=torch.int64), 65)
    with pytest.raises(AssertionError):
        B._seen(c, torch.zeros(2, 3, 1, dtype=torch.int32), 3)


# ------------------------------------------------------------------------------------------------ the oracle
def test_oracle_masks():
    w = S.window_mask(10, 4, 3, 2)
    assert [r.nonzero()[0].tolist() for r in w] == [[0, 1, 4, 5, 6], [0, 1, 5, 6, 7], [0, 1, 6, 7, 8], [0, 1, 7, 8, 9]]
    assert not S.window_mask(2, 4, 3, 0)[:2].any() and S.window_mask(2, 4, 3, 0)[2].tolist() == [True, False]
    seen, depth, bad = S.ancestors([-1, 0, 0, 1, -1, 3])
    assert depth == [0, 1, 1, 2, 0, 3] and not bad and seen == [1, 3, 5, 11, 16, 43]
    t = S.tree_mask(8, 6, seen)
    assert t[:, :2].all() and t[5, 2:].tolist() == [True, True, False, True, False, True]
    assert S.ancestors([-1, 1, 0, -7])[::2] == ([1, 2, 5, 8], True)
    # a chain is the causal mask
    chain, _, _ = S.ancestors(list(range(-1, 4)))
    assert (S.tree_mask(9, 5, chain) == S.window_mask(9, 5, 99, 0)).all()


def test_oracle_slide_keeps_what_is_seen():
    """Coming queries see the same tokens before and after."""
    rng = random.Random(0)
    for _ in range(300):
        page, n, w, s = rng.choice([32, 64]), rng.randint(0, 600), rng.randint(1, 400), rng.choice([0, 1, 4, 33, 64, 200])
        first, gone = S.slide(n, page, w, s)
        kept = [t for t in range(n) if not first * page <= t < (first + gone) * page]
        for new in range(1, 4):
            before = S.window_mask(n + new, 1, w, s)[0].nonzero()[0].tolist()
            after = S.window_mask(len(kept) + new, 1, w, s)[0].nonzero()[0].tolist()
            assert [(kept + list(range(n, n + new)))[t] for t in after] == before
        assert gone == 0 or n - w + 1 - (first + gone) * page < page
