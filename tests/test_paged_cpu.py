"""8-bit paged cache and rotary positions without a GPU: what the calls refuse before they launch anything, and pins of the oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import okq_paged_oracle as O
from paper_2609_11582_b200 import binding as B
from paper_2609_11582_b200 import build as build_mod

P16 = 1 << 20                      # an aligned address that no refused call looks at
S4 = (C.c_int64 * 4)(8, 8, 8, 8)


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return B.lib()


def cache(**kw):
    d = dict(n_layers=2, batch=3, n_kv_heads=4, n_q_heads=28, page_tokens=64, n_pages=10, max_pages=5, dtype=0, codes=P16, scales=P16,
             raw=P16, table=P16, refs=P16, seq_len=P16, status=P16)
    d.update(kw)
    return C.byref(B.okq_paged(*d.values()))


def rope(sections=(16, 24, 24), interleaved=0, freq=P16, positions=P16):
    return C.byref(B.okq_rope((C.c_int32 * 3)(*sections), interleaved, freq, positions))


def test_sizes(L):
    s = B.paged_sizes(2, 3, 4, 28, 10, 5, 64, torch.float16)
    rows = 2 * 10 * 4 * 2 * 64
    assert s == [rows * 128, rows // 32 * 4, 2 * 3 * 4 * 2 * 32 * 128 * 2, 3 * 5 * 4, 40, 24, 16]
    assert (s[0] + s[1]) * 8 / (rows * 128) == 8.0078125            # bits per element
    assert L.okq_paged_sizes(cache(), None) == B.ERR_INVALID_ARG
    assert L.okq_paged_workspace_bytes(cache(), 1, 1) > 0
    for bad in (dict(layer_count=0), dict(layer_count=3), dict(n_new=-1)):
        assert L.okq_paged_workspace_bytes(cache(), bad.get("layer_count", 1), bad.get("n_new", 1)) == 0


SHAPES = [(dict(page_tokens=48), B.ERR_UNSUPPORTED), (dict(page_tokens=512), B.ERR_UNSUPPORTED), (dict(dtype=2), B.ERR_UNSUPPORTED),
          (dict(n_q_heads=9), B.ERR_UNSUPPORTED), (dict(n_q_heads=36), B.ERR_UNSUPPORTED), (dict(n_layers=0), B.ERR_INVALID_ARG),
          (dict(batch=-1), B.ERR_INVALID_ARG), (dict(n_pages=0), B.ERR_INVALID_ARG), (dict(max_pages=0), B.ERR_INVALID_ARG),
          (dict(n_pages=1 << 30), B.ERR_UNSUPPORTED), (dict(max_pages=1 << 26), B.ERR_UNSUPPORTED), (dict(batch=1 << 24), B.ERR_UNSUPPORTED)]
POINTERS = [(dict([(n, v)]), e) for n in ("codes", "scales", "raw", "table", "refs", "seq_len", "status") for v, e in ((0, B.ERR_INVALID_ARG), (P16 + 8, B.ERR_ALIGNMENT))]


def append(L, c, layer=0, count=1, k=P16, n=2, new_len=P16, rp=None, s=S4):
    return L.okq_paged_append(c, layer, count, k, s, k, s, n, new_len, rp, None)


def attention(L, c, layer=0, count=1, k=P16, n=2, new_len=P16, rp=None, ws=P16, ws_bytes=1 << 30, out=P16, s=S4):
    return L.okq_paged_attention(c, layer, count, k, s, n, new_len, rp, 0.1, ws, ws_bytes, out, s, None)


@pytest.mark.parametrize("bad,want", SHAPES + POINTERS)
def test_bad_caches_are_refused(L, bad, want):
    c = cache(**bad)
    got = {"append": append(L, c), "attention": attention(L, c)}
    got["read"] = L.okq_paged_read(c, 0, 1, 0, 1, P16, P16, None)
    got["reserve"] = L.okq_pages_reserve(c, P16, None)
    got["fork"] = L.okq_pages_fork(c, P16, P16, 1, P16, 64, None)
    got["release"] = L.okq_pages_release(c, P16, 1, None)
    got["copy"] = L.okq_pages_copy(c, P16, P16, 1, None)
    got["compact"] = L.okq_pages_compact(c, None, P16, 1 << 20, None)
    assert set(got.values()) == {want}, got
    if bad in [b for b, _ in SHAPES]:
        assert L.okq_paged_sizes(c, (C.c_size_t * 7)()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(layer=-1), B.ERR_INVALID_ARG), (dict(layer=2), B.ERR_INVALID_ARG), (dict(count=3), B.ERR_INVALID_ARG), (dict(count=0), B.ERR_INVALID_ARG),
    (dict(layer=1, count=2), B.ERR_INVALID_ARG), (dict(layer=0x7fffffff, count=0x7fffffff), B.ERR_INVALID_ARG), (dict(k=0), B.ERR_INVALID_ARG),
    (dict(k=P16 + 8), B.ERR_ALIGNMENT), (dict(n=-1), B.ERR_INVALID_ARG), (dict(new_len=P16 + 2), B.ERR_ALIGNMENT), (dict(s=None), B.ERR_INVALID_ARG),
    (dict(s=(C.c_int64 * 4)(8, 8, 8, 4)), B.ERR_ALIGNMENT), (dict(rp=rope((16, 24, 25))), B.ERR_UNSUPPORTED), (dict(rp=rope((0, 0, 0))), B.ERR_INVALID_ARG),
    (dict(rp=rope((64, 8, 0))), B.ERR_UNSUPPORTED), (dict(rp=rope((-8, 8, 8))), B.ERR_INVALID_ARG), (dict(rp=rope(interleaved=2)), B.ERR_INVALID_ARG),
    (dict(rp=rope((16, 24, 24), 1)), B.ERR_INVALID_ARG), (dict(rp=rope(freq=0)), B.ERR_INVALID_ARG), (dict(rp=rope(positions=P16 + 4)), B.ERR_ALIGNMENT),
])
def test_bad_calls_are_refused(L, kw, want):
    assert append(L, cache(), **kw) == attention(L, cache(), **kw) == want


def test_nothing_to_do_is_fine(L):
    assert append(L, cache(), n=0, k=0) == attention(L, cache(), n=0, k=0) == B.OK
    assert L.okq_paged_read(cache(), 0, 1, 5, 0, None, None, None) == B.OK
    assert L.okq_pages_fork(cache(), None, None, 0, None, 0, None) == B.OK
    assert L.okq_pages_release(cache(), None, 0, None) == B.OK
    assert L.okq_pages_copy(cache(), None, None, 0, None) == B.OK


def test_other_refusals(L):
    c = cache()
    need = L.okq_paged_workspace_bytes(c, 1, 2)
    assert attention(L, c, ws=0) == B.ERR_WORKSPACE and attention(L, c, ws_bytes=need - 1) == B.ERR_WORKSPACE
    assert attention(L, c, ws=P16 + 4) == B.ERR_ALIGNMENT and attention(L, c, out=P16 + 4) == B.ERR_ALIGNMENT
    assert attention(L, c, out=0) == B.ERR_INVALID_ARG
    for begin, n, p, want in ((-1, 1, P16, B.ERR_INVALID_ARG), (0, -1, P16, B.ERR_INVALID_ARG), (0, 1, 0, B.ERR_INVALID_ARG), (0, 1, P16 + 2, B.ERR_ALIGNMENT),
                              (0x7fffffff, 1, P16, B.ERR_INVALID_ARG)):
        assert L.okq_paged_read(c, 0, 1, begin, n, p, p, None) == want
    assert L.okq_pages_reserve(c, None, None) == B.ERR_INVALID_ARG
    assert L.okq_pages_fork(c, P16, P16, 2, P16, 31, None) == B.ERR_WORKSPACE
    assert L.okq_pages_fork(c, P16, P16, -1, P16, 31, None) == B.ERR_INVALID_ARG
    assert L.okq_pages_fork(c, None, P16, 1, P16, 64, None) == B.ERR_INVALID_ARG
    assert L.okq_pages_release(c, None, 1, None) == B.ERR_INVALID_ARG
    assert L.okq_pages_copy(c, P16, P16 + 1, 1, None) == B.ERR_ALIGNMENT
    assert L.okq_pages_compact(c, None, P16, 8, None) == B.ERR_WORKSPACE
    assert L.okq_pages_compact(c, P16 + 2, P16, 1 << 20, None) == B.ERR_ALIGNMENT


@pytest.mark.parametrize("shape", [dict(), dict(batch=8, n_kv_heads=4, n_q_heads=28, max_pages=64), dict(n_kv_heads=1, n_q_heads=1, max_pages=3000)])
def test_scratch_serves_smaller_calls(L, shape):
    """Sizes grow with layers and queries, whichever kernel takes a call."""
    for layers in (1, 2):
        sizes = [L.okq_paged_workspace_bytes(cache(**shape), layers, n) for n in range(0, 300)]
        assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
        assert all(a <= L.okq_paged_workspace_bytes(cache(**shape), 2, n) for n, a in enumerate(sizes))


def test_plan_and_debug_refusals(L):
    assert L.okq_debug_paged_plan(cache(), 1, 100) == B.PLAN_PROMPT and L.okq_debug_paged_plan(cache(), 1, 1) != 0
    for c, layers, n in ((cache(dtype=2), 1, 1), (cache(), 0, 1), (cache(), 3, 1), (cache(), 1, 0), (cache(), 1, 1 << 27)):
        assert L.okq_debug_paged_plan(c, layers, n) == 0
    assert L.okq_debug_paged_timeout(cache(), 0, 1, P16, S4, 1, P16, 1 << 30, P16, S4, 0, None) == B.ERR_INVALID_ARG


def test_rope_refusals(L):
    def t(**kw):
        d = dict(in_=P16, out=P16, in_strides=(8, 8, 8), out_strides=(8, 8, 8), heads=2)
        d.update(kw)
        return C.byref(B.okq_rope_tensor(*d.values()))
    go = lambda q=t(), k=None, r=rope(), dtype=0, batch=1, n=1, inverse=0: L.okq_rope_apply(r, dtype, batch, n, q, k, inverse, None)  # noqa: E731
    assert go(n=0) == B.OK and go(batch=0) == B.OK and go(q=t(heads=0, in_=0, out=0)) == B.OK
    assert go(r=None) == B.ERR_INVALID_ARG and go(q=None) == B.ERR_INVALID_ARG and go(n=-1) == B.ERR_INVALID_ARG and go(inverse=2) == B.ERR_INVALID_ARG
    assert go(dtype=3) == B.ERR_UNSUPPORTED and go(q=t(heads=-1)) == B.ERR_INVALID_ARG and go(k=t(out=0)) == B.ERR_INVALID_ARG
    assert go(q=t(in_=P16 + 8)) == B.ERR_ALIGNMENT and go(k=t(out_strides=(8, 4, 8))) == B.ERR_ALIGNMENT
    assert go(q=t(in_strides=(8, 8, 2)), dtype=2) == B.ERR_ALIGNMENT
    assert go(q=t(heads=65535), k=t(heads=1)) == B.ERR_UNSUPPORTED
    assert go(r=rope((24, 24, 16), 1)) == B.ERR_INVALID_ARG         # the last pair of axis 1 would be 70


def test_tensors_of_the_host_are_refused():
    x = torch.zeros(1, 1, 1, 128, dtype=torch.float16)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        B.rope_apply(B.Rope(torch.zeros(3, 1, 1, dtype=torch.int32), torch.zeros(64, dtype=torch.float64), (16, 24, 24)), x, x)


def test_tensors_on_two_devices_are_refused():
    with pytest.raises(ValueError):
        B.Rope(torch.zeros(3, 1, 1, dtype=torch.int32, device="meta"), torch.zeros(64, dtype=torch.float64), (16, 24, 24))
    cache = B.PagedCache(1, 1, 1, 1, 2, 2, device="cpu")
    buffers = {n: getattr(cache, n) for n in ("codes", "scales", "raw", "table", "refs", "seq_len")}
    B.PagedCache(1, 1, 1, 1, buffers=buffers)
    for n in buffers:
        with pytest.raises(ValueError):
            B.PagedCache(1, 1, 1, 1, buffers={**buffers, n: buffers[n].to("meta")})


# ------------------------------------------------------------------------------------------------ the oracle
def test_oracle_axes():
    assert O.rope_axes((2, 3, 3), False) == [0, 0, 1, 1, 1, 2, 2, 2]
    axes = O.rope_axes((24, 20, 20), True)
    assert axes[:7] == [0, 1, 2, 0, 1, 2, 0] and [axes.count(i) for i in range(3)] == [24, 20, 20] and axes[58:] == [1, 2, 0, 0, 0, 0]


def test_oracle_rope_keeps_products_and_turns_back():
    """Equal axes: q . k depends on the difference of the positions alone; the inverse undoes; norms stay."""
    rng = np.random.RandomState(0)
    freq = 1e4 ** (-np.arange(64) / 64)
    q, k = rng.randn(1, 1, 1, 128), rng.randn(1, 1, 1, 128)
    at = lambda x, p: O.rope(x, np.full((3, 1, 1), p), freq, (16, 24, 24))  # noqa: E731
    dots = [(at(q, p + 5) * at(k, p)).sum() for p in (0, 17, 4000)]
    assert np.ptp(dots) < 1e-9
    assert np.allclose(O.rope(at(q, 33), np.full((3, 1, 1), 33), freq, (16, 24, 24), inverse=True), q, atol=1e-12)
    assert np.isclose(np.linalg.norm(at(q, 999)), np.linalg.norm(q))


def test_oracle_quantiser():
    rng = np.random.RandomState(1)
    x = rng.randn(32, 128).astype(np.float16).astype(np.float32)
    codes, scale = O.quantise(x)
    assert np.abs(codes).max() == 127 and codes.min() >= -127
    # half a step, and the roundings of scale and quotient
    assert np.abs(codes * np.float64(scale) - x).max() <= scale * (0.5 + 127 * 2.0 ** -23)
    assert O.quantise(np.zeros((3, 128)))[1] == 0 and np.isnan(O.quantise(np.full((1, 128), np.inf))[1])
    assert (O.quantise(np.full((1, 128), 1e-40))[0] == 127).all()        # a subnormal scale


def test_oracle_attention_is_the_softmax():
    rng = np.random.RandomState(2)
    q, k, v = rng.randn(3, 128), rng.randn(50, 128), rng.randn(50, 128)
    out, mag, _ = O.attention(q, k, v, 0.2, [50, 0, 7])
    w = torch.softmax(torch.from_numpy(q @ k.T * 0.2), -1)
    assert np.allclose(out[0], (w[0] @ torch.from_numpy(v)).numpy()) and (out[1] == 0).all()
    assert np.allclose(out[2], (torch.softmax(torch.from_numpy(k[:7] @ q[2] * 0.2), -1) @ torch.from_numpy(v[:7])).numpy())
    assert (mag[0] >= np.abs(out[0])).all()


def test_oracle_pages():
    p = O.Pages(3, 4, 6, 32)
    assert p.reserve([40, 0, 10]) and p.table[0][:2] == [0, 1] and p.table[2][0] == 2
    assert not p.reserve([0, 128, 0]) and not p.reserve([0, 129, 0])
    p.lens = [40, 0, 10]
    assert p.fork([0], [1]) and p.table[1] == [0, 3, -1, -1] and p.refs[:4] == [2, 1, 1, 1]
    assert not p.fork([0, 0, 1], [1, 0, 5])
    p.release([0, 0])
    assert p.refs == [1, 0, 1, 1, 0, 0] and p.compact() == 3 and p.table[1] == [0, 1, -1, -1] and p.refs == [1, 1, 1, 0, 0, 0]
