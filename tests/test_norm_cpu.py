"""Normed heads with rotation without a GPU: what the calls refuse before they launch anything, and pins of the oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import okq_norm_oracle as N
from oracle import okq_paged_oracle as O
from paper_2609_11582_b200 import binding as B
from paper_2609_11582_b200 import build as build_mod

P16 = 1 << 20                      # an aligned address that no refused call looks at


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return B.lib()


def rope(sections=(16, 24, 24), interleaved=0, freq=P16, positions=P16):
    return C.byref(B.okq_rope((C.c_int32 * 3)(*sections), interleaved, freq, positions))


def t(**kw):
    d = dict(in_=P16, grad_out=P16, out=P16, in_strides=(8, 8, 8), grad_strides=(8, 8, 8), out_strides=(8, 8, 8), weight=P16, weight_grad=P16,
             weight_dtype=2, heads=2)
    d.update(kw)
    return C.byref(B.okq_norm_tensor(*d.values()))


def apply(L, q=t(), k=None, r=rope(), eps=1e-6, dtype=0, batch=1, n=1):
    return L.okq_norm_rope_apply(r, eps, dtype, batch, n, q, k, None)


def grad(L, q=t(), k=None, r=rope(), eps=1e-6, dtype=0, batch=1, n=1, ws=P16, ws_bytes=1 << 30):
    return L.okq_norm_rope_grad(r, eps, dtype, batch, n, q, k, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), B.ERR_INVALID_ARG), (dict(n=-1), B.ERR_INVALID_ARG), (dict(batch=-1), B.ERR_INVALID_ARG), (dict(eps=0.0), B.ERR_INVALID_ARG),
    (dict(eps=-1e-6), B.ERR_INVALID_ARG), (dict(eps=1e-31), B.ERR_INVALID_ARG), (dict(eps=float("nan")), B.ERR_INVALID_ARG),
    (dict(eps=float("inf")), B.ERR_INVALID_ARG), (dict(dtype=3), B.ERR_UNSUPPORTED), (dict(dtype=-1), B.ERR_UNSUPPORTED),
    (dict(q=t(heads=-1)), B.ERR_INVALID_ARG), (dict(q=t(in_=0)), B.ERR_INVALID_ARG), (dict(k=t(out=0)), B.ERR_INVALID_ARG),
    (dict(q=t(weight_dtype=3)), B.ERR_UNSUPPORTED), (dict(k=t(weight=P16 + 8)), B.ERR_ALIGNMENT), (dict(q=t(in_=P16 + 8)), B.ERR_ALIGNMENT),
    (dict(k=t(out_strides=(8, 4, 8))), B.ERR_ALIGNMENT), (dict(q=t(in_strides=(8, 8, 2)), dtype=2), B.ERR_ALIGNMENT),
    (dict(q=t(heads=65535), k=t(heads=1)), B.ERR_UNSUPPORTED), (dict(r=rope((16, 24, 25))), B.ERR_UNSUPPORTED), (dict(r=rope((0, 0, 0))), B.ERR_INVALID_ARG),
    (dict(r=rope(interleaved=2)), B.ERR_INVALID_ARG), (dict(r=rope(freq=0)), B.ERR_INVALID_ARG), (dict(r=rope(positions=P16 + 4)), B.ERR_ALIGNMENT),
])
def test_bad_calls_are_refused(L, kw, want):
    assert apply(L, **kw) == grad(L, **kw) == want


def test_nothing_to_do_is_fine(L):
    assert apply(L, n=0) == apply(L, batch=0) == apply(L, r=None, n=0) == apply(L, q=t(heads=0, in_=0, out=0)) == B.OK
    assert grad(L, q=t(weight_grad=0), n=0, ws=0) == grad(L, q=t(heads=0, in_=0, out=0, grad_out=0, weight_grad=0)) == B.OK
    assert apply(L, q=t(weight=0, weight_dtype=77), n=0) == B.OK              # a type that no weight has


def test_refusals_of_the_gradient(L):
    assert grad(L, q=t(grad_out=0)) == B.ERR_INVALID_ARG and grad(L, q=t(grad_out=P16 + 4)) == B.ERR_ALIGNMENT
    assert grad(L, k=t(weight_grad=P16 + 4)) == B.ERR_ALIGNMENT and grad(L, q=t(grad_strides=(8, 8, 4))) == B.ERR_ALIGNMENT
    need = L.okq_norm_rope_workspace_bytes(1, 1, 2, 0)
    assert need > 0 and need % 16 == 0
    assert grad(L, ws=0) == B.ERR_WORKSPACE and grad(L, ws_bytes=need - 1) == B.ERR_WORKSPACE and grad(L, ws=P16 + 8) == B.ERR_ALIGNMENT
    for bad in ((-1, 1, 1, 1), (1, -1, 1, 1), (1, 1, -1, 1), (1, 1, 1, -1), (1, 1, 65535, 1)):
        assert L.okq_norm_rope_workspace_bytes(*bad) == 0
    assert all(L.okq_norm_rope_workspace_bytes(*size) <= L.okq_norm_rope_workspace_bytes(64, 4096, 32, 4) for size in ((1, 1, 1, 0), (7, 33, 5, 3)))


def test_tensors_that_do_not_fit_are_refused():
    x, w = torch.zeros(1, 2, 3, 128, dtype=torch.float16), torch.ones(128)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        B.norm_rope_apply(None, x, x, w)                                        # on the host


# ------------------------------------------------------------------------------------------------ the oracle
def test_oracle_norms_and_keeps_products():
    rng = np.random.RandomState(0)
    x = rng.randn(2, 3, 5, 128) * 7
    y, _ = N.norm_rope(x, np.ones(128), 1e-12)
    assert np.allclose((y * y).mean(-1), 1)
    pos, freq = np.full((3, 2, 5), 9), 1e4 ** (-np.arange(64) / 64)
    z, _ = N.norm_rope(x, np.ones(128), 1e-12, (pos, freq, (16, 24, 24), False))
    assert np.allclose((z * z).sum(-1), 128) and np.allclose(z, O.rope(y, pos, freq, (16, 24, 24)))


def test_oracle_gradient_is_that_of_differences():
    """Central differences in 64 bits: off by h^2 of third derivatives of order one and 2^-53 / h."""
    rng = np.random.RandomState(1)
    x, g, dx, w, dw = rng.randn(1, 2, 3, 128), rng.randn(1, 2, 3, 128), rng.randn(1, 2, 3, 128), rng.randn(128), rng.randn(128)
    turn = (rng.randint(0, 99, (3, 1, 3)), 1e4 ** (-np.arange(64) / 64), (24, 20, 20), True)
    gx, gw, _ = N.norm_rope_grad(x, w, g, 1e-6, turn)
    h = 1e-5
    f = lambda s, r: (N.norm_rope(x + s * dx, w + r * dw, 1e-6, turn)[0] * g).sum()  # noqa: E731
    assert abs((f(h, 0) - f(-h, 0)) / (2 * h) - (gx * dx).sum()) < 1e-6
    assert abs((f(0, h) - f(0, -h)) / (2 * h) - (gw * dw).sum()) < 1e-6
