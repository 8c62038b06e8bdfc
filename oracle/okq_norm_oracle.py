"""CPU oracle of the normed heads with rotary positions: the formulas in 64 bits (numpy).  Test infrastructure only."""
from __future__ import annotations

import numpy as np

from oracle import okq_paged_oracle as P

D = 128


def _turn(x, turn, inverse=False):
    """turn: None, or (positions [3, batch, n], freq, sections, interleaved)"""
    return x if turn is None else P.rope(x, *turn, inverse=inverse)


def norm_rope(x, w, eps, turn=None):
    """x [batch, heads, n, 128], w [128] (float64) -> (the normed and rotated numbers, the normed ones before the rotation)"""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return _turn(y, turn), y


def norm_rope_grad(x, w, g, eps, turn=None):
    """-> (gradient of x, gradient of w, g turned back): by the Jacobian of x_i s^-1/2, s = mean(x^2) + eps, which is
    s^-1/2 (delta_ij - x_i x_j / (128 s))"""
    u = _turn(g, turn, inverse=True)
    s = (x * x).mean(-1, keepdims=True) + eps
    wu = w * u
    return (wu - x * ((x * wu).sum(-1, keepdims=True) / (D * s))) / np.sqrt(s), (u * x / np.sqrt(s)).reshape(-1, D).sum(0), u
