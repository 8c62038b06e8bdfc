"""CPU oracle of the 8-bit paged cache and of the rotary positions with three axes: the formulas in 64 bits (numpy), the
quantiser in the widths that fix its codes bit for bit, the pages' bookkeeping as plain lists.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

D, BLOCK = 128, 32


def rope_axes(sections, interleaved):
    a, b, c = sections
    half = a + b + c
    if not interleaved:
        return [0 if i < a else 1 if i < a + b else 2 for i in range(half)]
    return [1 if i % 3 == 1 and i < 3 * b else 2 if i % 3 == 2 and i < 3 * c else 0 for i in range(half)]


def rope(x, positions, freq, sections, interleaved=False, inverse=False):
    """x [batch, heads, n, 128] (float64), positions [3, batch, n], freq [pairs] -> the rotated numbers, unrounded."""
    half = sum(sections)
    axes = rope_axes(sections, interleaved)
    angle = np.stack([positions[axes[i]].astype(np.float64) * freq[i] for i in range(half)], -1)[:, None]
    c, s = np.cos(angle), np.sin(angle) * (-1 if inverse else 1)
    out = np.array(x, np.float64)
    a, b = out[..., :half].copy(), out[..., half:2 * half].copy()
    out[..., :half] = a * c - b * s
    out[..., half:2 * half] = b * c + a * s
    return out


def quantise(x):
    """One block of one head and side: x [rows <= 32, 128] float32 -> (codes int8, scale float32)."""
    x = np.asarray(x, np.float32)
    amax = np.float32(np.abs(x).max()) if x.size else np.float32(0)
    if not np.isfinite(amax):
        return np.zeros(x.shape, np.int8), np.float32(np.nan)
    scale = amax / np.float32(127)
    if scale == 0:
        return np.zeros(x.shape, np.int8), scale
    return np.clip(np.rint(x / scale), -127, 127).astype(np.int8), scale


def dequantise(codes, scales):
    """codes int8 [tokens, 128], scales float32 [blocks] -> float64 [tokens, 128]."""
    per = np.repeat(np.asarray(scales, np.float64), BLOCK)[:codes.shape[0], None]
    return codes.astype(np.float64) * per


def attention(q, k, v, sm_scale, seen):
    """q [rows, 128], k, v [tokens, 128], all float64; row r sees the first seen[r] tokens.
    -> (out [rows, 128], sum p |v| [rows, 128], largest |score| of each row)"""
    out, mag, top = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[0])
    for r in range(q.shape[0]):
        n = int(min(max(seen[r], 0), k.shape[0]))
        if n == 0:
            continue
        s = k[:n] @ q[r] * sm_scale
        w = np.exp(s - s.max())
        w /= w.sum()
        out[r], mag[r], top[r] = w @ v[:n], w @ np.abs(v[:n]), np.abs(s).max()
    return out, mag, top


class Pages:
    """Tables and counts of a pool, kept as the calls of the library keep them."""

    def __init__(self, batch, max_pages, n_pages, page_tokens):
        self.table = [[-1] * max_pages for _ in range(batch)]
        self.refs = [0] * n_pages
        self.lens = [0] * batch
        self.page, self.max_pages = page_tokens, max_pages
        self.content = [None] * n_pages     # anything that names what a page holds

    def free(self):
        return [p for p, n in enumerate(self.refs) if n == 0]

    def reserve(self, tokens):
        want = [(b, j) for b, t in enumerate(tokens) for j in range(self.max_pages) if j * self.page < t and self.table[b][j] < 0]
        free = self.free()
        if any(t > self.max_pages * self.page for t in tokens) or len(want) > len(free):
            return False
        for (b, j), p in zip(want, free):
            self.table[b][j], self.refs[p] = p, 1
        return True

    def fork(self, src, dst):
        ok = True
        for a, d in zip(src, dst):
            n = self.lens[a] if 0 <= a < len(self.lens) else 0
            full, part = divmod(n, self.page)
            bad = not (0 <= a < len(self.lens) and 0 <= d < len(self.lens)) or a == d
            bad = bad or any(p >= 0 for p in self.table[d]) or any(p < 0 for p in self.table[a][:full + (part > 0)])
            if bad or (part and not self.free()):
                ok = False
                continue
            for j in range(full):
                self.table[d][j] = self.table[a][j]
                self.refs[self.table[a][j]] += 1
            if part:
                p = self.free()[0]
                self.table[d][full], self.refs[p], self.content[p] = p, 1, self.content[self.table[a][full]]
            self.lens[d] = n
        return ok

    def release(self, seqs):
        for b in seqs:
            for j, p in enumerate(self.table[b]):
                if p >= 0:
                    self.refs[p] -= 1
                    self.table[b][j] = -1
            self.lens[b] = 0

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        holes = [p for p in range(n) if self.refs[p] == 0]
        movers = [p for p in range(n, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a], self.content[b] = self.refs[a], 0, self.content[a]
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return n
