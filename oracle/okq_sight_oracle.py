"""CPU oracle of what queries see in the paged cache: windows with sinks, trees of drafted tokens, pages that slide out of sight.  Test
infrastructure only."""
from __future__ import annotations

import numpy as np


def window_mask(tokens, queries, window, sinks):
    """[queries, tokens]: query i is token tokens - queries + i"""
    p, t = tokens - queries + np.arange(queries)[:, None], np.arange(tokens)[None]
    return (t <= p) & ((p - t < window) | (t < sinks))


def ancestors(parents):
    """-> (bits of each node's ancestors and its own, depths, whether a parent was none); -1 and bad parents: the sequence itself"""
    seen, depth, bad = [], [], False
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            bad, p = True, -1
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return seen, depth, bad


def tree_mask(tokens, nodes, seen):
    """[nodes, tokens]: the sequence's newest `nodes` tokens are the nodes"""
    mask = np.zeros((nodes, tokens), bool)
    for i in range(nodes):
        for t in range(tokens):
            j = t - (tokens - nodes)
            mask[i, t] = j < 0 or bool(seen[i] >> j & 1)
    return mask


def slide(tokens, page, window, sinks):
    """(first page that goes, pages that go) of a sequence"""
    first = -(-sinks // page)
    return first, max(0, max(0, tokens - window + 1) // page - first)
