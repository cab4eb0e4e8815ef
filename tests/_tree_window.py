"""Masks of trees under a sliding window, node by node on the host."""
from __future__ import annotations


def windowed(masks, depth, base, window, sinks):
    """The ancestor masks without what the window hides: node j of node i at base + depth[j] <= base + depth[i] - window, unless
    it is one of the first `sinks` positions (base: the position of the roots)."""
    if not window:
        return list(masks)
    out = []
    for i, m in enumerate(masks):
        keep = 0
        for j in range(i + 1):
            if m >> j & 1 and (depth[j] > depth[i] - window or base + depth[j] < sinks):
                keep |= 1 << j
        out.append(keep)
    return out
