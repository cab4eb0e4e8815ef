"""Trees of drafted tokens on the host: shapes, masks, greedy walks, and attention under a mask in binary64."""
from __future__ import annotations

import math

import numpy as np
import torch

import _serving as S


def tree(n, kind, rng):
    """Parents of n nodes, every one before its children."""
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1) if n else []
    if kind == "forest":
        return [int(rng.integers(-1, i)) if i else -1 for i in range(n)]
    if kind == "roots":
        return [-1] * n
    return [-1 if i == 0 else int(rng.integers(max(0, i - 9), i)) for i in range(n)]


def closure(parents):
    """(masks as integers, depths) node by node; a parent that is no earlier node counts as none."""
    mask, depth = [], []
    for i, p in enumerate(parents):
        ok = 0 <= p < i
        mask.append((1 << i) | (mask[p] if ok else 0))
        depth.append(depth[p] + 1 if ok else 0)
    return mask, depth


def words_of(masks, words):
    out = np.zeros((len(masks), words), np.uint64)
    for i, m in enumerate(masks):
        for w in range(words):
            out[i, w] = (m >> (64 * w)) & (2 ** 64 - 1)
    return out.view(np.int64)


def walk(parents, draft, target, head=None):
    """(kept nodes, the choice after them)."""
    way, want = [], head
    while True:
        at = way[-1] if way else -1
        found = [i for i, p in enumerate(parents) if p == at and (want is None or draft[i] == want)]
        if not found:
            return way, -1 if want is None else want
        way.append(found[0])
        want = target[found[0]]


def seen_by(masks, pos, base, window, sinks):
    """bool [nodes][base + nodes]: what each node of a row sees."""
    n = len(masks)
    seen = torch.zeros((n, base + n), dtype=torch.bool)
    t = torch.arange(base)
    for i, m in enumerate(masks):
        p = max(pos[i], base)
        seen[i, :base] = ((t > p - window) | (t < sinks)) if window else True
        for j in range(n):
            seen[i, base + j] = bool(m >> j & 1)
    return seen


def attend_masked_ref(q, G, zk, zv, table, rows, seen, P, scale, unit):
    """(o, bound) as _serving.attend_ref gives them, for rows (first token, tokens, positions held) whose tokens see seen[row]."""
    L, Hq, N, d = q.shape
    H = G.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros(q.shape[:3], dtype=torch.float64)
    planes = math.sqrt(d) * (2.0 ** -15 if unit > 1e-5 else 2.0 ** -22)
    for b, (first, new, held) in enumerate(rows):
        if not new:
            continue
        pg = table[b][: -(-held // P)]
        for l in range(L):
            for h in range(H):
                K, V = (torch.from_numpy(z[l, pg, h].reshape(-1, d)[:held].copy()) for z in (zk, zv))
                Gk, Gv = S.full_gauge(G, l, 0, h), S.full_gauge(G, l, 1, h)
                for j in range(h * (Hq // H), (h + 1) * (Hq // H)):
                    x = q[l, j, first: first + new] @ Gk.T
                    ok = seen[b]
                    any_ = ok.any(1)
                    s = (scale * (x @ K.T)).masked_fill(~ok, -math.inf)
                    w = torch.exp(s - s.amax(1, keepdim=True).clamp(min=-1e300))
                    w = torch.where(any_[:, None], w / w.sum(1, keepdim=True).clamp(min=1e-300), torch.zeros_like(w))
                    for i in range(new):           # what a token does not see is left out (0 times NaN is not 0)
                        out[l, j, first + i] = (w[i, ok[i]] @ V[ok[i]]) @ Gv
                    A = abs(scale) * (x.abs() @ K.abs().T).masked_fill(~ok, 0).amax(1)
                    An = abs(scale) * K.norm(dim=1)[None, :].expand(new, -1).masked_fill(~ok, 0).amax(1) * x.norm(dim=1)
                    E = A * (2 * unit + d * 2.0 ** -24) + An * planes
                    rel = torch.expm1(2 * E) + 2 * unit + held * 2.0 ** -24 + planes
                    bound[l, j, first: first + new] = rel * V.norm(dim=1)[None, :].expand(new, -1).masked_fill(~ok, 0).amax(1)
    return out, bound
