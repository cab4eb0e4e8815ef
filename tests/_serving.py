"""References of the serving-step tests, in binary64 on the CPU, from the documented byte layouts."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2607_20538_amd import codec as cg

from _parity import unpack_rows


def haar(L, H, d, g, seed):
    """Orthogonal blocks, binary32 [L][2][H][R][g][g]."""
    a = np.random.default_rng(seed).standard_normal((L * 2 * H * (d // g), g, g))
    q, r = np.linalg.qr(a)
    q = q * np.sign(np.diagonal(r, axis1=-2, axis2=-1))[:, None, :]
    return q.reshape(L, 2, H, d // g, g, g).astype(np.float32)


def gauge_dev(G):
    L, _, H, R, g, _ = G.shape
    shp = cg.shape(L, H, R * g, g)
    Gd = cg.alloc_gauge(shp)
    cg.gauge_make(cg.GAUGE_USER, shp, params=G, G_host=None, G_dev=Gd)
    return shp, Gd


def full_gauge(G, l, s, h):
    """[d][d] in binary64."""
    return torch.block_diag(*torch.from_numpy(G[l, s, h].astype(np.float64)))


def random_pool(codec, L, pages, H, P, d, rng, spread=1.0):
    """(codes, side) bytes of a pool: random codes, ranges around zero of about `spread` deviations."""
    if codec.backend == cg.PASSTHROUGH:
        z = (spread * rng.standard_normal((L, pages, H, P, d))).astype(np.float32)
        return z.view(np.uint8).reshape(L, pages, H, P, 4 * d), None
    codes = rng.integers(0, 256, (L, pages, H, P, d * codec.bits // 8), dtype=np.uint8)
    side = np.empty((L, pages, H, P, d // codec.block_c, 2), np.float16)
    side[..., 0] = -spread * rng.uniform(1.0, 2.0, side.shape[:-1])
    side[..., 1] = spread * rng.uniform(2.0, 4.0, side.shape[:-1]) / (2 ** codec.bits - 1)
    return codes, side


def pool_dev(codec, s, codes, side):
    L, pages, H, P = codes.shape[:4]
    d = codes.shape[4] // 4 if side is None else codes.shape[4] * 8 // codec.bits
    c = cg.Cache(codec, s, L, pages, H, P, d)
    c.codes[: codes.size].copy_(torch.from_numpy(np.ascontiguousarray(codes).reshape(-1)))
    if side is not None:
        c.side[: side.nbytes].copy_(torch.from_numpy(np.ascontiguousarray(side).view(np.uint8).reshape(-1)))
    return c


def pool_values(codec, codes, side):
    """zhat [L][pages][H][P][d] in binary64."""
    if side is None:
        return np.ascontiguousarray(codes).view(np.float32).astype(np.float64)
    d = codes.shape[-1] * 8 // codec.bits
    q = unpack_rows(codes, d, codec.bits).astype(np.float64)
    s = np.repeat(side.astype(np.float64), codec.block_c, axis=-2)
    with np.errstate(invalid="ignore"):
        return s[..., 0] + q * s[..., 1]


def visible(p, n, window, sinks):
    """Which of positions 0 .. n - 1 a token at position p sees."""
    t = torch.arange(n)
    seen = t <= p
    return seen & ((t > p - window) | (t < sinks)) if window else seen


def attend_ref(q, G, zk, zv, table, rows, P, scale, window, sinks, unit):
    """(o, bound): outputs [L][Hq][N][d] in binary64 and the bound on the 2-norm of a token's error.

    q: [L][Hq][N][d] binary64, rows: (first token, tokens, positions held) per row.  The bound counts every
    rounding once at its worst.  With u = `unit` the rounding of an operand (2^-11: binary16; 2^-22: two
    planes) and A = |scale| max_t sum_c |q'_c zhat_c|, a score is off by at most E = A (2 u + d 2^-24) plus the
    two split planes of the gauge, 2^-15 sqrt(d) of the row's norm, inside A (2 u) for the shapes here; all
    probabilities change by a factor within exp(+-2 E); p and v round once more each (2 u), their sums in
    binary32 by T 2^-24, and G^T's planes by 2^-15 sqrt(d).  All relative to the largest |v_t|."""
    L, Hq, N, d = q.shape
    H = G.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros(q.shape[:3], dtype=torch.float64)
    planes = math.sqrt(d) * (2.0 ** -15 if unit > 1e-5 else 2.0 ** -22)
    for b, (first, new, held) in enumerate(rows):
        for l in range(L):
            for j in range(Hq):
                h = j // (Hq // H)
                pg = table[b][: -(-held // P)]
                K = torch.from_numpy(zk[l, pg, h].reshape(-1, d)[:held].copy())
                V = torch.from_numpy(zv[l, pg, h].reshape(-1, d)[:held].copy())
                Gk, Gv = full_gauge(G, l, 0, h), full_gauge(G, l, 1, h)
                for i in range(new):
                    p = held - new + i
                    t = visible(p, held, window, sinks)
                    x = Gk @ q[l, j, first + i]
                    k, v = K[t], V[t]
                    s = scale * (k @ x)
                    w = torch.softmax(s, 0)
                    o = Gv.T @ (w @ v)
                    A = abs(scale) * (k.abs() @ x.abs()).max().item()
                    An = abs(scale) * (k.norm(dim=1).max() * x.norm()).item()
                    E = A * (2 * unit + d * 2.0 ** -24) + An * planes
                    rel = math.expm1(2 * E) + 2 * unit + held * 2.0 ** -24 + planes
                    out[l, j, first + i] = o
                    bound[l, j, first + i] = rel * v.norm(dim=1).max().item()
    return out, bound


def rope_ref(x, pos, d_rot, layout, base=10000.0, scaling=cg.ROPE_NONE, factor=1.0, low=1.0, high=4.0, train_len=0,
             amplitude=1.0, inverse=False):
    """x [L][B][H][T][d] binary64 turned at pos [B][T]; angles in binary64."""
    i = torch.arange(d_rot // 2, dtype=torch.float64)
    f = base ** (-2.0 * i / d_rot)
    if scaling == cg.ROPE_LINEAR:
        f = f / factor
    if scaling == cg.ROPE_RAMP:
        w = ((train_len * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * (1 - w) / factor + f * w
    a = pos.double()[None, :, None, :, None] * f * (-1.0 if inverse else 1.0)
    c, s = amplitude * a.cos(), amplitude * a.sin()
    y = x.clone()
    if layout == cg.ROPE_HALF:
        u, v = slice(0, d_rot // 2), slice(d_rot // 2, d_rot)
    else:
        u, v = slice(0, d_rot, 2), slice(1, d_rot, 2)
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., u] * s + x[..., v] * c
    keep = (pos < 0)[None, :, None, :, None].expand_as(y)
    return torch.where(keep, x, y)


def page_map_ref(held, add, free, table, P, N):
    """The step request by request on the host: (cu, lens, pos, slots, table, free pages left)."""
    free, table = list(free), [list(r) for r in table]
    cu, lens, pos, slots = [0], [], [], []
    for b, (h, n) in enumerate(zip(held, add)):
        for i in range(-(-h // P), -(-(h + n) // P)):
            table[b][i] = free.pop()
        for t in range(h, h + n):
            pos.append(t)
            slots.append(table[b][t // P] * P + t % P)
        cu.append(cu[-1] + n)
        lens.append(h + n)
    rest = [-1] * (N - len(pos))
    return cu, lens, pos + rest, slots + rest, table, free
