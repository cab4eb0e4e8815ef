"""Operators of a step that checks trees of drafted tokens over paged, gauge-coded caches: what is timed and compared.

A server that drafts several continuations at once packs every request's drafts as a tree behind the positions that the
request holds, runs the model once over all of them and keeps the path that the model agrees with.  The operators of such
a step: positions and masks from the trees' parents (map), queries turned and keys and values turned, gauged and
appended in one go (append), attention of the drafts over the pools, each seeing what is held and its own ancestors
(attend), the path that the model agrees with (accept), and the path's entries moved together, the rest given back (keep).

`run` computes each in plain torch, or with `own` through paper_2607_20538_amd.codec.  Caches that exist before a
step are built here in plain torch by the documented byte layout.  Request lengths follow from the case, values and
trees from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------
# the cases: `rows` requests, the first of `new` drafted tokens, behind at most `ctx` held positions; a node of a tree has
# about `branch` children
# ------------------------------------------------------------------------------------------

def _map(**kw):
    return dict(dict(op="map", rows=32, new=16, ctx=8192, branch=3), **kw)


def _append(**kw):
    return dict(dict(op="append", L=1, H=8, grp=4, rows=32, new=16, ctx=8192, branch=3, d=128, g=128, bits=4, n=64, page=256,
                     rot=128, layout="half", scaling="none", dtype="bf16"), **kw)


def _attend(**kw):
    return dict(dict(op="attend", L=1, H=8, grp=4, rows=32, new=16, ctx=8192, branch=3, d=128, g=128, bits=4, n=64, page=256,
                     window=0, sinks=0, dtype="bf16"), **kw)


def _accept(**kw):
    return dict(dict(op="accept", rows=32, new=16, ctx=0, branch=3, head=False), **kw)


def _keep(**kw):
    return dict(dict(op="keep", L=4, H=8, rows=32, new=16, ctx=100, d=128, g=128, bits=0, n=64, page=64), **kw)


def listed():
    return [
        # trees of 16 drafts of 32 requests: latency
        _map(name="map_step"),
        # ... and of up to 250 drafts of 256 requests: many words of a mask each
        _map(name="map_wide", rows=256, new=250, branch=4),
        # the drafts of 32 requests, as each layer of a Llama-3-8B-shaped model appends them: latency
        _append(name="append_step"),
        # prompts of that shape at far positions (a prompt is a tree without branches), frequencies scaled for a long context
        _append(name="append_prompts", rows=8, new=1500, ctx=120000, branch=1, scaling="ramp"),
        # the smallest configuration: two heads of 64 channels, binary32, odd counts
        _attend(name="attend_tiny_f32", H=2, grp=2, rows=3, new=13, ctx=300, d=64, g=16, n=32, page=64, dtype="f32"),
        # trees of 16 drafts of 32 requests of the Llama-3-8B shape
        _attend(name="attend_step"),
        # 8 long requests whose trees have 60 nodes
        _attend(name="attend_wide", rows=8, new=60, ctx=20000, branch=5),
        # 27B-shaped heads at 3 bits, trees of 25 nodes behind a 4096-position window with 4 sinks
        _attend(name="attend_window", H=16, grp=2, rows=24, new=25, ctx=12000, g=32, bits=3, window=4096, sinks=4),
        # greedy checks of 32 trees whose roots are decided: latency
        _accept(name="accept_step"),
        # ... and of 256 forests of up to 250 nodes, whose roots are checked as well
        _accept(name="accept_wide", rows=256, new=250, branch=4, head=True),
        # the kept paths of 32 requests in four layers of error-free pools: latency
        _keep(name="keep_step"),
        # 64 requests with trees of 60 nodes in eight layers of 4-bit pools of 16 heads
        _keep(name="keep_wide", L=8, H=16, rows=64, new=60, g=32, bits=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["map", "append", "append", "accept", "keep"] + ["attend"] * 4)
    if op in ("map", "accept"):
        rows = _log_int(rng, 1, 300)
        kw = dict(rows=rows, new=_log_int(rng, 1, max(2, min(1000, 64000 // rows))), branch=rng.choice([1, 2, 3, 4, 8]))
        return _map(ctx=_log_int(rng, 1, 30000), **kw) if op == "map" else _accept(head=rng.random() < 0.5, **kw)
    H = rng.choice([1, 2, 4, 8, 16])
    if op == "append":
        d, dtype = rng.choice([(128, "bf16"), (128, "bf16"), (64, "bf16"), (96, "f32"), (256, "bf16"), (128, "f32")])
        g = rng.choice([g for g in (16, 32, 64, 128) if d % g == 0])
        L, grp, rows = rng.choice([1, 1, 2]), rng.choice([1, 2, 4, 8]), _log_int(rng, 1, 64)
        tokens = 9000 * 8 * 6 * 128 // (L * H * (grp + 2) * d * (2 if dtype == "f32" else 1))
        branch = rng.choice([1, 2, 3, 5])
        return _append(L=L, H=H, grp=grp, rows=rows, new=_log_int(rng, 1, max(2, min(1500 if branch == 1 else 250, tokens // rows))),
                       ctx=_log_int(rng, 10, 1000000), branch=branch, d=d, g=g,
                       bits=rng.choice([6, 8, 4] if g >= 64 else [6, 8, 0]), n=rng.choice([32, 32, d // 2]) if d != 96 else 32,
                       page=rng.choice([64, 128, 256]), rot=rng.choice([d, d, d // 2, d // 4]), layout=rng.choice(["half", "pairs"]),
                       scaling=rng.choice(["none", "linear", "ramp"]), dtype=dtype)
    if op == "keep":
        d = rng.choice([64, 128, 128, 256])
        g = rng.choice([g for g in (16, 32, 64, 128) if d % g == 0])
        bits = rng.choice([0, 2, 3, 4, 6, 8])
        L, rows = rng.choice([1, 2, 4]), _log_int(rng, 1, 40)
        return _keep(L=L, H=H, rows=rows, new=_log_int(rng, 1, max(2, min(250, 16000 * 128 // (L * H * rows) // d))),
                     ctx=_log_int(rng, 1, 120), d=d, g=g, bits=bits, n=rng.choice([32, 64]), page=rng.choice([64, 128]))
    # attend: mostly 128-channel heads in bf16; the work of a draw stays under the largest listed one's
    d, dtype = rng.choice([(128, "bf16")] * 5 + [(64, "bf16"), (64, "f32"), (128, "f32"), (256, "bf16"), (80, "bf16")])
    g = d if d == 80 else rng.choice([g for g in (16, 32, 64, 128) if d % g == 0])
    bits = 4 if d == 80 else rng.choice([2, 3, 4, 4, 6, 8])
    n = 80 if d == 80 else rng.choice([32, 64])
    grp, ctx, rows = rng.choice([1, 2, 4, 5, 8]), _log_int(rng, 30, 30000), _log_int(rng, 1, 48)
    tokens = 8 * 60 * 20000 * 32 * 128 // (ctx * H * grp * d * (3 if dtype == "f32" else 1))
    rows = max(1, min(rows, tokens, 24 * 12000 * 16 * 128 // (ctx * H * d)))
    window, sinks = rng.choice([(0, 0), (0, 0), (_log_int(rng, 16, 4096), rng.choice([0, 1, 4, 70]))])
    return _attend(H=H, grp=grp, rows=rows, new=_log_int(rng, 1, max(2, min(250, tokens // rows))), ctx=ctx, branch=rng.choice([1, 2, 3, 5]),
                   d=d, g=g, bits=bits, n=n, page=rng.choice([64, 128, 256]), window=window, sinks=sinks, dtype=dtype)


def _rows(c):
    """(positions held before, drafted tokens) of every request, from the case alone: the first one the longest."""
    rng = random.Random(f"{c['op']} {c['rows']} {c['new']} {c['ctx']}")
    row = lambda: (rng.randint(c["ctx"] // 4, c["ctx"]), rng.randint((c["new"] + 1) // 2, c["new"]))         # noqa: E731
    return [(c["ctx"], c["new"])] + [row() for _ in range(c["rows"] - 1)]


def _words(c):
    return -(-c["new"] // 64)


def _coded(c):
    """Bytes of a cached vector."""
    return c["d"] * c["bits"] // 8 + c["d"] // c["n"] * 4 if c["bits"] else 4 * c["d"]


def work(c):
    rows = _rows(c)
    N = sum(n for _, n in rows)
    if c["op"] == "map":
        return {"bytes": 8 * N + 8 * N * _words(c) + 8 * len(rows), "flops": 0}
    if c["op"] == "accept":
        return {"bytes": 16 * N + (16 if c["head"] else 12) * len(rows), "flops": 0}
    d, heads = c["d"], c["L"] * c["H"]
    if c["op"] == "keep":
        moved = 2 * heads * _moved(c)
        pool = 2 * heads * _pool_pages(c) * c["page"] if c["bits"] else 0       # recovered in bf16 for the comparison
        return {"bytes": 2 * moved * _coded(c) + pool * (_coded(c) + 2 * d) + 4 * N, "flops": 2 * d * c["g"] * pool}
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "append":
        vec, pool = 2 * heads * N, 2 * heads * _pool_pages(c) * c["page"] if c["bits"] else 0
        return {"bytes": vec * (size * d + _coded(c)) + 2 * heads * c["grp"] * N * size * d + 8 * N + pool * (_coded(c) + 2 * d),
                "flops": 2 * d * c["g"] * (vec + pool) + 3 * heads * (c["grp"] + 1) * N * c["rot"]}
    seen = lambda held: min(held, c["window"] + c["sinks"]) if c["window"] else held                         # noqa: E731
    pairs, read = sum(n * (seen(h) + 1) for h, n in rows), sum(seen(h) + n for h, n in rows)
    return {"bytes": heads * (2 * _coded(c) * read + 2 * size * c["grp"] * N * d) + 8 * N * _words(c),
            "flops": heads * c["grp"] * (4 * d * pairs + 4 * d * c["g"] * N)}


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------

def _gen(seed, *tags):
    g = torch.Generator(device=DEV)
    k = seed & 0xFFFFFFFF
    for t in tags:
        k = (k * 1000003 + t + 12345) & 0x7FFFFFFFFFFF
    g.manual_seed(k)
    return g


def _randn(shape, seed, *tags):
    return torch.randn(shape, generator=_gen(seed, *tags), device=DEV)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _gauge(L, H, d, g):
    """The model's gauge: orthogonal blocks, binary32 [L][2][H][R][g][g], the same for every input."""
    gen = torch.Generator().manual_seed(0x6A06E + 1000 * L + 100 * H + d + g)
    A = torch.randn((L * 2 * H * (d // g), g, g), generator=gen, dtype=torch.float64)
    Q, R = torch.linalg.qr(A)
    Q = (Q * torch.sign(torch.diagonal(R, dim1=-2, dim2=-1))[:, None, :]).float()
    return Q.reshape(L, 2, H, d // g, g, g).contiguous().to(DEV)


def _pool_pages(c):
    if c["op"] == "append":
        return -(-sum(n for _, n in _rows(c)) // c["page"]) + 2
    return sum(-(-(h + n) // c["page"]) for h, n in _rows(c)) + 2


def _key_scale(c, seed):
    """Per-channel scale of the keys: log-normal, a few outlier channels."""
    s = torch.exp(0.7 * _randn((c["L"], 1, c["H"], 1, c["d"]), seed, 7))
    out = torch.rand(s.shape, generator=_gen(seed, 8), device=DEV).argsort(-1)[..., : max(1, c["d"] // 32)]
    return s.scatter(-1, out, s.gather(-1, out) * 5.0)


def _half(v, up):
    """binary16 of v rounded up or down (no -0)."""
    h = v.to(torch.float16)
    off = (h.to(v.dtype) < v) if up else (h.to(v.dtype) > v)
    b = h.view(torch.int16)
    step = torch.where((b < 0) ^ (not up), -1, 1).to(torch.int16)
    b = torch.where(off, b + step, b)
    return torch.where(b == -32768, torch.zeros_like(b), b).view(torch.float16)


def _quantise(z, n, bits):
    """(codes, minima, scales) of z [..., d] with one range per n channels; codes [..., d / n, n]."""
    zb = z.reshape(*z.shape[:-1], -1, n)
    mn = _half(zb.amin(-1, keepdim=True), False)
    top = float(2 ** bits - 1)
    sc = _half((zb.amax(-1, keepdim=True) - mn.to(z.dtype)) / top, True)
    s = sc.to(z.dtype)
    inv = torch.where(s == 0, torch.zeros_like(s), 1.0 / s)
    return torch.clamp(torch.round((zb - mn.to(z.dtype)) * inv), 0, top), mn, sc


def _pack(codes, bits):
    """LSB-first bytes of the codes along the last dimension (a multiple of 8 codes)."""
    q = codes.to(torch.int64).reshape(*codes.shape[:-1], -1, 8)
    w = (q << (bits * torch.arange(8, device=DEV))).sum(-1)
    by = (w.unsqueeze(-1) >> (8 * torch.arange(bits, device=DEV))) & 255
    return by.to(torch.uint8).reshape(*codes.shape[:-1], -1)


def _unpack(by, d, bits):
    """The codes [..., d] of packed rows [..., d bits / 8]."""
    k = torch.arange(d, device=DEV) * bits
    ends = torch.nn.functional.pad(by, (0, 1)).to(torch.int32)
    return ((ends[..., k // 8] | (ends[..., k // 8 + 1] << 8)) >> (k % 8).to(torch.int32)) & (2 ** bits - 1)


def _rotate(x, G, dtype, inverse=False):
    """x [L][.][H][T][d] times the block-diagonal gauge G [L][H][R][g][g] (or its transpose)."""
    M = G.to(dtype)
    M = (M if inverse else M.transpose(-1, -2)).contiguous().unsqueeze(1)          # [L][1][H][R][g][g]
    L, B, H, T, d = x.shape
    y = x.to(dtype).reshape(L, B, H, T, M.shape[3], -1).transpose(3, 4).contiguous() @ M
    return y.transpose(3, 4).reshape(L, B, H, T, d)


def _heads(t):
    """[L][N][H][d] as a model lays its projections out -> the view [L][1][H][N][d]."""
    return t.transpose(1, 2).unsqueeze(1)


def _freqs(c):
    """Radians a position turns each pair by: base^(-2 i / rot), scaled for contexts past the trained one."""
    f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / c["rot"])
    if c["scaling"] == "linear":
        return f / 4.0
    if c["scaling"] == "ramp":                        # turns over the trained 8192 positions: between 1 and 4 blended
        keep = torch.clamp((8192.0 * f / (2 * math.pi) - 1.0) / 3.0, 0, 1)
        return f / 8.0 * (1 - keep) + f * keep
    return f


def _trees(c, seed, roots=1):
    """What every tree step knows: requests, packed tokens, and the nodes' parents within their request (-1: a root; the
    first `roots` nodes), parents before their children."""
    rows = _rows(c)
    ns = torch.tensor([n for _, n in rows], device=DEV)
    cu = torch.cat((ns.new_zeros(1), ns.cumsum(0)))
    row = torch.repeat_interleave(torch.arange(len(rows), device=DEV), ns)
    i = torch.arange(int(sum(n for _, n in rows)), device=DEV) - cu[row]
    back = torch.randint(0, 3 if c["branch"] > 1 else 1, i.shape, generator=_gen(seed, 21), device=DEV)
    up = ((i - roots) // c["branch"] - back).clamp(min=0)
    parent = torch.where(i < roots, -1, torch.minimum(up, i - 1))
    return {"c": c, "rows": rows, "row": row, "node": i, "parent": parent.to(torch.int32), "cu": cu.to(torch.int32),
            "held": _ints([h for h, _ in rows]), "lens": _ints([h + n for h, n in rows])}


def _ancestors(st, n):
    """bool [N][n]: node j of the same tree is the token itself or one of its ancestors."""
    up = torch.where(st["parent"] < 0, -1, st["cu"][st["row"]] + st["parent"]).long()
    seen = torch.nn.functional.one_hot(st["node"], n).bool()
    for _ in range(max(1, n - 1).bit_length()):                         # twice as far up every time
        seen = seen | (seen[up] & (up >= 0)[:, None])
        up = torch.where(up >= 0, up[up], up)
    return seen


def _bits(seen, words):
    """bool [N][n] as int64 words [N][words], node j in bit j mod 64 of word j / 64."""
    b = torch.nn.functional.pad(seen, (0, 64 * words - seen.shape[1])).to(torch.int64).unflatten(1, (words, 64))
    return (b << torch.arange(64, device=DEV)).sum(-1)


def _inputs(c, seed):
    return {"map": _map_inputs, "append": _append_inputs, "attend": _attend_inputs, "accept": _accept_inputs,
            "keep": _keep_inputs}[c["op"]](c, seed)


def prepare(c, seed):
    st = _inputs(c, seed)
    if own:
        from paper_2607_20538_amd import codec as cg

        st["cg"] = cg
        {"map": _plan_map, "append": _plan_append, "attend": _plan_attend, "accept": _plan_accept, "keep": _plan_keep}[c["op"]](c, st, cg)
    return st


def _map_inputs(c, seed):
    return _trees(c, seed, roots=1 + seed % 3)


def _plan_map(c, st, cg):
    st["pos"] = torch.empty_like(st["parent"])
    st["mask"] = torch.empty((len(st["parent"]), _words(c)), dtype=torch.int64, device=DEV)


def _plan_codec(c, st, cg):
    L, H, d, P, pages = c["L"], c["H"], c["d"], c["page"], _pool_pages(c)
    shp = st["shp"] = cg.shape(L, H, d, c["g"])
    st["codec"] = cg.Codec(cg.BLOCK_UNIFORM, c["bits"], c["n"]) if c["bits"] else cg.Codec(cg.PASSTHROUGH)
    st["Gd"] = cg.alloc_gauge(shp)
    cg.gauge_make(cg.GAUGE_USER, shp, params=st["G"].cpu().numpy(), G_host=None, G_dev=st["Gd"])
    st["pools"] = [cg.Cache(st["codec"], s, L, pages, H, P, d) for s in (0, 1)]
    if c["op"] != "attend" and c["bits"]:
        st["out"] = [torch.empty((L, pages, H, P, d), dtype=torch.bfloat16, device=DEV) for _ in (0, 1)]
    if "codes" in st:
        for s in (0, 1):
            st["pools"][s].codes.copy_(st["codes"][s].reshape(-1).view(torch.uint8))
            if c["bits"]:
                st["pools"][s].side.copy_(st["side"][s].reshape(-1).view(torch.uint8))


def _append_inputs(c, seed):
    st = _trees(c, seed)
    L, H, d, P, N = c["L"], c["H"], c["d"], c["page"], len(st["row"])
    mk = lambda heads, tag: _heads(_randn((L, N, heads, d), seed, tag).to(DTYPES[c["dtype"]]))             # noqa: E731
    depth = st["node"] if c["branch"] == 1 else _ancestors(st, c["new"]).sum(-1) - 1
    t = torch.arange(N, device=DEV)
    page = torch.randperm(_pool_pages(c), generator=_gen(seed, 5), device=DEV)
    st.update(G=_gauge(L, H, d, c["g"]), q=mk(H * c["grp"], 1), k=mk(H, 2), v=mk(H, 3),
              pos=(st["held"][st["row"]] + depth).to(torch.int32), slots=(page[t // P] * P + t % P).to(torch.int32))
    return st


def _plan_append(c, st, cg):
    _plan_codec(c, st, cg)
    st["qo"] = torch.empty_like(st["q"])
    st["plan"] = cg.rope_make(c["rot"], cg.ROPE_HALF if c["layout"] == "half" else cg.ROPE_PAIRS, base=10000.0,
                              scaling={"none": cg.ROPE_NONE, "linear": cg.ROPE_LINEAR, "ramp": cg.ROPE_RAMP}[c["scaling"]],
                              factor=4.0 if c["scaling"] == "linear" else 8.0, low=1.0, high=4.0, train_len=8192)


def _pools(c, st, seed):
    """Pools of coded random vectors and the requests' tables."""
    L, H, d, P, pages, rows = c["L"], c["H"], c["d"], c["page"], _pool_pages(c), st["rows"]
    st["G"] = _gauge(L, H, d, c["g"])
    scale = _key_scale(c, seed)
    st["codes"], st["side"] = [], []
    for s in (0, 1):
        codes, side = [], []
        for l in range(L):                        # a layer at a time: the pools of a long context are large
            x = _randn((1, pages, H, P, d), seed, 1 + s, l) * (scale[l:l + 1] if s == 0 else 1.0)
            z = _rotate(x, st["G"][l:l + 1, s], torch.float32)[0]
            if not c["bits"]:
                codes.append(z)
                continue
            q, mn, sc = _quantise(z, c["n"], c["bits"])
            codes.append(_pack(q.reshape(pages, H, P, d), c["bits"]))
            side.append(torch.cat((mn, sc), -1).reshape(pages, H, P, d // c["n"], 2))
        st["codes"].append(torch.stack(codes))
        st["side"].append(torch.stack(side) if side else None)
    perm = torch.randperm(pages, generator=_gen(seed, 5), device=DEV).to(torch.int32)
    need = [-(-(h + n) // P) for h, n in rows]
    st["table"] = torch.full((len(rows), max(need)), -1, dtype=torch.int32, device=DEV)
    st["table"][torch.arange(max(need), device=DEV)[None, :] < _ints(need)[:, None]] = perm[: sum(need)]
    st["free"], st["count"] = torch.zeros(pages, dtype=torch.int32, device=DEV), _ints([pages - sum(need)])
    st["free"][: pages - sum(need)] = perm[sum(need):]


def _attend_inputs(c, seed):
    st = _trees(c, seed)
    _pools(c, st, seed)
    seen = _ancestors(st, c["new"])
    st["mask"] = _bits(seen, _words(c))
    st["pos"] = (st["held"][st["row"]] + seen.sum(-1) - 1).to(torch.int32)
    st["q"] = _heads(_randn((c["L"], len(st["row"]), c["H"] * c["grp"], c["d"]), seed, 4).to(DTYPES[c["dtype"]]))
    return st


def _plan_attend(c, st, cg):
    _plan_codec(c, st, cg)
    st["pt"], st["out"] = cg.page_table(st["table"], c["page"]), _heads(torch.empty_like(st["q"][:, 0].transpose(1, 2)))
    nws = cg.attend_tree_workspace_bytes(st["shp"], c["L"], len(st["row"]), c["rows"], st["q"].shape[2], st["table"].shape[1], c["page"])
    st["ws"] = torch.empty(max(nws, 16), dtype=torch.uint8, device=DEV)


def _accept_inputs(c, seed):
    """Drafts of few different tokens, so that some siblings are alike; the model agrees with a child of most nodes."""
    roots = 1 + (2 if c["head"] else 0)
    st = _trees(c, seed, roots)
    N, B = len(st["row"]), c["rows"]
    draft = torch.randint(0, 50, (N,), generator=_gen(seed, 31), device=DEV)
    target = torch.randint(0, 50, (N + B,), generator=_gen(seed, 32), device=DEV)      # the last B: after the held positions
    liked = torch.where(torch.rand(N, generator=_gen(seed, 33), device=DEV) < 0.6, torch.arange(N, device=DEV), -1)
    up = torch.where(st["parent"] < 0, N + st["row"], st["cu"][st["row"]] + st["parent"])
    best = torch.full((N + B,), -1, device=DEV).scatter_reduce(0, up, liked, "amax")
    target = torch.where(best >= 0, draft[best.clamp(min=0)], target)
    st.update(draft=draft.to(torch.int32), target=target[:N].to(torch.int32), head=target[N:].to(torch.int32) if c["head"] else None)
    return st


def _plan_accept(c, st, cg):
    st["path"], st["kept"], st["next"] = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (len(st["row"]), c["rows"], c["rows"]))


def _paths(c, seed):
    """Every request's kept nodes, ascending.  A kept node that moves lies behind all places that are written, so that
    a pass can be repeated."""
    rng, paths = random.Random(seed * 7919 + 13), []
    for _, n in _rows(c):
        m = min(n, 1 + min(rng.randrange(8), rng.randrange(12)))
        stay = rng.randint(1, m)
        if n - m < m - stay:
            stay = m
        paths.append(list(range(stay)) + sorted(rng.sample(range(m, n), m - stay)))
    return paths


def _moved(c):
    return sum(min(n, 3) for _, n in _rows(c))           # of the paths above, on average


def _keep_inputs(c, seed):
    st = _trees(dict(c, branch=3), seed)
    _pools(c, st, seed)
    paths = _paths(c, seed)
    path = [p + [-1] * (n - len(p)) for p, (_, n) in zip(paths, st["rows"])]
    st.update(paths=paths, path=_ints(sum(path, [])), kept=_ints([len(p) for p in paths]))
    return st


def _plan_keep(c, st, cg):
    _plan_codec(c, st, cg)
    parts = [st["table"], st["free"], st["count"], st["lens"]]
    st["before"] = torch.cat([t.reshape(-1) for t in parts])
    st["now"] = st["before"].clone()
    now, at = [], 0
    for t in parts:
        now.append(st["now"][at: at + t.numel()].view(t.shape))
        at += t.numel()
    st["pages"], st["pool"], st["lens_now"] = now[0], cg.PagePool(_pool_pages(c)), now[3]
    st["pool"].free, st["pool"].count = now[1], now[2]
    st["pt"], st["held_now"] = cg.page_table(st["pages"], c["page"]), torch.empty_like(st["lens"])


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------

def run(st):
    c = st["c"]
    if own:
        return {"map": _own_map, "append": _own_append, "attend": _own_attend, "accept": _own_accept,
                "keep": _own_keep}[c["op"]](st, c, st["cg"])
    return {"map": _plain_map, "append": _plain_append, "attend": _plain_attend, "accept": _plain_accept,
            "keep": _plain_keep}[c["op"]](st, c)


def _own_map(st, c, cg):
    cg.kv_tree_map(st["parent"], st["cu"], st["lens"], st["pos"], st["mask"])
    return [st["pos"], st["mask"]]


def _own_pools(st, c, cg):
    """The pools' contents: error-free ones as they lie, coded ones recovered."""
    if not c["bits"]:
        return [p.codes.view(torch.float32).view(c["L"], -1, c["H"], c["page"], c["d"]) for p in st["pools"]]
    for s in (0, 1):
        cg.kv_decode(s, st["pools"][s], st["Gd"], st["shp"], st["codec"], 0, st["out"][s])
    return st["out"]


def _own_append(st, c, cg):
    cg.kv_append_rope(0, c["L"], st["plan"], st["k"], st["v"], st["pos"], st["slots"], st["Gd"], st["shp"], st["codec"],
                      *st["pools"], q=st["q"], q_out=st["qo"])
    return [st["qo"], *_own_pools(st, c, cg)]


def _own_attend(st, c, cg):
    cg.kv_attend_tree_paged(0, c["L"], st["q"], st["cu"], c["new"], st["mask"], *st["pools"], st["pt"], st["Gd"], st["shp"],
                            st["codec"], st["lens"], 1.0 / math.sqrt(c["d"]), st["out"], st["pos"], c["window"], c["sinks"],
                            workspace=st["ws"])
    return [st["out"]]


def _own_accept(st, c, cg):
    cg.kv_tree_accept(st["parent"], st["cu"], st["draft"], st["target"], st["path"], st["kept"], st["next"], head=st["head"])
    return [st["path"], st["kept"], st["next"]]


def _own_keep(st, c, cg):
    st["now"].copy_(st["before"])                      # every pass gives the same pages back
    cg.kv_tree_keep(0, c["L"], st["path"], st["kept"], st["cu"], st["lens_now"], st["pt"], st["codec"], *st["pools"], st["held_now"])
    cg.kv_page_trim(st["lens_now"], st["held_now"], st["pool"], st["pages"], c["page"])
    return [*_own_pools(st, c, cg), st["lens_now"], st["pages"], st["pool"].free, st["pool"].count]


def _plain_map(st, c):
    seen = _ancestors(st, c["new"])
    pos = st["held"][st["row"]] + seen.sum(-1) - 1
    return [pos.to(torch.int32), _bits(seen, _words(c))]


def _turned(x, cos, sin, c):
    """x [..., d] with its pairs turned; cos and sin [T][rot / 2]."""
    r = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., : r // 2], x[..., r // 2: r]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((y, x[..., r:]), -1)


def _recovered(z, G, s):
    """Gauge-space pool values [L][pages][H][P][d] back in the model's coordinates, bf16."""
    return _rotate(z, G[:, s], torch.float32, inverse=True).to(torch.bfloat16)


def _plain_append(st, c):
    ang = st["pos"].double()[:, None] * _freqs(c)
    cos, sin = ang.cos().float(), ang.sin().float()
    out = [_turned(st["q"].float(), cos, sin, c).to(st["q"].dtype)]
    slots = st["slots"].long()
    for s, x in enumerate((_turned(st["k"].float(), cos, sin, c), st["v"].float())):
        z = _rotate(x, st["G"][:, s], torch.float32)
        if c["bits"]:
            q, mn, sc = _quantise(z, c["n"], c["bits"])
            z = (mn.float() + q * sc.float()).reshape(z.shape)
        pool = torch.zeros((c["L"], _pool_pages(c), c["page"], c["H"], c["d"]), device=DEV)
        pool.flatten(1, 2)[:, slots] = z[:, 0].transpose(1, 2)
        pool = pool.transpose(2, 3)
        out.append(_recovered(pool, st["G"], s) if c["bits"] else pool.contiguous())
    return out


def _values(codes, side, c, dtype):
    """zhat [..., d] of coded rows."""
    if not c["bits"]:
        return codes.to(dtype)
    q, side = _unpack(codes, c["d"], c["bits"]).to(dtype).unflatten(-1, (-1, c["n"])), side.to(dtype)
    return (side[..., 0:1] + q * side[..., 1:2]).flatten(-2)


def _plain_attend(st, c):
    L, H, grp, d, B = c["L"], c["H"], c["grp"], c["d"], c["rows"]
    row, node, held = st["row"], st["node"], st["held"].long()
    q = torch.zeros((L, B, c["new"], H * grp, d), device=DEV)                                              # rows padded
    q[:, row, node] = st["q"][:, 0].transpose(1, 2).float()
    q = q.unflatten(3, (H, grp)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)                                   # [L][B][H][new grp][d]
    table = st["table"].long().clamp(min=0)
    take = lambda t: t[:, table].transpose(2, 3).flatten(3, 4)                                             # noqa: E731
    k, v = (_values(take(st["codes"][s]), take(st["side"][s]), c, torch.float32) for s in (0, 1))          # [L][B][H][T][d]
    T = k.shape[3]
    t = torch.arange(T, device=DEV)
    seen = torch.zeros((B, c["new"], T), dtype=torch.bool, device=DEV)
    far = t[None, :] < held[row][:, None]
    if c["window"]:
        far &= (t[None, :] > st["pos"].long()[:, None] - c["window"]) | (t[None, :] < c["sinks"])
    j = t[None, :] - held[row][:, None]                                        # node at this position
    word = st["mask"].gather(1, (j >> 6).clamp(0, _words(c) - 1))
    seen[row, node] = far | ((j >= 0) & (j < c["new"]) & ((word >> (j & 63)) & 1).bool())
    score = _rotate(q, st["G"][:, 0], torch.float32) @ k.transpose(-1, -2).contiguous()
    score = (score / math.sqrt(d)).unflatten(3, (c["new"], grp)).masked_fill(~seen[None, :, None, :, None], -math.inf)
    score = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    o = (score.flatten(3, 4) @ v) / score.sum(-1).flatten(3, 4)[..., None]
    o = _rotate(o, st["G"][:, 1], torch.float32, inverse=True).unflatten(3, (c["new"], grp))
    o = o.permute(0, 1, 3, 2, 4, 5)[:, row, node].flatten(2, 3)                                            # [L][N][Hq][d]
    return [_heads(o).to(st["q"].dtype)]


def _plain_accept(st, c):
    N, B, row = len(st["row"]), c["rows"], st["row"]
    i = torch.arange(N, device=DEV)
    up = torch.where(st["parent"] < 0, N + row, st["cu"][row] + st["parent"])          # places N ..: before the roots
    wanted = torch.cat((st["target"], st["head"] if c["head"] else st["target"].new_zeros(B)))[up]
    good = (st["draft"] == wanted) | (torch.zeros_like(i) if c["head"] else st["parent"] < 0).bool()
    first = torch.full((N + B,), N, device=DEV).scatter_reduce(0, up, torch.where(good, i, N), "amin")
    good = torch.cat((good & (i == first[up]), torch.ones(B, dtype=torch.bool, device=DEV)))
    far = torch.cat((up, N + torch.arange(B, device=DEV)))
    for _ in range(max(1, c["new"]).bit_length()):                              # all ancestors, twice as far up every time
        good, far = good & good[far], far[far]
    good = good[:N]
    before = torch.cat((i.new_zeros(1), good.long().cumsum(0)))[st["cu"].long()]       # kept nodes of the rows before
    kept = before[1:] - before[:-1]
    path = torch.full((N,), -1, dtype=torch.int32, device=DEV)
    at = st["cu"][row] + good.long().cumsum(0) - 1 - before[:-1][row]
    path[at[good]] = st["node"][good].to(torch.int32)
    last = torch.full((B,), -1, device=DEV).scatter_reduce(0, row, torch.where(good, i, -1), "amax")
    none = st["head"] if c["head"] else torch.full_like(st["held"], -1)
    return [path, kept.to(torch.int32), torch.where(last >= 0, st["target"][last.clamp(min=0)], none)]


def _plain_keep(st, c):
    P, row = c["page"], st["row"]
    j = torch.nonzero(st["path"] >= 0)[:, 0]                                    # place of a kept node in its row: node[j]
    where = lambda p: st["table"][row[j], (p // P)].long() * P + p % P                                     # noqa: E731
    base = st["held"][row[j]].long()
    src, dst = where(base + st["path"][j]), where(base + st["node"][j])
    out = []
    for s in (0, 1):
        moved = []
        for t in (st["codes"][s], st["side"][s]):
            if t is not None:
                flat = t.transpose(2, 3).flatten(1, 2)                          # [L][slot][H]..
                new = flat.clone()
                new[:, dst] = flat[:, src]
                moved.append(new.unflatten(1, (-1, P)).transpose(2, 3).contiguous())
        z = _values(moved[0], moved[-1], c, torch.float32)
        out.append(_recovered(z, st["G"], s) if c["bits"] else z)
    lens = st["held"] + st["kept"]
    had, need = (st["lens"] + P - 1) // P, (lens + P - 1) // P
    i = torch.arange(st["table"].shape[1], device=DEV)[None, :]
    gone = (i >= need[:, None]) & (i < had[:, None])
    free, count = st["free"].clone(), st["count"].long()
    free[count + torch.arange(int(gone.sum()), device=DEV)] = st["table"][gone]
    return [*out, lens, torch.where(gone, -1, st["table"]), free, (count + gone.sum()).to(torch.int32)]


# ------------------------------------------------------------------------------------------
# the definitions: whole numbers node by node on the host, the others in 64 bits, one layer and head at a time
# ------------------------------------------------------------------------------------------

def exact(c, seed):
    if c["op"] == "attend" and c["L"] * c["H"] * c["grp"] * sum(n * (h + n) for h, n in _rows(c)) * c["d"] > 1e11:
        return None
    return {"map": _exact_map, "append": _exact_append, "attend": _exact_attend, "accept": _exact_accept,
            "keep": _exact_keep}[c["op"]](c, _inputs(c, seed))


def _forest(st):
    """Every request's nodes as lists of parents."""
    p, cu = st["parent"].tolist(), st["cu"].tolist()
    return [p[a:b] for a, b in zip(cu, cu[1:])]


def _exact_map(c, st):
    pos, mask = [], []
    for (held, _), tree in zip(st["rows"], _forest(st)):
        seen, depth = [], []
        for i, p in enumerate(tree):
            seen.append((1 << i) | (seen[p] if p >= 0 else 0))
            depth.append(depth[p] + 1 if p >= 0 else 0)
        pos += [held + k for k in depth]
        for m in seen:
            words = [(m >> (64 * w)) & (2 ** 64 - 1) for w in range(_words(c))]
            mask.append([w - 2 ** 64 if w >= 2 ** 63 else w for w in words])
    return [_ints(pos), torch.tensor(mask, dtype=torch.int64, device=DEV)]


def _exact_accept(c, st):
    draft, target, cu = st["draft"].tolist(), st["target"].tolist(), st["cu"].tolist()
    path, kept, after = [], [], []
    for b, tree in enumerate(_forest(st)):
        d, t, way = draft[cu[b]: cu[b + 1]], target[cu[b]: cu[b + 1]], []
        want = int(st["head"][b]) if c["head"] else None
        while True:
            at = way[-1] if way else -1
            found = [i for i, p in enumerate(tree) if p == at and want in (None, d[i])]
            if not found:
                break
            way.append(found[0])
            want = t[found[0]]
        path += way + [-1] * (len(tree) - len(way))
        kept.append(len(way))
        after.append(-1 if want is None else want)
    return [_ints(path), _ints(kept), _ints(after)]


def _full(st, l, s, h):
    return torch.block_diag(*st["G"][l, s, h].double())                          # [d][d]


def _coded64(z, c):
    """The values that z [N][d] is held as."""
    if not c["bits"]:
        return z
    blocks, top = z.unflatten(-1, (-1, c["n"])), 2 ** c["bits"] - 1

    def beside(v, up):                               # the nearest binary16 not above (not below) v
        near = v.to(torch.float16).view(torch.int16)[..., None] + torch.tensor([-1, 0, 1], dtype=torch.int16, device=DEV)
        near = near.view(torch.float16).double()
        v = v[..., None]
        near = near.where((near >= v) if up else (near <= v), torch.full_like(near, math.inf if up else -math.inf))
        return near.amin(-1) if up else near.amax(-1)

    low = beside(blocks.amin(-1), False)[..., None]
    step = beside((blocks.amax(-1)[..., None] - low) / top, True)
    code = torch.where(step > 0, (blocks - low) / step, torch.zeros_like(blocks)).round().clamp(0, top)
    return (low + code * step).flatten(-2)


def _exact_append(c, st):
    """Every pair as a complex number times exp(i pos f)."""
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), st["pos"].double()[:, None] * _freqs(c))
    r, slots = c["rot"], st["slots"].long()
    pairs = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))

    def turned(x):
        y = x.double()
        w = torch.complex(y[..., pairs[0]], y[..., pairs[1]]) * turn
        y[..., pairs[0]], y[..., pairs[1]] = w.real, w.imag
        return y

    out = [turned(st["q"])]
    for s, x in enumerate((turned(st["k"]), st["v"].double())):
        pool = torch.zeros((c["L"], _pool_pages(c) * c["page"], c["H"], c["d"]), dtype=torch.float64, device=DEV)
        for l in range(c["L"]):
            for h in range(c["H"]):
                full = _full(st, l, s, h)
                z = _coded64(x[l, 0, h] @ full.T, c)
                pool[l, slots, h] = z @ full if c["bits"] else z
        out.append(pool.unflatten(1, (-1, c["page"])).transpose(2, 3))
    return out


def _exact_attend(c, st):
    """softmax(q Khat^T / sqrt(d)) Vhat with Khat, Vhat out of the gauge, a request and query head at a time."""
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    cu, P = st["cu"].tolist(), c["page"]
    for b, ((held, new), tree) in enumerate(zip(st["rows"], _forest(st))):
        n, at = held + new, cu[b]
        seen = torch.zeros((new, n), dtype=torch.bool)
        for i, p in enumerate(tree):
            if p >= 0:
                seen[i, held:] = seen[p, held:]
            seen[i, held + i] = True
            mine = held + int(seen[i, held:].sum()) - 1
            first = max(0, mine - c["window"] + 1) if c["window"] else 0
            seen[i, min(first, held): held] = True
            seen[i, : min(held, c["sinks"])] = True
        seen = seen.to(DEV)
        pg = st["table"][b, : -(-n // P)].long()
        for l in range(c["L"]):
            for h in range(c["H"]):
                K, V = (_values(st["codes"][s][l, pg, h].flatten(0, 1)[:n], st["side"][s][l, pg, h].flatten(0, 1)[:n], c, torch.float64)
                        @ _full(st, l, s, h) for s in (0, 1))
                for j in range(h * c["grp"], (h + 1) * c["grp"]):
                    x = st["q"][l, 0, j, at: at + new].double() @ K.T / math.sqrt(c["d"])
                    out[l, 0, j, at: at + new] = torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ V
    return [out]


def _exact_keep(c, st):
    P, table, lens = c["page"], st["table"].tolist(), []
    stack = st["free"].tolist()
    top, moves = int(st["count"]), []
    for b, ((held, new), way) in enumerate(zip(st["rows"], st["paths"])):
        slot = lambda p: table[b][p // P] * P + p % P                                                      # noqa: E731, B023
        moves += [(slot(held + a), slot(held + j)) for j, a in enumerate(way)]
        lens.append(held + len(way))
        for i in range(-(-lens[-1] // P), -(-(held + new) // P)):
            stack[top], table[b][i] = table[b][i], -1
            top += 1
    src, dst = torch.tensor(moves, device=DEV).T
    out = []
    for s in (0, 1):
        pool = torch.zeros((c["L"], c["H"], _pool_pages(c) * P, c["d"]), dtype=torch.float64, device=DEV)
        for l in range(c["L"]):
            for h in range(c["H"]):
                side = st["side"][s][l, :, h].flatten(0, 1) if c["bits"] else None
                z = _values(st["codes"][s][l, :, h].flatten(0, 1), side, c, torch.float64)
                z[dst] = z[src]
                pool[l, h] = z @ _full(st, l, s, h) if c["bits"] else z
        out.append(pool.unflatten(2, (-1, P)).transpose(1, 2))
    return [*out, _ints(lens), _ints(table), _ints(stack), _ints([top])]
