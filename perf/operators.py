"""Operators of a serving step over paged, gauge-coded caches: what is timed and compared.

One step of a server that batches requests of any lengths: block tables and slots from the
requests' lengths (map), rotary positions of the new queries and keys (rope), the new keys and
values encoded into the page pools through their slots (append), and attention of the new tokens
over the pools, causal or with a sliding window and visible first tokens (attend).

`run` computes each in plain torch, or with `own` through paper_2607_20538_amd.codec.  Caches that
exist before a step are built here in plain torch by the documented byte layout.  Request lengths
follow from the case, values from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------

def _map(**kw):
    return dict(dict(op="map", rows=64, new=1, ctx=8192, page=256), **kw)


def _rope(**kw):
    return dict(dict(op="rope", L=1, B=1, Hq=32, H=8, T=1024, d=128, rot=128, layout="half", scaling="none",
                     far=8192, inverse=False, dtype="bf16"), **kw)


def _append(**kw):
    return dict(dict(op="append", L=1, H=8, N=1024, pad=0, d=128, g=128, bits=4, n=64, page=256, dtype="bf16"), **kw)


def _attend(**kw):
    return dict(dict(op="attend", L=1, H=8, grp=4, d=128, g=128, bits=4, n=64, page=256, chunks=1, new=1024, singles=0,
                     ctx=4096, window=0, sinks=0, dtype="bf16"), **kw)


def listed():
    return [
        # tables and slots of a decode step of 64 requests: latency
        _map(name="map_step"),
        # ... and of 256 prompts of up to 250 new tokens, two thirds of them continued
        _map(name="map_prompts", rows=256, new=250, ctx=4000, page=64),
        # queries and keys of 32 single tokens, as each layer of a Llama-3-8B-shaped model calls it: latency
        _rope(name="rope_step", T=32),
        # a prompt of 8192 tokens of that shape at far positions, frequencies scaled for a long context
        _rope(name="rope_prompt", T=8192, scaling="ramp", far=120000),
        # gradient of an interleaved rotation of three quarters of 64-channel heads, binary32, odd count
        _rope(name="rope_grad_f32", L=2, B=3, Hq=16, H=16, T=1021, d=64, rot=48, layout="pairs", inverse=True,
              dtype="f32"),
        # one new token of 32 requests into eight layers' pools: latency
        _append(name="append_step", L=8, N=32),
        # ragged prompts of 6000 tokens in small gauge groups at 6 bits (27B-shaped: 16 KV heads)
        _append(name="append_prompts", L=2, H=16, N=6000, pad=144, g=32, bits=6),
        # the smallest configuration: two heads of 64 channels, binary32, a few odd rows
        _attend(name="attend_tiny_f32", H=2, grp=2, d=64, g=16, n=32, page=64, chunks=3, new=37, ctx=300, dtype="f32"),
        # a chunk of 4096 tokens of one long prompt of the Llama-3-8B shape
        _attend(name="attend_prompt", new=4096, ctx=20000),
        # a mixed batch: two chunks and 30 single tokens, contexts up to 8192
        _attend(name="attend_mixed", chunks=2, new=700, singles=30, ctx=8192),
        # 27B-shaped heads at 3 bits with a 1024-position window, four chunks
        _attend(name="attend_window", H=16, grp=2, g=32, bits=3, chunks=4, new=1500, ctx=6000, window=1024, sinks=4),
        # single tokens of 32 requests behind a 4096-position window with 4 sinks
        _attend(name="attend_window_step", chunks=0, singles=32, ctx=32000, window=4096, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["map", "rope", "rope", "append", "append"] + ["attend"] * 5)
    if op == "map":
        rows = _log_int(rng, 1, 512)
        return _map(rows=rows, new=_log_int(rng, 1, max(2, 100000 // rows)), ctx=_log_int(rng, 64, 30000),
                    page=rng.choice([64, 128, 256]))
    if op == "rope":
        d = rng.choice([32, 64, 80, 96, 128, 128, 256])
        H = rng.choice([1, 2, 8, 16])
        L, B, grp = rng.choice([1, 1, 4]), rng.choice([1, 1, 3]), rng.choice([1, 2, 4, 8])
        top = 8192 * 40 * 128 // (L * B * H * (grp + 1) * d)
        return _rope(L=L, B=B, Hq=H * grp, H=H, T=_log_int(rng, 1, max(2, min(20000, top))), d=d,
                     rot=rng.choice([d, d, d // 2, d // 4]), layout=rng.choice(["half", "pairs"]),
                     scaling=rng.choice(["none", "linear", "ramp"]), far=_log_int(rng, 100, 1000000),
                     inverse=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f32"]))
    H = rng.choice([1, 2, 4, 8, 16])
    if op == "append":
        d, dtype = rng.choice([(128, "bf16"), (128, "bf16"), (64, "bf16"), (96, "f32"), (256, "bf16")])
        g = rng.choice([g for g in (16, 32, 64, 128) if d % g == 0])
        L = rng.choice([1, 2, 4, 8])
        return _append(L=L, H=H, N=_log_int(rng, 1, max(2, 192000 * 128 // (L * H * d))), pad=rng.choice([0, 0, 7]), d=d, g=g,
                       bits=rng.choice([6, 8, 4]) if g >= 64 else rng.choice([6, 8]), n=rng.choice([32, 32, d // 2]) if d != 96 else 32,
                       page=rng.choice([64, 128, 256]), dtype=dtype)
    # attend: mostly 128-channel heads in bf16; the work of a draw stays under the largest listed one's
    d, dtype = rng.choice([(128, "bf16")] * 5 + [(64, "bf16"), (64, "f32"), (128, "f32"), (256, "bf16"), (80, "bf16")])
    g = d if d == 80 else rng.choice([g for g in (16, 32, 64, 128) if d % g == 0])
    bits = 4 if d == 80 else rng.choice([2, 3, 4, 4, 6, 8])
    n = 80 if d == 80 else rng.choice([32, 64])
    grp = rng.choice([1, 2, 4, 5, 8])
    chunks, singles = rng.choice([(1, 0), (1, 0), (3, 0), (2, 9), (0, 1), (0, 7), (0, 24)])
    ctx = _log_int(rng, 30, 30000)
    heads = H * grp * (4 if dtype == "f32" else 1)
    new = _log_int(rng, 2, max(3, min(4096, 1200000000 * 128 // (d * heads * max(1, chunks) * (ctx + 2000)))))
    window, sinks = rng.choice([(0, 0), (0, 0), (_log_int(rng, 16, 4096), rng.choice([0, 1, 4, 70]))])
    return _attend(H=H, grp=grp, d=d, g=g, bits=bits, n=n, page=rng.choice([64, 128, 256]), chunks=chunks, new=new,
                   singles=singles, ctx=ctx, window=window, sinks=sinks, dtype=dtype)


def _rows(c):
    """(positions held before, new tokens) of every request, from the case alone: the first one the longest."""
    rng = random.Random(f"{c['op']} {c.get('rows')} {c.get('chunks')} {c['new']} {c['ctx']} {c['page']}")
    if c["op"] == "map":
        return [(c["ctx"], c["new"])] + [(0 if c["new"] > 1 and rng.random() < 0.3 else rng.randint(0, c["ctx"]),
                                          rng.randint(1, c["new"])) for _ in range(c["rows"] - 1)]
    ctx = lambda i: c["ctx"] if i == 0 else rng.randint(c["ctx"] // 4, c["ctx"])                   # noqa: E731
    rows = [(ctx(i), c["new"] if i == 0 else rng.randint(1, c["new"])) for i in range(c["chunks"])]
    return rows + [(ctx(len(rows) + i), 1) for i in range(c["singles"])]


def _visible(c):
    """Positions that the tokens of a case see together (each token its own), and those read at least once."""
    pairs = read = 0
    w, s = c["window"], c["sinks"]
    for held, new in _rows(c):
        for p in range(held, held + new):
            pairs += p + 1 if not w or p < w else w + min(s, p + 1 - w)
        lo = max(0, held + 1 - w) if w else 0
        read += held + new - lo + min(s, lo)
    return pairs, read


def work(c):
    if c["op"] == "map":
        rows = _rows(c)
        pages = sum(-(-(h + n) // c["page"]) for h, n in rows)
        return {"bytes": 4 * (5 * len(rows) + 2 * sum(n for _, n in rows) + 2 * pages), "flops": 0}
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rope":
        el = c["L"] * c["B"] * c["T"] * (c["Hq"] + c["H"]) * c["d"]
        return {"bytes": 2 * size * el + 4 * c["B"] * c["T"], "flops": 3 * el * c["rot"] // c["d"]}
    if c["op"] == "append":
        vec = 2 * c["L"] * c["H"] * c["N"]                     # encoded, then recovered in bf16 for the comparison
        pool = 2 * c["L"] * c["H"] * _pool_pages(c) * c["page"]
        coded = c["d"] * c["bits"] // 8 + c["d"] // c["n"] * 4
        return {"bytes": vec * (size * c["d"] + coded) + pool * (coded + 2 * c["d"]),
                "flops": 2 * c["d"] * c["g"] * vec + 2 * c["d"] * c["g"] * pool}
    pairs, read = _visible(c)
    tokens = sum(n for _, n in _rows(c))
    coded = c["d"] * c["bits"] // 8 + c["d"] // c["n"] * 4
    heads = c["L"] * c["H"]
    return {"bytes": heads * (2 * coded * read + 2 * size * c["grp"] * tokens * c["d"]),
            "flops": heads * c["grp"] * (4 * c["d"] * pairs + 4 * c["d"] * c["g"] * tokens)}


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


def _gauge(L, H, d, g):
    """The model's gauge: orthogonal blocks, binary32 [L][2][H][R][g][g], the same for every input."""
    gen = torch.Generator().manual_seed(0x6A06E + 1000 * L + 100 * H + d + g)
    A = torch.randn((L * 2 * H * (d // g), g, g), generator=gen, dtype=torch.float64)
    Q, R = torch.linalg.qr(A)
    Q = (Q * torch.sign(torch.diagonal(R, dim1=-2, dim2=-1))[:, None, :]).float()
    return Q.reshape(L, 2, H, d // g, g, g).contiguous().to(DEV)


def _pool_pages(c):
    if c["op"] == "append":
        return -(-c["N"] // c["page"]) + 2
    return sum(-(-(h + n) // c["page"]) for h, n in _rows(c)) + 2


def _key_scale(c, seed):
    """Per-channel scale of the keys: log-normal, a few outlier channels, as in synth.py."""
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


def _freqs(c, dtype=torch.float64):
    """Radians a position turns each pair by: base^(-2 i / rot), scaled for contexts past the trained one."""
    f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=dtype, device=DEV) / c["rot"])
    if c["scaling"] == "linear":
        return f / 4.0
    if c["scaling"] == "ramp":                        # turns over the trained 8192 positions: between 1 and 4 blended
        keep = torch.clamp((8192.0 * f / (2 * math.pi) - 1.0) / 3.0, 0, 1)
        return f / 8.0 * (1 - keep) + f * keep
    return f


def _inputs(c, seed):
    return {"map": _map_inputs, "rope": _rope_inputs, "append": _cache_inputs, "attend": _cache_inputs}[c["op"]](c, seed)


def prepare(c, seed):
    st = _inputs(c, seed)
    if own:
        from paper_2607_20538_amd import codec as cg

        {"map": _plan_map, "rope": _plan_rope, "append": _plan_cache, "attend": _plan_cache}[c["op"]](c, st, cg)
    return st


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _map_inputs(c, seed):
    st = {"c": c}
    rows, P = _rows(c), c["page"]
    st["max_pages"] = -(-max(h + n for h, n in rows) // P) + 1
    total = sum(-(-(h + n) // P) for h, n in rows) + 5
    perm = torch.randperm(total, generator=_gen(seed, 1), device=DEV).to(torch.int32)
    had = [-(-h // P) for h, _ in rows]
    table = torch.full((len(rows), st["max_pages"]), -1, dtype=torch.int32, device=DEV)
    live = torch.arange(st["max_pages"], device=DEV)[None, :] < _ints(had)[:, None]
    table[live] = perm[: sum(had)]
    free = torch.zeros(total, dtype=torch.int32, device=DEV)
    free[: total - sum(had)] = perm[sum(had):]
    st.update(held=_ints([h for h, _ in rows]), add=_ints([n for _, n in rows]), free=free,
              count=_ints([total - sum(had)]), table=table, N=sum(n for _, n in rows) + 3)
    return st


def _plan_map(c, st, cg):
    rows = c["rows"]
    st["cg"], st["pool"], st["pages"] = cg, cg.PagePool(len(st["free"])), st["table"].clone()
    st["pool"].free.copy_(st["free"])
    st["cu"], st["lens"], st["pos"], st["slots"] = (_ints([0] * n) for n in (rows + 1, rows, st["N"], st["N"]))


def _rope_inputs(c, seed):
    st = {"c": c}
    dt = DTYPES[c["dtype"]]
    # projections [L][B][T][heads][d] as a model makes them, seen as [L][B][heads][T][d]
    mk = lambda H, tag: _randn((c["L"], c["B"], c["T"], H, c["d"]), seed, tag).to(dt).transpose(2, 3)   # noqa: E731
    start = torch.randint(0, max(1, c["far"] - c["T"]), (c["B"], 1), generator=_gen(seed, 3), device=DEV)
    st.update(q=mk(c["Hq"], 1), k=mk(c["H"], 2), pos=(start + torch.arange(c["T"], device=DEV)).to(torch.int32))
    return st


def _plan_rope(c, st, cg):
    st["cg"], st["qo"], st["ko"] = cg, torch.empty_like(st["q"]), torch.empty_like(st["k"])
    st["plan"] = cg.rope_make(c["rot"], cg.ROPE_HALF if c["layout"] == "half" else cg.ROPE_PAIRS, base=10000.0,
                              scaling={"none": cg.ROPE_NONE, "linear": cg.ROPE_LINEAR, "ramp": cg.ROPE_RAMP}[c["scaling"]],
                              factor=4.0 if c["scaling"] == "linear" else 8.0, low=1.0, high=4.0, train_len=8192)


def _cache_inputs(c, seed):
    st = {"c": c}
    L, H, d, P = c["L"], c["H"], c["d"], c["page"]
    dt, pages = DTYPES[c["dtype"]], _pool_pages(c)
    G = st["G"] = _gauge(L, H, d, c["g"])
    scale = _key_scale(c, seed) if c["op"] == "attend" else 1.0
    if c["op"] == "append":
        st["X"] = [_heads(_randn((L, c["N"] + c["pad"], H, d), seed, 1 + s).to(dt)) for s in (0, 1)]
        # few tokens: one of each request, anywhere; many: prompts in order through their pages
        t = torch.arange(c["N"], device=DEV)
        slots = torch.randperm(pages * P if c["N"] < P else pages, generator=_gen(seed, 5), device=DEV)
        slots = slots[t] if c["N"] < P else slots[t // P] * P + t % P
        st["slots"] = torch.cat((slots, slots.new_full((c["pad"],), -1))).to(torch.int32)
    else:
        rows = st["rows"] = _rows(c)
        N = sum(n for _, n in rows)
        st["q"] = _heads(_randn((L, N, H * c["grp"], d), seed, 4).to(dt))
        perm = torch.randperm(pages, generator=_gen(seed, 5), device=DEV).to(torch.int32)
        need = [-(-(h + n) // P) for h, n in rows]
        table = torch.full((len(rows), max(need)), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(max(need), device=DEV)[None, :] < _ints(need)[:, None]] = perm[: sum(need)]
        st.update(table=table, lens=_ints([h + n for h, n in rows]),
                  cu=_ints([sum(n for _, n in rows[:b]) for b in range(len(rows) + 1)]))
        st["codes"], st["side"] = [], []
        for s in (0, 1):
            codes, side = [], []
            for l in range(L):                        # a layer at a time: the pools of a long context are large
                x = _randn((1, pages, H, P, d), seed, 1 + s, l) * (scale[l:l + 1] if s == 0 else 1.0)
                q, mn, sc = _quantise(_rotate(x, G[l:l + 1, s], torch.float32), c["n"], c["bits"])
                codes.append(_pack(q.reshape(pages, H, P, d), c["bits"]))
                side.append(torch.cat((mn, sc), -1).reshape(pages, H, P, d // c["n"], 2))
            st["codes"].append(torch.stack(codes))
            st["side"].append(torch.stack(side))
    return st


def _plan_cache(c, st, cg):
    L, H, d, P, pages = c["L"], c["H"], c["d"], c["page"], _pool_pages(c)
    shp = cg.shape(L, H, d, c["g"])
    st.update(cg=cg, shp=shp, codec=cg.Codec(cg.BLOCK_UNIFORM, c["bits"], c["n"]), Gd=cg.alloc_gauge(shp))
    cg.gauge_make(cg.GAUGE_USER, shp, params=st["G"].cpu().numpy(), G_host=None, G_dev=st["Gd"])
    st["pools"] = [cg.Cache(st["codec"], s, L, pages, H, P, d) for s in (0, 1)]
    if c["op"] == "append":
        st["out"] = [torch.empty((L, pages, H, P, d), dtype=torch.bfloat16, device=DEV) for _ in (0, 1)]
        return
    for s in (0, 1):
        st["pools"][s].codes.copy_(st["codes"][s].reshape(-1))
        st["pools"][s].side.copy_(st["side"][s].reshape(-1).view(torch.uint8))
    rows, N, Hq = st["rows"], st["q"].shape[3], st["q"].shape[2]
    st.update(pt=cg.page_table(st["table"], P), max_q=max(n for _, n in rows))
    st["out"] = _heads(torch.empty((L, N, Hq, d), dtype=st["q"].dtype, device=DEV))
    nws = cg.attend_chunk_workspace_bytes(shp, L, N, len(rows), st["max_q"], Hq, st["table"].shape[1], P, c["window"],
                                          c["sinks"])
    st["ws"] = torch.empty(max(nws, 16), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------

def run(st):
    c = st["c"]
    if own:
        return {"map": _own_map, "rope": _own_rope, "append": _own_append, "attend": _own_attend}[c["op"]](st, c, st["cg"])
    return {"map": _plain_map, "rope": _plain_rope, "append": _plain_append, "attend": _plain_attend}[c["op"]](st, c)


def _own_map(st, c, cg):
    st["pool"].count.copy_(st["count"])                # every pass takes the same pages
    cg.kv_page_map(st["held"], st["add"], st["pool"], st["pages"], c["page"], st["cu"], st["lens"], st["pos"], st["slots"])
    return [st["pages"], st["pool"].count, st["cu"], st["lens"], st["pos"], st["slots"]]


def _own_rope(st, c, cg):
    cg.kv_rope(st["plan"], st["q"], st["qo"], st["pos"], st["k"], st["ko"], inverse=c["inverse"])
    return [st["qo"], st["ko"]]


def _own_append(st, c, cg):
    cg.kv_append_slots(0, c["L"], *st["X"], st["slots"], st["Gd"], st["shp"], st["codec"], *st["pools"])
    for s in (0, 1):
        cg.kv_decode(s, st["pools"][s], st["Gd"], st["shp"], st["codec"], 0, st["out"][s])
    return st["out"]


def _own_attend(st, c, cg):
    cg.kv_attend_chunk_paged(0, c["L"], st["q"], st["cu"], st["max_q"], *st["pools"], st["pt"], st["Gd"], st["shp"],
                             st["codec"], st["lens"], 1.0 / math.sqrt(c["d"]), st["out"], c["window"], c["sinks"],
                             st["ws"])
    return [st["out"]]


def _plain_map(st, c):
    held, add, P, N = st["held"].long(), st["add"].long(), c["page"], st["N"]
    lens = held + add
    zero = lens.new_zeros(1)
    cu = torch.cat((zero, add.cumsum(0)))
    had, need = (held + P - 1) // P, (lens + P - 1) // P
    first = torch.cat((zero, (need - had).cumsum(0)))                # new pages taken by the rows before
    i = torch.arange(st["max_pages"], device=DEV)[None, :]
    new = (i >= had[:, None]) & (i < need[:, None])
    rank = torch.where(new, first[:-1, None] + i - had[:, None], 0)
    table = torch.where(new, st["free"][(st["count"].long() - 1 - rank).clamp(min=0)], st["table"])
    tok = torch.arange(N, device=DEV)
    row = torch.searchsorted(cu, tok, right=True) - 1
    live = tok < cu[-1]
    row = row.clamp(max=len(held) - 1)
    pos = torch.where(live, held[row] + tok - cu[row], -1)
    slot = torch.where(live, table[row, pos.clamp(min=0) // P].long() * P + pos % P, -1)
    out = [table, st["count"] - first[-1], cu, lens, pos, slot]
    return [t.to(torch.int32) for t in out]


def _turned(x, cos, sin, c):
    """x [..., d] with its pairs turned; cos and sin [B][1][T][rot / 2]."""
    r = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., : r // 2], x[..., r // 2: r]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((y, x[..., r:]), -1)


def _plain_rope(st, c):
    ang = (st["pos"].double()[:, None, :, None] * _freqs(c)) * (-1.0 if c["inverse"] else 1.0)
    cos, sin = ang.cos().float(), ang.sin().float()
    return [_turned(x.float(), cos, sin, c).to(x.dtype) for x in (st["q"], st["k"])]


def _plain_append(st, c):
    out = []
    live = torch.nonzero(st["slots"] >= 0)[:, 0]
    slots = st["slots"][live].long()
    for s, X in enumerate(st["X"]):
        z = _rotate(X[:, :, :, live], st["G"][:, s], torch.float32)
        q, mn, sc = _quantise(z, c["n"], c["bits"])
        y = _rotate((mn.float() + q * sc.float()).reshape(z.shape), st["G"][:, s], torch.float32, inverse=True)
        pool = torch.zeros((c["L"], _pool_pages(c), c["page"], c["H"], c["d"]), dtype=torch.bfloat16, device=DEV)
        pool.flatten(1, 2)[:, slots] = y[:, 0].transpose(1, 2).to(torch.bfloat16)
        out.append(pool.transpose(2, 3))
    return out


def _row_cache(st, c, s, b, n, dtype):
    """zhat [L][H][n][d] of row b's first n positions, through the table."""
    pg = st["table"][b, : -(-n // c["page"])].long()
    take = lambda t: t[s][:, pg].transpose(1, 2).flatten(2, 3)[:, :, :n]                          # noqa: E731
    q = _unpack(take(st["codes"]), c["d"], c["bits"]).to(dtype).unflatten(-1, (-1, c["n"]))
    side = take(st["side"]).to(dtype)
    return (side[..., 0:1] + q * side[..., 1:2]).flatten(-2)


def _mask(c, held, new, n):
    """Which of n positions the new tokens of a row see."""
    p = torch.arange(held, held + new, device=DEV)[:, None]
    t = torch.arange(n, device=DEV)[None, :]
    seen = t <= p
    return seen & ((t > p - c["window"]) | (t < c["sinks"])) if c["window"] else seen


def _plain_attend(st, c):
    L, H, grp, d = c["L"], c["H"], c["grp"], c["d"]
    q = st["q"][:, 0].float().unflatten(1, (H, grp))                   # [L][H][grp][N][d]
    out = torch.empty_like(q)
    at = 0
    for b, (held, new) in enumerate(st["rows"]):                       # rows of any lengths: one after the other
        n = held + new
        k, v = (_row_cache(st, c, s, b, n, torch.float32) for s in (0, 1))
        x = q[:, :, :, at: at + new].flatten(2, 3)                     # [L][H][grp new][d]
        x = _rotate(x.unsqueeze(1), st["G"][:, 0], torch.float32)[:, 0] / math.sqrt(d)
        score = (x @ k.transpose(-1, -2).contiguous()).unflatten(2, (grp, new))
        score = score.masked_fill(~_mask(c, held, new, n), -math.inf)
        score = torch.exp(score - score.amax(-1, keepdim=True))
        o = (score.flatten(2, 3) @ v) / score.sum(-1).flatten(2, 3)[..., None]
        o = _rotate(o.unsqueeze(1), st["G"][:, 1], torch.float32, inverse=True)[:, 0]
        out[:, :, :, at: at + new] = o.unflatten(2, (grp, new))
        at += new
    return [out.flatten(1, 2).unsqueeze(1).to(st["q"].dtype)]


# ------------------------------------------------------------------------------------------
# the definitions in 64 bits, one request, layer and head at a time
# ------------------------------------------------------------------------------------------

def exact(c, seed):
    if c["op"] == "map":
        return _exact_map(c, seed)
    if c["op"] == "attend" and c["L"] * c["H"] * c["grp"] * c["d"] * _visible(c)[0] > 6e11:
        return None
    return {"rope": _exact_rope, "append": _exact_append, "attend": _exact_attend}[c["op"]](c, _inputs(c, seed))


def _exact_map(c, seed):
    """The requests one after the other, page by page and token by token, on the host."""
    st = _inputs(c, seed)
    stack = st["free"].tolist()[: int(st["count"])]
    table, P = st["table"].tolist(), c["page"]
    cu, lens, pos, slots = [0], [], [], []
    for b, (held, add) in enumerate(zip(st["held"].tolist(), st["add"].tolist())):
        for t in range(held, held + add):
            if table[b][t // P] < 0:
                table[b][t // P] = stack.pop()
            pos.append(t)
            slots.append(table[b][t // P] * P + t % P)
        cu.append(cu[-1] + add)
        lens.append(held + add)
    rest = [-1] * (st["N"] - len(pos))
    return [_ints(v) for v in (table, [len(stack)], cu, lens, pos + rest, slots + rest)]


def _exact_rope(c, st):
    """Every pair as a complex number times exp(i pos f)."""
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       st["pos"].double()[:, None, :, None] * _freqs(c) * (-1 if c["inverse"] else 1))
    out, r = [], c["rot"]
    for x in (st["q"], st["k"]):
        y = x.double()
        pairs = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
        w = torch.complex(y[..., pairs[0]], y[..., pairs[1]]) * turn
        y[..., pairs[0]], y[..., pairs[1]] = w.real, w.imag
        out.append(y)
    return out


def _exact_append(c, st):
    g, out = c["g"], []
    slots = st["slots"].long()
    for s in (0, 1):
        pool = torch.zeros((c["L"], _pool_pages(c) * c["page"], c["H"], c["d"]), dtype=torch.float64, device=DEV)
        for l in range(c["L"]):
            for h in range(c["H"]):
                full = torch.block_diag(*st["G"][l, s, h].double())    # [d][d]
                z = st["X"][s][l, 0, h, : c["N"]].double() @ full.T
                q, mn, sc = _quantise(z, c["n"], c["bits"])
                pool[l, slots[: c["N"]], h] = (mn.double() + q * sc.double()).reshape(z.shape) @ full
        out.append(pool.unflatten(1, (-1, c["page"])).transpose(2, 3))
    return out


def _exact_attend(c, st):
    """softmax(q Khat^T / sqrt(d)) Vhat with Khat, Vhat out of the gauge, a query head at a time."""
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b, (held, new) in enumerate(st["rows"]):
        n = held + new
        seen = _mask(c, held, new, n)
        kz, vz = (_row_cache(st, c, s, b, n, torch.float64) for s in (0, 1))
        for l in range(c["L"]):
            for h in range(c["H"]):
                K = kz[l, h] @ torch.block_diag(*st["G"][l, 0, h].double())
                V = vz[l, h] @ torch.block_diag(*st["G"][l, 1, h].double())
                for j in range(h * c["grp"], (h + 1) * c["grp"]):
                    s = st["q"][l, 0, j, at: at + new].double() @ K.T / math.sqrt(c["d"])
                    out[l, 0, j, at: at + new] = torch.softmax(s.masked_fill(~seen, -math.inf), -1) @ V
        at += new
    return [out]
