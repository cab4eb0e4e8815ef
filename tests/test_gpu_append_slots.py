"""Packed tokens encoded through their slots (kv_append_slots) against the oracle's encoding of the same tokens, and a
whole serving step: tables and slots, rotary positions, keys and values into the pools, attention."""
import math

import numpy as np
import pytest
import torch

import oracle as O
from paper_2607_20538_amd import codec as cg
from paper_2607_20538_amd import synth

import _serving as S
from _parity import cache_to_host, check_fused_codes, group_rel_err, to_cg, x_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


def _pools(c, L, pages, H, P, d, fill=0xA5):
    pools = [cg.Cache(c, s, L, pages, H, P, d) for s in (0, 1)]
    for p in pools:
        for buf in (p.codes, p.side):
            if buf is not None:
                buf.fill_(fill)
    return pools


def _rows(host, slots, P):
    """Pool bytes [L][pages][H][P][...] at the slots -> [L][1][H][N][...]; everything else must hold the fill."""
    out = {"residual": None}
    for key in ("codes", "side"):
        a = host[key]
        if a is None:
            out[key] = None
            continue
        live = [i for i, s in enumerate(slots) if s >= 0]
        rows = np.stack([a[:, slots[i] // P, :, slots[i] % P] for i in live], axis=2)[:, None]
        out[key] = rows
        mask = np.ones(a.shape[1] * P, bool)
        mask[[slots[i] for i in live]] = False
        rest = np.moveaxis(a, 2, 1).reshape(a.shape[0], a.shape[2], -1, *a.shape[4:])[:, :, mask]
        assert (np.ascontiguousarray(rest).view(np.uint8) == 0xA5).all(), "bytes outside the slots were written"
    return out


CODECS = [
    # oracle codec, d, g, dtype, N
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=64), 128, 128, "bf16", 1),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=64), 128, 128, "bf16", 37),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=64), 128, 128, "bf16", 1500),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=6, block_c=64), 128, 32, "bf16", 1501),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=3, block_c=32), 128, 64, "bf16", 1033),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=8, block_c=16), 128, 16, "bf16", 1033),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=2, block_c=32), 128, 8, "bf16", 1033),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=128), 128, 128, "bf16", 700),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=32), 64, 16, "bf16", 700),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=32), 96, 32, "f32", 300),
    (O.Codec(backend=O.BLOCK_UNIFORM, bits=8, block_c=80), 80, 80, "bf16", 50),
    (O.Codec(backend=O.PASSTHROUGH), 128, 128, "bf16", 1100),
    (O.Codec(backend=O.PASSTHROUGH), 64, 64, "f32", 33),
]


@pytest.mark.parametrize("tokens_first", [True, False])
@pytest.mark.parametrize("oc,d,g,dtype,N", CODECS, ids=[str(i) for i in range(len(CODECS))])
def test_slots_match_the_oracle(oc, d, g, dtype, N, tokens_first):
    L, H, P = 2, 3, 64
    w = synth.Workload("slots", L=L, B=1, H=H, T=N, d=d, dtype=dtype, g=g, backend="bu", bits=4, data_seed=0x510 + N)
    G = O.gauge_make(O.GAUGE_HAAR, L, H, d, g, seed=9)
    shp = cg.shape(L, H, d, g)
    Gd = cg.alloc_gauge(shp)
    cg.gauge_make(cg.GAUGE_USER, shp, params=G, G_host=None, G_dev=Gd)
    c = to_cg(oc)
    pages = -(-N // P) + 2
    rng = np.random.default_rng(N)
    slots = rng.permutation(pages * P)[:N].astype(np.int64)
    skipped = rng.random(N) < 0.1
    if N > 1:
        slots[skipped] = -1 - rng.integers(0, 5, int(skipped.sum()))
    pools = _pools(c, L, pages, H, P, d)
    xs = [synth.kv_tensor(w, s) for s in (0, 1)]
    dev = []
    for x in xs:
        t = x_dev(x)
        dev.append(t.transpose(2, 3).contiguous().transpose(2, 3) if tokens_first else t)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    cg.kv_append_slots(0, L, *dev, torch.from_numpy(slots).to(torch.int32).cuda(), Gd, shp, c, *pools, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    live = slots >= 0
    for s in (0, 1):
        got = _rows(cache_to_host(pools[s], oc, s), slots.tolist(), P)
        x = np.ascontiguousarray(xs[s][:, :, :, live])
        z, _ = O.kv_encode(O.Codec(backend=O.PASSTHROUGH), s, x, G, T_cap=int(live.sum()))
        if oc.backend == O.PASSTHROUGH:
            zg = np.ascontiguousarray(got["codes"]).view(np.float32).reshape(z["codes"].shape)
            assert group_rel_err(z["codes"], zg, g) <= 1e-5
            continue
        want, _ = O.kv_encode(oc, s, x, G, T_cap=int(live.sum()))
        check_fused_codes(got, want, z["codes"], oc, s, d, int(live.sum()))


@pytest.mark.parametrize("N", [20, 1200, 2100])
def test_slots_flags_and_layers(N):
    """Layers [1, 2) alone are written; slots past the pool are flagged and skipped; a non-finite token is flagged
    and changes no other token."""
    L, H, d, P, pages = 3, 2, 128, 64, max(20, N // 64 + 2)
    oc = O.Codec(backend=O.BLOCK_UNIFORM, bits=4, block_c=64)
    c = to_cg(oc)
    G = S.haar(L, H, d, 32, 3)
    shp, Gd = S.gauge_dev(G)
    x = [torch.randn((1, 1, H, N, d), device="cuda").to(torch.bfloat16) for _ in (0, 1)]
    slots = torch.randperm(pages * P, device="cuda")[:N].to(torch.int32)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = _pools(c, L, pages, H, P, d)
    cg.kv_append_slots(1, 2, *x, slots, Gd, shp, c, *good, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    for p in good:
        for buf in (p.codes, p.side):
            v = buf.view(L, -1)
            assert (v[0] == 0xA5).all() and (v[2] == 0xA5).all() and not (v[1] == 0xA5).all()
    x2 = [t.clone() for t in x]
    x2[0][0, 0, 1, 7, 40] = float("inf")
    x2[1][0, 0, 0, N - 1, 3] = float("nan")
    far = slots.clone()
    far[3] = pages * P
    far[5] = 2 ** 31 - 1
    bad = _pools(c, L, pages, H, P, d)
    cg.kv_append_slots(1, 2, *x2, far, Gd, shp, c, *bad, err)
    torch.cuda.synchronize()
    assert int(err.item()) & cg.CG_FLAG_POS_RANGE and int(err.item()) & cg.CG_FLAG_NONFINITE
    sl = slots.cpu().tolist()
    for s in (0, 1):
        a, b = (cache_to_host(p, oc, s) for p in (good[s], bad[s]))
        for key in ("codes", "side"):
            same = a[key] == b[key]
            for i, v in enumerate(sl):
                eq = same[1, v // P, :, v % P]
                if i in (3, 5):
                    assert (np.ascontiguousarray(b[key][1, v // P, :, v % P]).view(np.uint8) == 0xA5).all()
                elif s == 0 and i == 7:
                    assert eq[0].all()
                elif s == 1 and i == N - 1:
                    assert eq[1].all()
                else:
                    assert eq.all(), (s, key, i)


def test_slots_append_continues_paged_rows(monkeypatch):
    """Slots from kv_page_map put a token where kv_append_paged puts it, byte for byte."""
    L, H, d, P, B = 2, 2, 128, 64, 5
    c = cg.Codec(cg.BLOCK_UNIFORM, 4, 64)
    G = S.haar(L, H, d, 128, 4)
    shp, Gd = S.gauge_dev(G)
    held = [0, 63, 64, 100, 5]
    pool = cg.PagePool(16)
    pages = torch.full((B, 4), -1, dtype=torch.int32)
    free = pool.free.cpu().tolist()
    for b, h in enumerate(held):
        for i in range(-(-h // P)):
            pages[b, i] = free.pop()
    pool.count.fill_(len(free))
    pages = pages.cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, cu, pos, slots, err = i32(held), i32([0] * (B + 1)), i32([0] * B), i32([0] * B), i32([0])
    cg.kv_page_map(lens, i32([1] * B), pool, pages, P, cu, lens, pos, slots, err)
    k, v = (torch.randn((L, B, H, 1, d), device="cuda").to(torch.bfloat16) for _ in (0, 1))
    one, two = _pools(c, L, 16, H, P, d), _pools(c, L, 16, H, P, d)
    cg.kv_append_paged(0, L, k, v, pos, cg.page_table(pages, P), Gd, shp, c, *one, err)
    packed = [t.permute(0, 3, 2, 1, 4) for t in (k, v)]
    cg.kv_append_slots(0, L, *packed, slots, Gd, shp, c, *two, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    for a, b in zip(one, two):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.side, b.side)


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
def test_a_serving_run(window, sinks):
    """Three requests of any lengths over four steps, two layers: prompts in chunks, single tokens beside them, one
    request done and its pages taken by a new one.  Every step's outputs against attention in binary64 over the keys
    and values that the pools decode to at the rows' positions; the keys against the rotated inputs by the codec's
    step.  8 bits, so that a wrong position or slot stands far out."""
    L, H, grp, d, P, maxp = 2, 2, 2, 128, 64, 6
    c = cg.Codec(cg.BLOCK_UNIFORM, 8, 64)
    G = S.haar(L, H, d, 32, 8)
    shp, Gd = S.gauge_dev(G)
    npages = 14
    pool = cg.PagePool(npages)
    pools = [cg.Cache(c, s, L, npages, H, P, d) for s in (0, 1)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    B, Nmax = 3, 200
    lens, pages = i32([0] * B), torch.full((B, maxp), -1, dtype=torch.int32, device="cuda")
    cu, pos, slots, err = i32([0] * (B + 1)), i32([0] * Nmax), i32([0] * Nmax), i32([0])
    plan = cg.rope_make(d, cg.ROPE_HALF)
    rng = np.random.default_rng(12)
    past = [[[], []] for _ in range(B)]            # rotated keys and values of every row, [L][H][t][d]
    scale = 1 / math.sqrt(d)
    for step, add in enumerate(([130, 0, 40], [60, 1, 1], [1, 90, 1], [1, 1, 100])):
        if step == 3:
            done = i32([0, 0, 1])
            cg.kv_page_release(lens, done, pool, pages, P, err)
            past[2] = [[], []]
        cg.kv_page_map(lens, i32(add), pool, pages, P, cu, lens, pos, slots, err)
        q = torch.from_numpy(rng.standard_normal((L, Nmax, H * grp, d))).to(torch.bfloat16).cuda().transpose(1, 2).unsqueeze(1)
        k, v = (torch.from_numpy(rng.standard_normal((L, Nmax, H, d))).to(torch.bfloat16).cuda().transpose(1, 2).unsqueeze(1)
                for _ in (0, 1))
        raw = q.double().cpu(), k.double().cpu()
        cg.kv_rope(plan, q, q, pos.view(1, -1), k, k)
        cg.kv_append_slots(0, L, k, v, slots, Gd, shp, c, *pools, err)
        out = torch.full_like(q, 7.0)
        ws = torch.empty(max(16, cg.attend_chunk_workspace_bytes(shp, L, Nmax, B, 130, H * grp, maxp, P, window, sinks)),
                         dtype=torch.uint8, device="cuda")
        cg.kv_attend_chunk_paged(0, L, q, cu, 130, *pools, cg.page_table(pages, P), Gd, shp, c, lens, scale, out, window,
                                 sinks, ws, err)
        dec = [torch.empty((L, npages, H, P, d), dtype=torch.float32, device="cuda") for _ in (0, 1)]
        for s in (0, 1):
            cg.kv_decode(s, pools[s], Gd, shp, c, 0, dec[s])
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        n = sum(add)
        posh = pos.cpu().view(1, -1)
        for got, x in ((q, raw[0]), (k, raw[1])):
            want = S.rope_ref(x, posh, d, cg.ROPE_HALF)
            assert ((got.double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19)[:, :, :, :n].all()
        table, first = pages.cpu(), cu.cpu().tolist()
        got = out[:, 0].double().cpu()
        assert (got[:, :, n:] == 7.0).all()
        for b in range(B):
            a0, a1, held = first[b], first[b + 1], int(lens[b])
            for s, x in enumerate((k, v)):
                past[b][s].append(x[:, 0, :, a0:a1].double().cpu())
            if a1 == a0:
                continue
            K, V = (dec[s].double().cpu()[:, table[b, : -(-held // P)].long()].transpose(1, 2).flatten(2, 3)[:, :, :held]
                    for s in (0, 1))
            for s, D in ((0, K), (1, V)):
                X = torch.cat(past[b][s], 2)
                # half a step of 8 bits over a range of at most 10 sigma, in the 2-norm of 128 channels
                assert (X - D).norm(dim=-1).max() <= 10 / 255 / 2 * math.sqrt(d)
            for l in range(L):
                for j in range(H * grp):
                    x = q[l, 0, j, a0:a1].double().cpu()
                    t = torch.stack([S.visible(held - (a1 - a0) + i, held, window, sinks) for i in range(a1 - a0)])
                    sc = (scale * x @ K[l, j // grp].T).masked_fill(~t, -math.inf)
                    o = torch.softmax(sc, -1) @ V[l, j // grp]
                    # scores below 40 in binary16 operands: 2 (2 2^-11 sum |q k| scale) and the result's rounding
                    A = scale * (x.abs() @ K[l, j // grp].abs().T).max().item()
                    lim = (math.expm1(4 * 2 * 2.0 ** -11 * A) + 2.0 ** -9) * V[l, j // grp].norm(dim=-1).max() + 2.0 ** -8 * o.norm(dim=-1)
                    assert ((got[l, j, a0:a1] - o).norm(dim=-1) <= lim).all()


@pytest.mark.parametrize("bits,n", [(4, 64), (6, 16), (3, 32)])
def test_slots_long_ranges_of_a_workgroup(monkeypatch, bits, n):
    """The bytes do not depend on how many tiles of tokens a workgroup takes, nor on the tokens beside a skipped one."""
    L, H, d, P, N = 1, 2, 128, 64, 2501
    pages = N // P + 2
    c = cg.Codec(cg.BLOCK_UNIFORM, bits, n)
    shp, Gd = S.gauge_dev(S.haar(L, H, d, 64, 7))
    torch.manual_seed(N + bits)
    x = [torch.randn((L, 1, N, H, d), device="cuda").to(torch.bfloat16).transpose(2, 3) for _ in (0, 1)]
    x[0][0, 0, 1, 2200, 5] = float("inf")
    slots = torch.randperm(pages * P, device="cuda")[:N].to(torch.int32)
    slots[::97] = -1
    got = []
    for tiles in ("1", "3", "40", ""):
        monkeypatch.setenv("CG_TILES_PER_WG", tiles)
        pools = _pools(c, L, pages, H, P, d)
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        cg.kv_append_slots(0, L, *x, slots, Gd, shp, c, *pools, err)
        torch.cuda.synchronize()
        # the infinite token's block ranges are infinite in binary16 too
        assert int(err.item()) == cg.CG_FLAG_NONFINITE | cg.CG_FLAG_SIDE_OVERFLOW
        got.append([(p.codes.clone(), p.side.clone()) for p in pools])
    for g in got[1:]:
        for (ca, sa), (cb, sb) in zip(got[0], g):
            assert torch.equal(ca, cb) and torch.equal(sa, sb)


def test_captured_steps_follow_the_lengths():
    """A step of single tokens captured once (tables, rotary positions, append, attention) and replayed six times, the
    lengths moving on the device, eager work between the replays: the same bytes and outputs as eager steps."""
    L, H, grp, d, P, maxp, B = 2, 2, 4, 128, 64, 8, 3
    c = cg.Codec(cg.BLOCK_UNIFORM, 4, 64)
    shp, Gd = S.gauge_dev(S.haar(L, H, d, 128, 8))
    plan = cg.rope_make(d)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    torch.manual_seed(3)
    x = [torch.randn((6, L, B, h, d), device="cuda").to(torch.bfloat16) for h in (H * grp, H, H)]

    class Server:
        def __init__(self):
            self.pool = cg.PagePool(20)
            self.pools = [cg.Cache(c, s, L, 20, H, P, d) for s in (0, 1)]
            self.lens, self.add = i32([0, 62, 300]), i32([1, 1, 1])
            self.pages = torch.full((B, maxp), -1, dtype=torch.int32, device="cuda")
            self.cu, self.pos, self.slots, self.err = i32([0] * (B + 1)), i32([0] * B), i32([0] * B), i32([0])
            # the pages of what the rows hold already: all zeros
            cu, pos, slots = i32([0] * (B + 1)), i32([0] * 400), i32([0] * 400)
            cg.kv_page_map(i32([0, 0, 0]), self.lens.clone(), self.pool, self.pages, P, cu, self.lens, pos, slots, self.err)
            self.q, self.k, self.v = (torch.zeros((L, B, h, d), dtype=torch.bfloat16, device="cuda").transpose(1, 2).unsqueeze(1)
                                      for h in (H * grp, H, H))
            self.out = torch.zeros_like(self.q)
            n = cg.attend_chunk_workspace_bytes(shp, L, B, B, 1, H * grp, maxp, P)
            self.ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")

        def load(self, i):
            for t, src in zip((self.q, self.k, self.v), x):
                t.copy_(src[i].transpose(1, 2).unsqueeze(1))

        def step(self):
            cg.kv_page_map(self.lens, self.add, self.pool, self.pages, P, self.cu, self.lens, self.pos, self.slots, self.err)
            cg.kv_rope(plan, self.q, self.q, self.pos.view(1, -1), self.k, self.k)
            cg.kv_append_slots(0, L, self.k, self.v, self.slots, Gd, shp, c, *self.pools, self.err)
            cg.kv_attend_chunk_paged(0, L, self.q, self.cu, 1, *self.pools, cg.page_table(self.pages, P), Gd, shp, c, self.lens,
                                     1 / math.sqrt(d), self.out, workspace=self.ws, err_flag=self.err)

        def state(self):
            return [t.clone() for t in (self.out, self.lens, self.pages, self.pool.count, self.pos, self.slots, self.err,
                                        *(b for p in self.pools for b in (p.codes, p.side)))]

    eager, want = Server(), []
    for i in range(6):
        eager.load(i)
        eager.step()
        torch.cuda.synchronize()
        want.append(eager.state())
    assert int(eager.err.item()) == 0 and eager.lens.tolist() == [6, 68, 306]
    s = Server()
    first = [t.clone() for t in (s.lens, s.pages, s.pool.count)]
    s.load(0)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        s.step()
    for t, v in zip((s.lens, s.pages, s.pool.count), first):
        t.copy_(v)
    for i in range(6):
        s.load(i)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(s.state(), want[i]):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("d,g,N", [(128, 128, 70), (128, 32, 2200), (64, 64, 70)])
def test_slices_of_a_fused_projection(d, g, N):
    """Queries, keys and values as slices of one [N][(Hq + 2 H) d] tensor, rows 16 channels apart, turned in place:
    the same bytes and outputs as from tensors of their own, and nothing else of the projection changes."""
    H, Hq, P = 2, 6, 64
    pages = -(-N // P) + 1
    c = cg.Codec(cg.BLOCK_UNIFORM, 4, 32)
    shp, Gd = S.gauge_dev(S.haar(1, H, d, g, 5))
    plan = cg.rope_make(d, cg.ROPE_PAIRS)
    torch.manual_seed(N + d)
    wide = (Hq + 2 * H) * d + 16
    fused = torch.randn((N, wide), device="cuda").to(torch.bfloat16)
    before = fused.clone()

    def cut(t):
        h = t[:, : (Hq + 2 * H) * d].view(N, Hq + 2 * H, d).transpose(0, 1)[None, None]
        return h[:, :, :Hq], h[:, :, Hq: Hq + H], h[:, :, Hq + H:]

    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    table = torch.randperm(pages, device="cuda").to(torch.int32)[None]
    slots = (table[0, (pos // P).long()] * P + pos % P).to(torch.int32)
    res = []
    for own in (False, True):
        q, k, v = (t.contiguous() if own else t for t in cut(before.clone() if own else fused))
        cg.kv_rope(plan, q, q, pos.view(1, -1), k, k)
        pools = _pools(c, 1, pages, H, P, d)
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        cg.kv_append_slots(0, 1, k, v, slots, Gd, shp, c, *pools, err)
        out = torch.zeros((N, wide), dtype=torch.bfloat16, device="cuda")
        o = torch.zeros_like(q) if own else cut(out)[0]
        n = cg.attend_chunk_workspace_bytes(shp, 1, N, 1, N, Hq, pages, P, 500, 4)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        cg.kv_attend_chunk_paged(0, 1, q, i32([0, N]), N, *pools, cg.page_table(table, P), Gd, shp, c, i32([N]), d ** -0.5, o, 500,
                                 4, ws, err)
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        if not own:
            assert (out[:, Hq * d:] == 0).all()
            assert torch.equal(fused[:, (Hq + H) * d:], before[:, (Hq + H) * d:])
        res.append([q.clone(), k.clone(), o.clone(), *(b.clone() for p in pools for b in (p.codes, p.side))])
    for a, b in zip(*res):
        assert torch.equal(a, b)
