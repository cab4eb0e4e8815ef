"""Attention of trees of drafted tokens (kv_attend_tree_paged) against softmax attention under the same masks in binary64.

Batches, pools and error bounds are those of the chunk attention's tests; behind a row's last position the pools
hold NaN and infinities."""
import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

import _serving as S
import _tree as T
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


class Tree(Case):
    """A batch whose new tokens are the nodes of trees; masks: any, by kind; extra words beside what is needed."""

    def __init__(self, rows, kind="near", words=0, masks=None, **kw):
        super().__init__(rows, **kw)
        rng = np.random.default_rng(kw.get("seed", 1) + 77)
        self.words = max(2, -(-self.max_q // 64)) + words
        self.masks, self.hpos, self.seen = [], [], []
        for b, (held, n) in enumerate(rows):
            m, depth = T.closure(T.tree(n, kind, rng))
            if masks == "random":                          # any nodes, later ones and none among them
                m = [sum(1 << j for j in range(n) if rng.random() < 0.4) for _ in range(n)]
            elif masks == "empty":
                m = [0] * n
            pos = [held + k for k in depth]
            self.masks.append(m)
            self.hpos.append(pos)
            self.seen.append(T.seen_by(m, pos, held, self.window, self.sinks))
        w = np.full((self.N, self.words), -1, np.int64)
        pos = np.full(self.N, -1, np.int32)
        used = int(self.first[-1])
        if used:
            w[:used] = np.concatenate([T.words_of(m, self.words) for m in self.masks])
            pos[:used] = sum(self.hpos, [])
        # bits that no node has may hold anything
        for b, (_, n) in enumerate(rows):
            if n and n % 64 and n // 64 < self.words:
                w[self.first[b]: self.first[b + 1], n // 64] |= np.int64(-1) << np.int64(n % 64)
        self.mask, self.pos = torch.from_numpy(w).cuda(), torch.from_numpy(pos).cuda()

    def workspace(self, max_q=None):
        n = cg.attend_tree_workspace_bytes(self.shp, self.shp.L, self.N, len(self.rows), self.Hq, self.table.shape[1], self.P)
        return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda"), n

    def call(self, ws=None, max_q=None, stream=None):
        ws = self.workspace()[0] if ws is None else ws
        cg.kv_attend_tree_paged(0, self.shp.L, self.qd, self.cu, max_q or self.max_q, self.mask, self.kc, self.vc,
                                cg.page_table(self.pages, self.P), self.Gd, self.shp, self.codec, self.lens, self.scale, self.out,
                                self.pos if self.window else None, self.window, self.sinks, ws, self.err, stream)
        return ws

    def ref(self):
        unit = 2.0 ** -11 if self.out.dtype == torch.bfloat16 else 2.0 ** -22
        rows = [(int(self.first[b]), t, self.held[b]) for b, (_, t) in enumerate(self.rows)]
        return T.attend_masked_ref(self.q.double(), self.G, *(S.pool_values(self.codec, *p) for p in self.pools), self.table, rows,
                                   self.seen, self.P, self.scale, unit)


RAGGED = [(0, 1), (0, 16), (130, 0), (63, 1), (64, 33), (200, 70), (1, 5)]

CASES = {
    "b4": dict(rows=RAGGED),
    "b2": dict(rows=RAGGED, bits=2),
    "b3": dict(rows=RAGGED, bits=3),
    "b6": dict(rows=RAGGED, bits=6, g=128),
    "b8": dict(rows=RAGGED, bits=8, g=64),
    "n128": dict(rows=RAGGED, n=128),
    "n32": dict(rows=RAGGED, n=32, H=1),
    "n16": dict(rows=RAGGED, n=16, H=1),
    "n8_g8": dict(rows=RAGGED, n=8, H=1, g=8),
    "pass": dict(rows=RAGGED, backend=cg.PASSTHROUGH, H=1),
    "layers_p128": dict(rows=[(300, 40), (129, 3)], L=2, P=128, grp=4, g=128),
    "p192": dict(rows=[(300, 40), (191, 3)], P=192, grp=1),
    "grp3": dict(rows=[(10, 50), (100, 9)], grp=3),
    "grp5": dict(rows=[(10, 50), (100, 9)], grp=5, H=1),
    "grp40": dict(rows=[(10, 6), (100, 9)], grp=40, H=1),
    "grp130": dict(rows=[(10, 2), (100, 3)], grp=130, H=1),
    "heads_first": dict(rows=RAGGED, tokens_first=False),
    "d64": dict(rows=RAGGED, d=64, g=64, n=32),
    "d64_n64_b3": dict(rows=RAGGED, d=64, g=16, n=64, bits=3),
    "d32": dict(rows=RAGGED, d=32, g=16, n=32, H=1),
    "d8": dict(rows=[(0, 9), (70, 3)], d=8, g=8, n=8, H=1),
    "d80_g80": dict(rows=[(0, 9), (70, 33)], d=80, g=80, n=80, H=1),
    "d96_g32": dict(rows=[(0, 9), (70, 33)], d=96, g=32, n=32, H=1),
    "d256": dict(rows=[(0, 9), (170, 33)], d=256, g=128, n=64, H=1),
    "g4": dict(rows=[(0, 9), (170, 33)], g=4, H=1),
    "f32": dict(rows=RAGGED, dtype=torch.float32),
    "f32_d64": dict(rows=RAGGED, d=64, g=16, n=32, dtype=torch.float32),
    "f32_pass": dict(rows=[(0, 9), (70, 33)], backend=cg.PASSTHROUGH, dtype=torch.float32, H=1),
    "f32_d256": dict(rows=[(0, 9), (70, 33)], d=256, g=64, dtype=torch.float32, H=1),
    "f32_out": dict(rows=RAGGED, out_dtype=torch.float32),
    "bf16_out": dict(rows=RAGGED, dtype=torch.float32, out_dtype=torch.bfloat16),
    "chain": dict(rows=RAGGED, kind="chain"),
    "star": dict(rows=RAGGED, kind="star"),
    "forest": dict(rows=RAGGED, kind="forest"),
    "roots": dict(rows=RAGGED, kind="roots"),
    "random": dict(rows=RAGGED, masks="random"),
    "random_f32": dict(rows=RAGGED, masks="random", dtype=torch.float32, H=1),
    "empty": dict(rows=[(0, 9), (70, 33), (64, 3)], masks="empty"),
    "more_words": dict(rows=RAGGED, words=2),
    "window": dict(rows=RAGGED, window=50, sinks=3),
    "window_small": dict(rows=RAGGED, window=1, sinks=0),
    "window_sinks": dict(rows=[(300, 33), (700, 20), (130, 9)], window=130, sinks=70),
    "window_wide": dict(rows=RAGGED, window=10 ** 9, sinks=5),
    "window_f32": dict(rows=[(300, 33), (129, 9)], window=100, sinks=1, dtype=torch.float32, H=1),
    "window_pass": dict(rows=[(300, 33), (129, 9)], window=100, sinks=1, backend=cg.PASSTHROUGH, H=1),
    "long": dict(rows=[(5000, 30), (4099, 1), (3, 17)], P=256, H=1, grp=4),
    "long_window": dict(rows=[(5000, 30), (4099, 1), (3, 17)], P=256, H=1, grp=4, window=1000, sinks=4),
    "wide_rows": dict(rows=[(70, 1024), (0, 300)], H=1, grp=1, d=64, g=16, n=32),
    "negative_scale": dict(rows=RAGGED, scale=-0.05, H=1),
    "zero_scale": dict(rows=RAGGED, scale=0.0, H=1),
    "many_rows": dict(rows=[(k % 90, k % 4) for k in range(600)], H=1, grp=2),
    "one_token": dict(rows=[(700, 1)], pad=0),
    "ones": dict(rows=[(700, 1), (0, 1), (64, 1), (130, 0), (63, 1), (131, 1)]),
}


@pytest.mark.parametrize("name", CASES)
def test_against_binary64(name):
    c = Tree(**CASES[name])
    c.call()
    c.check()


NARROW = [(0, 1), (0, 8), (130, 0), (63, 1), (64, 5), (1200, 8), (127, 2)]   # all of a row's queries in one group of 32


@pytest.mark.parametrize("d,n", [(128, 64), (128, 32), (128, 128), (64, 64)])
@pytest.mark.parametrize("bits", [2, 3, 4, 6, 8])
def test_narrow_and_wide_tiles_of_every_width(bits, d, n):
    for rows, grp in ((NARROW, 4), (RAGGED, 2)):
        c = Tree(rows, bits=bits, d=d, n=n, g=32 if bits % 4 else 64, grp=grp, seed=bits)
        c.call()
        c.check()


@pytest.mark.parametrize("kw", [
    dict(rows=RAGGED), dict(rows=RAGGED, bits=3, d=64, g=16, n=32), dict(rows=NARROW, bits=6, grp=4),
    dict(rows=[(300, 33), (700, 20), (130, 9)], window=130, sinks=70), dict(rows=RAGGED, masks="random"),
])
def test_the_kernel_of_every_other_shape(monkeypatch, kw):
    """The shapes of the kernel over block-uniform pools, through the one that takes all of them."""
    monkeypatch.setenv("CG_KERNELS", "generic")
    c = Tree(**kw)
    c.call()
    c.check()


def test_one_layer_of_two():
    """Views of one layer read the pool's that l0 names."""
    c = Tree([(300, 40), (129, 3)], L=2, grp=4)
    c.call()
    torch.cuda.synchronize()
    both = c.out.clone()
    c.base.fill_(7.0)
    for l in (0, 1):
        cg.kv_attend_tree_paged(l, l + 1, c.qd[l: l + 1], c.cu, c.max_q, c.mask, c.kc, c.vc, cg.page_table(c.pages, c.P), c.Gd, c.shp,
                                c.codec, c.lens, c.scale, c.out[l: l + 1], None, 0, 0, c.workspace()[0], c.err)
    torch.cuda.synchronize()
    _, bound = c.ref()
    err, size = (c.out - both)[:, 0].double().cpu().norm(dim=-1), both[:, 0].double().cpu().norm(dim=-1)
    used = int(c.first[-1])    # (parts of other lengths: the error's bound from either side)
    assert (err <= 2 * bound + 2.0 ** -7 * size)[:, :, :used].all() and int(c.err.item()) == 0


def test_two_graphs_that_share_a_workspace():
    """Captured into two graphs with one workspace, replayed in turn, lengths changed in between: as eager calls."""
    cases = [Tree([(500, 30), (64, 3)], seed=1), Tree([(77, 16), (900, 9), (3, 5)], bits=3, seed=2)]
    ws = torch.empty(max(c.workspace()[1] for c in cases), dtype=torch.uint8, device="cuda")
    stream, graphs = torch.cuda.Stream(), []
    for c in cases:
        with torch.cuda.stream(stream):
            c.call(ws)
            stream.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                c.call(ws)
        graphs.append(g)
    for step in range(4):
        for c, g in zip(cases, graphs):
            c.lens.copy_(torch.tensor([h - step for h in c.held], dtype=torch.int32))
            c.base.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            got = c.out.clone()
            c.base.fill_(7.0)
            c.call(ws)
            torch.cuda.synchronize()
            assert torch.equal(got, c.out) and (got != 7.0).any()


def test_masks_of_chains_give_what_the_chunk_attention_gives():
    """The same batch through both: two roundings to bf16 and the operands' 11 bits apart (the bound of the reference, twice)."""
    rows = [(300, 40), (64, 1), (5, 17)]
    a, b = Tree(rows, kind="chain"), Case(rows)
    a.call()
    b.call()
    torch.cuda.synchronize()
    _, bound = a.ref()
    used = int(a.first[-1])
    got, want = (t.out[:, 0].double().cpu()[:, :, :used] for t in (a, b))
    assert ((got - want).norm(dim=-1) <= 2 * bound[:, :, :used] + 2.0 ** -7 * want.norm(dim=-1)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,n", [(128, 64), (64, 32), (128, 16)])
def test_hidden_positions_that_are_no_numbers(dtype, d, n):
    """Ranges of NaN, infinity and beyond binary16 at positions that some nodes see and others do not: a node that sees none of them is
    exact, one that sees a NaN gives NaN, values beyond binary16 count as they are."""
    c = Tree([(200, 20), (70, 9)], kind="roots", d=d, g=32, n=n, dtype=dtype, window=100, sinks=2)
    pool = [p[1] for p in c.pools]
    slot = lambda b, p: (c.table[b, p // 64], p % 64)  # noqa: E731
    pg, t = slot(0, 30)                                # behind every window
    for side in pool:
        side[:, pg, :, t] = np.float16("nan")
    pg, t = slot(0, 205)                               # node 5 alone
    for side in pool:
        side[:, pg, :, t] = np.float16("inf")
    pg, t = slot(0, 207)                               # node 7 alone: values up to 2^24 or so
    pool[1][:, pg, :, t, :, 1] = np.float16(60000.0)
    c.upload()
    c.call()
    torch.cuda.synchronize()
    got = c.out[:, 0].double().cpu()
    assert torch.isnan(got[:, :, 5]).all(-1).all()
    want, bound = c.ref()
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for i in list(range(5)) + list(range(6, 29)):
        err = (got - want)[:, :, i].norm(dim=-1)
        assert (err <= bound[:, :, i] + step * want[:, :, i].norm(dim=-1)).all(), i


def test_rows_that_cannot_be_taken():
    c = Tree([(60, 9), (60, 9), (60, 9), (60, 9)], H=1)
    c.lens.copy_(torch.tensor([69, 8, 10 ** 6, 69], dtype=torch.int32))
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    assert (c.out[:, 0, :, 9:27] == 0).all()
    want, bound = c.ref()
    got = c.out[:, 0].double().cpu()
    for a in (0, 27):
        assert ((got - want)[:, :, a: a + 9].norm(dim=-1) <= bound[:, :, a: a + 9] + 2.0 ** -8 * want[:, :, a: a + 9].norm(dim=-1)).all()
    c = Tree([(60, 9), (60, 9), (60, 9)], H=1)
    c.call(max_q=8)                                    # more nodes than max_q: left as they were
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE and (c.out == 7.0).all()
    c = Tree([(60, 9), (60, 9), (60, 9)], H=1)
    c.cu.copy_(torch.tensor([0, 9, 5, 27], dtype=torch.int32))
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE and (c.out[:, 0, :, 9:] == 7.0).all() and (c.out[:, 0, :, :9] != 7.0).any()


def test_rows_that_overlap():
    """More tokens in the rows than there are: no row reads or writes past the batch."""
    c = Tree([(60, 40), (60, 40), (60, 40)], H=1)
    c.cu.copy_(torch.tensor([0, 120, 0, 120], dtype=torch.int32))
    c.lens.copy_(torch.tensor([180, 180, 180], dtype=torch.int32))
    c.call(max_q=64)
    c.call(max_q=120)
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    assert (c.out[:, :, :, 120:] == 7.0).all()


def test_pages_outside_the_pool_contribute_nothing():
    c = Tree([(200, 9), (70, 3)], H=1)
    c.pages[0, 1] = 10 ** 6
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    c.seen[0][:, 64:128] = False
    want, bound = c.ref()
    got = c.out[:, 0].double().cpu()[:, :, :12]
    assert ((got - want[:, :, :12]).norm(dim=-1) <= bound[:, :, :12] + 2.0 ** -8 * want[:, :, :12].norm(dim=-1)).all()


def test_repeated_calls_are_equal_and_stay_in_their_workspace():
    c = Tree([(5000, 30), (900, 16)], P=256, H=2, grp=4, spare_pages=12)
    _, need = c.workspace()
    buf = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(3):
        c.base.fill_(7.0)
        c.call(buf[:need])
        torch.cuda.synchronize()
        outs.append(c.out.clone())
        assert (buf[need:] == 0x5A).all()
    assert need > 0 and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    c.check()


def test_a_workspace_that_is_too_small_is_refused():
    c = Tree([(5000, 30)], P=256, H=1)
    with pytest.raises(ValueError):
        c.call(torch.zeros(16, dtype=torch.uint8, device="cuda"))


def test_on_another_stream():
    c = Tree([(500, 30), (64, 3)])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.call()
    s.synchronize()
    c.check()


def test_pools_of_more_than_4_gib():
    """Append, attention, keep in the last pages of pools whose codes pass 2^32 bytes: the bytes of a small pool."""
    L, H, grp, d, P, n = 1, 8, 4, 128, 256, 64
    codec = cg.Codec(cg.BLOCK_UNIFORM, 8, n)
    many, few = 17000, 6                               # 17000 pages of 256 KiB: 4.15 GiB of codes
    shp, Gd = S.gauge_dev(S.haar(L, H, d, 128, 3))
    torch.manual_seed(5)
    rows, N = [(300, 20), (0, 12), (500, 33)], 65
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu, lens = i32([0, 20, 32, 65]), i32([320, 12, 533])
    low = np.array([[0, 1, -1, -1], [2, -1, -1, -1], [3, 4, 5, -1]], np.int32)
    rng = np.random.default_rng(3)
    masks, parent, pos = [], [], []
    for h, t in rows:
        par = T.tree(t, "near", rng)
        m, depth = T.closure(par)
        masks.append(T.words_of(m, 2))
        parent += list(par)
        pos += [h + k for k in depth]
    mask, pos = torch.from_numpy(np.concatenate(masks)).cuda(), i32(pos)
    path = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    kept = i32([2, 1, 3])
    path[0:2], path[20], path[32:35] = i32([0, 5]), 0, i32([0, 7, 20])
    x = [torch.randn((L, 1, h, N, d), device="cuda").to(torch.bfloat16) for h in (H * grp, H, H)]
    old = [torch.randn((L, 1, H, 512, d), device="cuda").to(torch.bfloat16) for _ in (0, 1)]
    plan, res = cg.rope_make(d), []
    for pages, shift in ((few, 0), (many, many - few)):
        pools = [cg.Cache(codec, s, L, pages, H, P, d) for s in (0, 1)]
        table = torch.from_numpy(np.where(low >= 0, low + shift, -1).astype(np.int32)).cuda()
        slot = lambda b, p: int(low[b][p // P] + shift) * P + p % P  # noqa: E731
        for b, (h, _) in enumerate(rows):
            if h:
                cg.kv_append_slots(0, L, *(t[:, :, :, :h] for t in old), i32([slot(b, p) for p in range(h)]), Gd, shp, codec, *pools)
        slots = i32([slot(b, h + i) for b, (h, t) in enumerate(rows) for i in range(t)])
        q, out, err, held = torch.empty_like(x[0]), torch.zeros_like(x[0]), i32([0]), i32([0, 0, 0])
        cg.kv_append_rope(0, L, plan, x[1], x[2], pos, slots, Gd, shp, codec, *pools, x[0], q, err)
        ws = torch.empty(cg.attend_tree_workspace_bytes(shp, L, N, 3, H * grp, 4, P), dtype=torch.uint8, device="cuda")
        pt = cg.page_table(table, P)
        cg.kv_attend_tree_paged(0, L, q, cu, 33, mask, *pools, pt, Gd, shp, codec, lens, d ** -0.5, out, None, 0, 0, ws, err)
        cg.kv_tree_keep(0, L, path, kept, cu, lens, pt, codec, *pools, held, err)
        torch.cuda.synchronize()
        assert int(err.item()) == 0 and held.tolist() == [302, 1, 503]
        res.append([out] + [t.view(torch.uint8).view(pages, -1)[shift: shift + few].clone() for p in pools for t in (p.codes, p.side)])
        del pools
    assert all(torch.equal(a, b) for a, b in zip(*res))
    assert (res[0][0] != 0).any(-1).all()
