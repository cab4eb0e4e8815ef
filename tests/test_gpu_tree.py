"""Trees of drafted tokens: positions and masks, greedy checks, kept paths moved together, rows shortened, against the
same things done node by node on the host; and a whole step, eager and captured."""
import math

import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

import _serving as S
import _tree as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def packed(sizes, kinds, rng):
    """(trees, cu, all parents)"""
    trees = [T.tree(n, kinds[b % len(kinds)], rng) for b, n in enumerate(sizes)]
    return trees, np.cumsum([0] + list(sizes)).tolist(), sum(trees, [])


SIZES = {"one": [1], "small": [1, 0, 2, 16, 33], "words": [63, 64, 65, 0, 128, 127, 129], "wide": [300, 5, 1024, 1023],
         "many": [7] * 500}
KINDS = ["near", "chain", "star", "forest", "roots"]


# ------------------------------------------------------------------------------------------
# positions and masks
# ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
@pytest.mark.parametrize("first", range(3))
def test_tree_map(sizes, first):
    rng = np.random.default_rng(first)
    trees, cu, parents = packed(sizes, KINDS[first:] + KINDS[:first], rng)
    pad, words = 3, -(-max(sizes) // 64) + first
    words = max(1, words)
    N = cu[-1] + pad
    held = rng.integers(0, 100000, len(sizes)).tolist()
    pos, mask = torch.full((N,), 77, dtype=torch.int32, device="cuda"), torch.full((N, words), 5, dtype=torch.int64, device="cuda")
    err = i32([0])
    cg.kv_tree_map(i32(parents + [9] * pad), i32(cu), i32([h + n for h, n in zip(held, sizes)]), pos, mask, err)
    torch.cuda.synchronize()
    want_pos, want = [], []
    for h, t in zip(held, trees):
        m, depth = T.closure(t)
        want_pos += [h + k for k in depth]
        want += m
    assert int(err.item()) == 0
    assert pos.tolist() == want_pos + [-1] * pad
    assert np.array_equal(mask.cpu().numpy(), np.concatenate([T.words_of(want, words), np.zeros((pad, words), np.int64)]))


def test_tree_map_flags():
    """Parents that are no earlier nodes, lengths below the nodes, rows that cannot be taken: each its own row's matter."""
    N = 12
    parents = [-1, 0, 5, -7, -1, 0, 1, -1, 0, -1, 0, 1]
    # row 0: nodes 0 .. 3 (parents 5 and -7 are none); row 1: length 2 of 3 nodes; row 2: runs backwards; row 3 after it: past N
    for cu, lens, bad in (([0, 4, 7, 5, 13], [10, 2, 9, 9], True), ([0, 2, 4, 7, 12], [10, 12, 13, 15], True)):
        pos, mask, err = torch.full((N,), 77, dtype=torch.int32, device="cuda"), torch.full((N, 1), 5, dtype=torch.int64, device="cuda"), i32([0])
        cg.kv_tree_map(i32(parents), i32(cu), i32(lens), pos, mask, err)
        torch.cuda.synchronize()
        assert int(err.item()) == cg.CG_FLAG_POS_RANGE
        if cu[1] == 4:
            assert pos.tolist() == [6, 7, 6, 6] + [-1] * 3 + [77] * 5
            assert mask[:, 0].tolist() == [1, 3, 4, 8] + [1, 3, 7] + [5] * 5
    # more nodes than a mask holds
    pos, mask, err = torch.full((70,), 77, dtype=torch.int32, device="cuda"), torch.full((70, 1), 5, dtype=torch.int64, device="cuda"), i32([0])
    cg.kv_tree_map(i32([-1] * 70), i32([0, 65, 70]), i32([65, 5]), pos, mask, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE and pos.tolist() == [77] * 65 + [0] * 5


# ------------------------------------------------------------------------------------------
# greedy checks
# ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
@pytest.mark.parametrize("head", [False, True])
@pytest.mark.parametrize("vocab", [1, 3, 100])
def test_tree_accept(sizes, head, vocab):
    rng = np.random.default_rng(vocab)
    trees, cu, parents = packed(sizes, KINDS, rng)
    N = cu[-1] + 2
    draft, target = rng.integers(0, vocab, N).tolist(), rng.integers(0, vocab, N).tolist()
    heads = rng.integers(0, vocab, len(sizes)).tolist()
    path, kept, nxt, err = i32([9] * N), i32([9] * len(sizes)), i32([9] * len(sizes)), i32([0])
    cg.kv_tree_accept(i32(parents + [0] * 2), i32(cu), i32(draft), i32(target), path, kept, nxt, i32(heads) if head else None, err)
    torch.cuda.synchronize()
    want, lens, after = [], [], []
    for b, t in enumerate(trees):
        way, last = T.walk(t, draft[cu[b]: cu[b + 1]], target[cu[b]: cu[b + 1]], heads[b] if head else None)
        want += way + [-1] * (len(t) - len(way))
        lens.append(len(way))
        after.append(last)
    assert int(err.item()) == 0
    assert path.tolist() == want + [-1] * 2 and kept.tolist() == lens and nxt.tolist() == after


def test_tree_accept_flags():
    path, kept, nxt, err = i32([9] * 6), i32([9] * 2), i32([9] * 2), i32([0])
    # node 1 has itself as its parent, node 2 a later one: neither is kept
    cg.kv_tree_accept(i32([-1, 1, 3, 0, 0, 0]), i32([0, 4, 9]), i32([5] * 6), i32([5] * 6), path, kept, nxt, None, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE
    assert path.tolist() == [0, 3, -1, -1, 9, 9] and kept.tolist() == [2, 0] and nxt.tolist() == [5, -1]


# ------------------------------------------------------------------------------------------
# kept paths
# ------------------------------------------------------------------------------------------

class Pools:
    def __init__(self, rows, codec, L, H, P, d, seed):
        rng = self.rng = np.random.default_rng(seed)
        self.rows, self.codec, self.P = rows, codec, P
        need = [-(-(h + n) // P) for h, n in rows]
        pages = sum(need) + 2
        perm = rng.permutation(pages).astype(np.int32)
        self.table = np.full((len(rows), max(1, max(need)) + 1), -1, np.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = perm[at: at + k]
            at += k
        self.host = [S.random_pool(codec, L, pages, H, P, d, rng) for _ in (0, 1)]
        self.dev = [S.pool_dev(codec, s, *self.host[s]) for s in (0, 1)]
        self.pages = torch.from_numpy(self.table).cuda()
        self.free = perm[at:].tolist()
        self.pool = cg.PagePool(pages)
        self.pool.free[: len(self.free)].copy_(i32(self.free))
        self.pool.count.fill_(len(self.free))
        self.cu = np.cumsum([0] + [n for _, n in rows]).tolist()
        self.lens = [h + n for h, n in rows]

    def slot(self, b, p):
        return self.table[b, p // self.P], p % self.P

    def moved(self, paths, l0, l1):
        """The pools' bytes after the paths' entries moved."""
        out = []
        for codes, side in self.host:
            new = [None if t is None else t.copy() for t in (codes, side)]
            for b, ((base, _), way) in enumerate(zip(self.rows, paths)):
                for j, a in enumerate(way):
                    (ps, ts), (pd, td) = self.slot(b, base + a), self.slot(b, base + j)
                    for t, n in zip((codes, side), new):
                        if t is not None:
                            n[l0:l1, pd, :, td] = t[l0:l1, ps, :, ts]
            out.append(new)
        return out

    def same(self, want):
        for dev, (codes, side) in zip(self.dev, want):
            assert np.array_equal(dev.codes.cpu().numpy(), np.ascontiguousarray(codes).view(np.uint8).reshape(-1))
            if side is not None:
                assert np.array_equal(dev.side.cpu().numpy(), np.ascontiguousarray(side).view(np.uint8).reshape(-1))


BU = lambda bits, n: cg.Codec(cg.BLOCK_UNIFORM, bits, n)  # noqa: E731
PASS = cg.Codec(cg.PASSTHROUGH)

KEEPS = {
    "b4": (BU(4, 64), 2, 3, 64, 128, [(0, 16), (60, 16), (200, 1), (127, 64), (64, 0), (1, 37)]),
    "b3": (BU(3, 32), 1, 2, 64, 64, [(0, 16), (60, 16), (200, 1), (127, 64)]),
    "b2_d80": (BU(2, 16), 1, 2, 64, 80, [(60, 30), (3, 70)]),
    "b6_d96": (BU(6, 32), 1, 2, 128, 96, [(60, 30), (120, 170)]),
    "b8_d8": (BU(8, 8), 3, 1, 64, 8, [(60, 30), (3, 70)]),
    "b4_d8": (BU(4, 8), 1, 1, 64, 8, [(60, 30), (3, 70)]),
    "pass": (PASS, 2, 2, 64, 128, [(0, 16), (60, 16), (200, 1), (127, 64)]),
    "pass_d256_long": (PASS, 1, 1, 64, 256, [(33, 1024), (60, 130)]),
    "b4_long": (BU(4, 64), 1, 2, 64, 128, [(33, 1024), (60, 1000), (0, 1)]),
    "rows": (BU(4, 64), 4, 8, 64, 128, [(k % 90, 1 + k % 23) for k in range(300)]),
}


@pytest.mark.parametrize("how", ["any", "all", "none", "last", "shifted"])
@pytest.mark.parametrize("name", KEEPS)
def test_kept_paths_move_together(name, how):
    codec, L, H, P, d, rows = KEEPS[name]
    p = Pools(rows, codec, L, H, P, d, 5)
    paths = []
    for _, n in rows:
        m = int(p.rng.integers(0, n + 1))
        paths.append({"any": sorted(p.rng.permutation(n)[:m].tolist()), "all": list(range(n)), "none": [],
                      "last": [n - 1] if n else [], "shifted": list(range(1, n))}[how])
    path = sum((w + [-1] * (n - len(w)) for w, (_, n) in zip(paths, rows)), [])
    held, err, lens = i32([9] * len(rows)), i32([0]), i32(p.lens)
    l0, l1 = (1, L) if L > 2 else (0, L)
    cg.kv_tree_keep(l0, l1, i32(path + [3]), i32([len(w) for w in paths]), i32(p.cu), lens, cg.page_table(p.pages, P), codec,
                    *p.dev, held, err)
    cg.kv_page_trim(lens, held, p.pool, p.pages, P, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    p.same(p.moved(paths, l0, l1))
    table, free = p.table.copy(), list(p.free)
    want = [h + len(w) for (h, _), w in zip(rows, paths)]
    for b, (h, n) in enumerate(rows):
        for i in range(-(-want[b] // P), -(-(h + n) // P)):
            free.append(int(table[b, i]))
            table[b, i] = -1
    assert held.tolist() == want and lens.tolist() == want
    assert np.array_equal(p.pages.cpu().numpy(), table)
    assert int(p.pool.count.item()) == len(free) and p.pool.free[: len(free)].tolist() == free


def test_paths_that_cannot_be_kept():
    """A path that does not ascend, leaves its row, or is longer than it; lengths below the nodes: the row is left, the others go on."""
    rows = [(10, 8)] * 7
    p = Pools(rows, BU(4, 64), 1, 2, 64, 128, 6)
    ways = [[0, 3, 3], [0, 2, 9], [1, 4], [4, 1], [0, 1], [-1, 2], [0, 5]]
    kept = [3, 3, 2, 2, 9, 2, 2]
    path = sum((w + [-1] * (8 - len(w)) for w in ways), [])
    lens, held, err = i32([18, 18, 18, 18, 18, 18, 7]), i32([9] * 7), i32([0])
    cg.kv_tree_keep(0, 1, i32(path), i32(kept), i32(p.cu), lens, cg.page_table(p.pages, 64), p.codec, *p.dev, held, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE
    assert held.tolist() == [10, 10, 12, 10, 10, 10, 7]
    p.same(p.moved([[], [], [1, 4], [], [], [], []], 0, 1))


def test_lengths_that_are_none():
    """Lengths that no row has, down to the least int32: flagged, nothing of the row moved, read or written."""
    low, high = -2 ** 31, 2 ** 31 - 1
    pos, mask, err = torch.full((8,), 77, dtype=torch.int32, device="cuda"), torch.zeros((8, 1), dtype=torch.int64, device="cuda"), i32([0])
    cg.kv_tree_map(i32([-1, 0] * 4), i32([0, 2, 4, 6, 8]), i32([low, low + 1, -1, 9]), pos, mask, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE and pos.tolist() == [-1] * 6 + [7, 8] and mask[:, 0].tolist() == [1, 3] * 4
    rows = [(10, 8)] * 5
    p = Pools(rows, BU(4, 64), 1, 2, 64, 128, 6)
    lens, held, err = i32([low, low + 7, -1, high, 18]), i32([9] * 5), i32([0])
    pt = cg.page_table(p.pages, 64)
    cg.kv_tree_keep(0, 1, i32(([0, 3, 5] + [-1] * 5) * 5), i32([3] * 5), i32(p.cu), lens, pt, p.codec, *p.dev, held, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE and held.tolist() == [low, low + 7, -1, high - 8, 13]
    p.same(p.moved([[], [], [], [], [0, 3, 5]], 0, 1))
    before, err = p.pages.clone(), i32([0])
    cg.kv_page_trim(lens, i32([low, low + 7, -1, 3, 13]), p.pool, p.pages, 64, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE and lens.tolist() == [low, low + 7, -1, high, 13] and torch.equal(before, p.pages)


def test_pages_outside_the_pool_are_not_moved():
    rows = [(60, 10), (5, 4)]
    p = Pools(rows, BU(4, 64), 1, 2, 64, 128, 7)
    p.pages[0, 1] = 10 ** 6                             # positions 64 .. 69: nodes 4 .. 9
    held, err = i32([9, 9]), i32([0])
    cg.kv_tree_keep(0, 1, i32([1, 3, 5, 9] + [-1] * 6 + [0, 2, -1, -1]), i32([4, 2]), i32(p.cu), i32(p.lens),
                    cg.page_table(p.pages, 64), p.codec, *p.dev, held, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE and held.tolist() == [64, 7]
    want = p.moved([[1, 3], [0, 2]], 0, 1)
    p.same(want)


def test_trim():
    """Rows kept whole, shortened to any length and emptied; rows that cannot be are left; many rows over one round."""
    P = 64
    rows = [(0, 200), (0, 200), (0, 64), (0, 1), (0, 130), (0, 130), (0, 0)] + [(0, 65 + k % 100) for k in range(1200)]
    keep = [200, 64, 0, 0, -1, 131, 0] + [k % 66 for k in range(1200)]
    need = [-(-n // P) for _, n in rows]
    rng = np.random.default_rng(8)
    perm = rng.permutation(sum(need) + 3).astype(np.int32)
    table = np.full((len(rows), 5), -1, np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = perm[at: at + k]
        at += k
    pool = cg.PagePool(len(perm))
    pool.free[:3].copy_(torch.from_numpy(perm[at:].copy()))
    pool.count.fill_(3)
    pages, lens, err = torch.from_numpy(table).cuda(), i32([n for _, n in rows]), i32([0])
    cg.kv_page_trim(lens, i32(keep), pool, pages, P, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE
    free, want = perm[at:].tolist(), []
    for b, (_, n) in enumerate(rows):
        k = keep[b] if 0 <= keep[b] <= n else n
        want.append(k)
        for i in range(-(-k // P), need[b]):
            free.append(int(table[b, i]))
            table[b, i] = -1
    assert lens.tolist() == want and np.array_equal(pages.cpu().numpy(), table)
    assert int(pool.count.item()) == len(free) and pool.free[: len(free)].tolist() == free


# ------------------------------------------------------------------------------------------
# a whole step
# ------------------------------------------------------------------------------------------

class Step:
    """One step that checks trees, on buffers of fixed size; every other request brings a tree, the others one token."""

    def __init__(self, H=2, grp=2, d=128, g=64, P=64, bits=4, dtype=torch.bfloat16, seed=3, window=0, sinks=0, held=(100, 0, 63, 200, 130)):
        self.rng = rng = np.random.default_rng(seed)
        self.sizes, self.P, self.window, self.sinks, self.d, self.H, self.grp = [16, 9, 1, 33, 12], P, window, sinks, d, H, grp
        B, N = len(self.sizes), sum(self.sizes) + 4
        self.codec = cg.Codec(cg.BLOCK_UNIFORM, bits, 64)
        self.G = S.haar(1, H, d, g, seed)
        self.shp, self.Gd = S.gauge_dev(self.G)
        self.pool = cg.PagePool(40)
        self.dev = [cg.Cache(self.codec, s, 1, 40, H, P, d) for s in (0, 1)]
        host = [S.random_pool(self.codec, 1, 40, H, P, d, rng) for _ in (0, 1)]
        for c, (codes, side) in zip(self.dev, host):
            c.codes.copy_(torch.from_numpy(codes.reshape(-1)))
            c.side.copy_(torch.from_numpy(side.view(np.uint8).reshape(-1)))
        self.pages = torch.full((B, 8), -1, dtype=torch.int32, device="cuda")
        self.lens, self.add, self.cu = i32([0] * B), i32(list(held)), i32([0] * (B + 1))
        big = torch.zeros(N + 600, dtype=torch.int32, device="cuda")
        cg.kv_page_map(self.lens, self.add, self.pool, self.pages, P, self.cu, self.lens, big, big.clone())
        self.add = i32(self.sizes)
        self.pos0, self.pos, self.slots, self.path = (i32([0] * N) for _ in range(4))
        self.mask = torch.zeros((N, 1), dtype=torch.int64, device="cuda")
        self.kept, self.next, self.held = (i32([0] * B) for _ in range(3))
        self.plan = cg.rope_make(d)
        mk = lambda heads: torch.zeros((1, N, heads, d), dtype=dtype, device="cuda").transpose(1, 2).unsqueeze(1)  # noqa: E731
        self.k, self.v, self.q, self.qo, self.out = mk(H), mk(H), mk(H * grp), mk(H * grp), mk(H * grp)
        self.parent, self.draft, self.target = (i32([0] * N) for _ in range(3))
        self.ws = torch.zeros(max(16, cg.attend_tree_workspace_bytes(self.shp, 1, N, B, H * grp, 8, P)), dtype=torch.uint8, device="cuda")
        self.err = i32([0])
        self.N = N

    def fill(self, seed):
        """Another step's inputs."""
        rng = np.random.default_rng(seed)
        self.trees, self.first, parents = packed(self.sizes, ["near", "forest", "near", "star", "chain"], rng)
        for t in self.trees:
            t[0] = -1
        self.parent.copy_(i32(sum(self.trees, []) + [0] * 4))
        self.hd, self.ht = rng.integers(0, 3, self.N).tolist(), rng.integers(0, 3, self.N).tolist()
        self.draft.copy_(i32(self.hd))
        self.target.copy_(i32(self.ht))
        for t in (self.k, self.v, self.q):
            t.copy_(torch.from_numpy(rng.standard_normal(t.shape)).to(t.dtype))

    def run(self):
        cg.kv_page_map(self.lens, self.add, self.pool, self.pages, self.P, self.cu, self.lens, self.pos0, self.slots, self.err)
        cg.kv_tree_map(self.parent, self.cu, self.lens, self.pos, self.mask, self.err)
        cg.kv_append_rope(0, 1, self.plan, self.k, self.v, self.pos, self.slots, self.Gd, self.shp, self.codec, *self.dev, self.q,
                          self.qo, self.err)
        pt = cg.page_table(self.pages, self.P)
        cg.kv_attend_tree_paged(0, 1, self.qo, self.cu, 33, self.mask, *self.dev, pt, self.Gd, self.shp, self.codec, self.lens,
                                1 / math.sqrt(self.d), self.out, self.pos, self.window, self.sinks, self.ws, self.err)
        cg.kv_tree_accept(self.parent, self.cu, self.draft, self.target, self.path, self.kept, self.next, None, self.err)
        cg.kv_tree_keep(0, 1, self.path, self.kept, self.cu, self.lens, pt, self.codec, *self.dev, self.held, self.err)
        cg.kv_page_trim(self.lens, self.held, self.pool, self.pages, self.P, self.err)

    def state(self):
        torch.cuda.synchronize()
        used = int(self.cu[-1])
        return [t.clone() for t in (self.lens, self.pages, self.pool.count, self.pos, self.mask, self.path, self.kept, self.next,
                                    self.out[:, :, :, :used], self.qo[:, :, :, :used])]


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_a_step_keeps_what_sequential_decoding_would(window, sinks):
    """After three steps, the chunk attention of one more token per row over the pools equals the same over pools that were filled
    with the kept tokens alone, one after the other, by kv_append_rope (as bytes: the pools' rows are equal)."""
    st = Step(window=window, sinks=sinks)
    ref = Step(window=window, sinks=sinks)
    for step in range(3):
        st.fill(step)
        before = st.lens.tolist()
        st.run()
        torch.cuda.synchronize()
        assert int(st.err.item()) == 0
        ways = [T.walk(t, st.hd[a:], st.ht[a:])[0] for t, a in zip(st.trees, st.first)]
        assert st.kept.tolist() == [len(w) for w in ways] and st.lens.tolist() == [h + len(w) for h, w in zip(before, ways)]
        # the kept tokens alone, as chains
        idx = [a + i for w, a in zip(ways, st.first) for i in w]
        N = len(idx)
        pos0, slots = i32([0] * N), i32([0] * N)
        cu = i32([0] * 6)
        cg.kv_page_map(ref.lens, i32([len(w) for w in ways]), ref.pool, ref.pages, 64, cu, ref.lens, pos0, slots, ref.err)
        take = lambda t: t[:, :, :, idx].contiguous()  # noqa: E731
        q = take(st.q)
        cg.kv_append_rope(0, 1, st.plan, take(st.k), take(st.v), pos0, slots, st.Gd, st.shp, st.codec, *ref.dev, q, q, ref.err)
        chain = torch.zeros((N, 1), dtype=torch.int64, device="cuda")
        out = torch.empty_like(q)
        cg.kv_attend_chunk_paged(0, 1, q, cu, 33, *ref.dev, cg.page_table(ref.pages, 64), st.Gd, st.shp, st.codec, ref.lens,
                                 1 / math.sqrt(128), out, window, sinks,
                                 torch.zeros(max(16, cg.attend_chunk_workspace_limit(st.shp, 1, N, 5, 4, 8, 64)), dtype=torch.uint8, device="cuda"),
                                 ref.err)
        torch.cuda.synchronize()
        del chain
        assert ref.lens.tolist() == st.lens.tolist() and int(ref.err.item()) == 0
        assert torch.equal(q, st.qo[:, :, :, idx])
        for b, n in enumerate(st.lens.tolist()):
            for a, r in zip(st.dev, ref.dev):
                for buf, other in ((a.codes, r.codes), (a.side, r.side)):
                    x, y = (t.view(1, 40, 2, 64, -1)[0, p[b, : -(-n // 64)].long()].transpose(1, 2).flatten(0, 1)[before[b]:n]
                            for t, p in ((buf, st.pages), (other, ref.pages)))
                    assert torch.equal(x, y)
        # the same result in bf16, whichever kernel and order of sums: two roundings apart at most, relative to the rows' largest
        got, want = st.out[:, :, :, idx].float(), out.float()
        assert (got - want).norm(dim=-1).max() <= 4 * 2.0 ** -8 * want.norm(dim=-1).max()


def test_a_captured_step():
    """Captured once, replayed with eager work between the replays: every replay gives what the eager step gives."""
    eager, graphed = Step(), Step()
    graphed.fill(0)
    side = torch.cuda.Stream()
    start = [t.clone() for t in (graphed.lens, graphed.pages, graphed.pool.free, graphed.pool.count, *(c.codes for c in graphed.dev), *(c.side for c in graphed.dev))]
    with torch.cuda.stream(side):
        graphed.run()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            graphed.run()
    for t, s in zip((graphed.lens, graphed.pages, graphed.pool.free, graphed.pool.count, *(c.codes for c in graphed.dev), *(c.side for c in graphed.dev)), start):
        t.copy_(s)
    torch.cuda.synchronize()
    for step in range(4):
        eager.fill(10 + step)
        graphed.fill(10 + step)
        eager.run()
        g.replay()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)
    assert int(graphed.err.item()) == 0


def test_two_steps_on_two_streams():
    """Steps of their own buffers at the same time give what they give one after the other."""
    alone, a, b = Step(), Step(), Step(seed=3, held=(1, 64, 128, 5, 77))
    other = Step(seed=3, held=(1, 64, 128, 5, 77))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for st in (alone, a):
        st.fill(1)
    for st in (b, other):
        st.fill(2)
    alone.run()
    other.run()
    torch.cuda.synchronize()
    for _ in range(1):
        with torch.cuda.stream(s1):
            a.run()
        with torch.cuda.stream(s2):
            b.run()
    torch.cuda.synchronize()
    for x, y in zip(alone.state() + other.state(), a.state() + b.state()):
        assert torch.equal(x, y)
