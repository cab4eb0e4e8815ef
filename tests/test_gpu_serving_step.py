"""A serving step's operators where calls follow one another: shared workspaces, pages that run out, precision of
single tokens, long rows whose results do not average away."""
import math

import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

import _serving as S
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


def test_one_workspace_for_calls_of_any_size():
    """A workspace of attend_chunk_workspace_limit bytes for the largest batch serves smaller ones, which split into
    more parts: the results are those of workspaces of their own, and nothing behind it is written."""
    cases = [Case(rows, H=8, grp=4, P=256, seed=k, spare_pages=40 - max(-(-(h + t) // 256) for h, t in rows))
             for k, rows in enumerate(([(8000, 2000), (40, 1)], [(9000, 700)], [(9000, 40), (8000, 1)], [(9500, 1)], [(100, 1), (3, 70)]))]
    N = max(c.N for c in cases)
    limit = cg.attend_chunk_workspace_limit(cases[0].shp, 1, N, 2, 32, 40, 256)
    buf = torch.full((limit + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    sizes = []
    for c in cases:
        need = c.workspace()[1]
        assert need <= limit
        sizes.append(need)
        c.call()
        torch.cuda.synchronize()
        want = c.out.clone()
        c.base.fill_(7.0)
        c.call(buf[:limit])
        torch.cuda.synchronize()
        assert torch.equal(c.out, want) and int(c.err.item()) == 0
        assert (buf[limit:] == 0x5A).all()
    assert max(sizes) > 0 and sizes[0] < max(sizes)


def test_tokens_of_a_row_with_a_negative_length_get_no_slot():
    """Not even those whose position is not negative: what the row's table holds may be another row's page."""
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for N in (12, 3000):                               # in the rows' launch, and in one of its own
        pool = cg.PagePool(8)
        pages = torch.tensor([[3, 4], [5, -1], [6, 7]], dtype=torch.int32, device="cuda")
        cu, lens, pos, slots, err = i32([9] * 4), i32([9] * 3), i32([9] * N), i32([9] * N), i32([0])
        cg.kv_page_map(i32([-3, 2, 2 ** 31 - 3]), i32([6, 2, 4]), pool, pages, 64, cu, lens, pos, slots, err)
        torch.cuda.synchronize()
        assert int(err.item()) & cg.CG_FLAG_POS_RANGE and cu.tolist() == [0, 6, 8, 12]
        assert lens.tolist() == [3, 4, 2 ** 31 - 1] and pages.tolist() == [[3, 4], [5, -1], [6, 7]]
        assert slots.tolist() == [-1] * 6 + [5 * 64 + 2, 5 * 64 + 3] + [-1] * (N - 8)
        assert int(pool.count.item()) == 8


def test_page_map_with_room_for_the_most_tokens():
    """N = 2^31 - 1: every entry of pos and slots is written, those behind the tokens as -1."""
    N, i32 = 2 ** 31 - 1, lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pool, pages = cg.PagePool(4), torch.full((2, 2), -1, dtype=torch.int32, device="cuda")
    pos, slots = (torch.full((N,), 9, dtype=torch.int32, device="cuda") for _ in (0, 1))
    cu, lens, err = i32([9] * 3), i32([9] * 2), i32([0])
    cg.kv_page_map(i32([0, 0]), i32([2, 1]), pool, pages, 64, cu, lens, pos, slots, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and pages.tolist() == [[0, -1], [1, -1]] and int(pool.count.item()) == 2
    assert pos[:3].tolist() == [0, 1, 0] and slots[:3].tolist() == [0, 1, 64]
    assert all(bool((t[3:] == -1).all()) for t in (pos, slots))


@pytest.mark.parametrize("bits,n", [(2, 64), (3, 64), (4, 64), (6, 64), (8, 64), (3, 128), (4, 128), (8, 128), (4, 32)])
@pytest.mark.parametrize("new", [1, 2])
def test_binary32_results_hold_22_bits(bits, n, new):
    """Two positions whose scores of about 60 lie within 3 of each other, one key in channel 5, the other in channel 77, and
    opposite values: o = v tanh(D / 2), D the scores' difference.  A query's two channels are all that counts.

    Bound: with A the larger score and operands of 22 bits (2^-22 of a value at most) the two products of a score are off by
    2^-22 A together (of a code's distance from the middle, the other channel's part included), scale and
    query by two binary32 roundings (2^-23 A), the products' sum, block offset, and their sum by four (2^-22 A): 2.5 2^-22 A
    per score, E = 5 2^-22 A for D.  tanh(D / 2) moves by E / 2 at most; weights, their sum, the division, the values'
    operands and sums: eight roundings of 2^-22 of |v|.  Operands of 16 bits are off by up to 2^-16 A and 2^-18 A at the
    median, far past it in some of the 4 x 24 queries."""
    rows = [(2 - new, new)] * 24
    c = Case(rows, H=1, grp=4, bits=bits, n=n, g=128, dtype=torch.float32, pad=0, spare_pages=0, scale=0.25, seed=bits + n)
    c.G = np.eye(128, dtype=np.float32).reshape(1, 1, 1, 1, 128, 128).repeat(2, axis=1)
    c.shp, c.Gd = S.gauge_dev(c.G)
    top, rng = 2 ** bits - 1, np.random.default_rng(7)
    scale_h = np.float16(120.0 / top)
    q = np.zeros((1, c.N, 4, 128), np.float32)
    x = rng.uniform(1.9, 2.0, (c.N, 4)).astype(np.float32)
    q[0, :, :, 5], q[0, :, :, 77] = x, x * rng.uniform(0.96, 1.04, x.shape).astype(np.float32)
    c.q = torch.from_numpy(q).permute(c.perm)
    c.qd = torch.from_numpy(q).cuda().permute(c.perm).unsqueeze(1)
    codes = [np.zeros((1, c.kc.B, 1, 64, 128), np.uint8) for _ in (0, 1)]
    codes[0][..., 0, 5] = codes[0][..., 1, 77] = top
    codes[1][..., 0, :] = rng.integers(0, 2, 128) * top
    codes[1][..., 1, :] = top - codes[1][..., 0, :]
    weights = 1 << np.arange(bits)
    for s in (0, 1):
        b = ((codes[s][..., None] & weights) > 0).astype(np.uint8).reshape(1, c.kc.B, 1, 64, -1)
        c.pools[s][0] = np.packbits(b, axis=-1, bitorder="little")
        c.pools[s][1][..., 0] = 0.0 if s == 0 else np.float16(-0.5)
        c.pools[s][1][..., 1] = scale_h if s == 0 else np.float16(1.0 / 2 ** bits)
    c.upload()
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == 0
    zk, zv = (S.pool_values(c.codec, *p)[0, 0, 0] for p in c.pools)
    assert zk[0, 5] == zk[1, 77] == top * float(scale_h) and np.count_nonzero(zk[:2]) == 2
    qd = torch.from_numpy(q[0]).double()[new - 1::new]                     # a row's last token sees both
    got = c.out[0, 0].double().cpu().transpose(0, 1)[new - 1::new]
    sc = c.scale * qd @ torch.from_numpy(zk[:2]).T
    want = torch.softmax(sc, -1) @ torch.from_numpy(zv[:2])
    A, v = sc.max(-1).values, float(np.abs(zv[:2]).max())
    assert 50 < float(A.min()) and float((sc[..., 0] - sc[..., 1]).abs().max()) < 3
    err = (got - want).abs().amax(-1)
    lim = (2.5 * 2.0 ** -22 * A + 8 * 2.0 ** -22) * v
    assert (err <= lim).all(), float((err / lim).max())


class Plain(Case):
    """A case whose gauge is the identity, keys, values and queries set channel by channel."""

    def set(self, q=None, k=None, v=None):
        """q [N][Hq][d]; k, v [pages][64][d] of the error-free pools' (one layer and head)."""
        d = self.d
        self.G = np.eye(d, dtype=np.float32).reshape(1, 1, 1, 1, d, d).repeat(2, axis=1)
        self.shp, self.Gd = S.gauge_dev(self.G)
        if q is not None:
            self.q = torch.from_numpy(q.astype(np.float32))[None].to(self.q.dtype).permute(self.perm)
            self.qd = self.q.permute(self.perm).contiguous().cuda().permute(self.perm).unsqueeze(1)
        for s, x in enumerate((k, v)):
            if x is not None:
                self.pools[s][0] = np.ascontiguousarray(x[None, :, None].astype(np.float32)).view(np.uint8)
        self.upload()
        return self

    def results(self):
        """(got, zk, zv) of the one row: outputs [Hq][new][d], positions' keys and values, in binary64."""
        self.call()
        torch.cuda.synchronize()
        assert int(self.err.item()) == 0
        n = self.held[0]
        zk, zv = (torch.from_numpy(S.pool_values(self.codec, *p)[0, self.table[0][: -(-n // 64)], 0].reshape(-1, self.d)[:n])
                  for p in self.pools)
        return self.out[0, 0].double().cpu()[:, : self.rows[0][1]], zk, zv


@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [1, 3])
def test_error_free_values_of_small_channels(d, dtype, new):
    """Channels from 1 down to 1e-8 beside each other, growing and falling over the positions, equal weights: every
    channel's mean within the roundings of its own values.

    Operands: u = 2^-11, or 2^-22 and 2^-40 of the largest value (two planes); the sums over T positions T 2^-24, their
    planes for the gauge 2^-15 (2^-22), the rest 2^-22, relative to the mean of |v|; one rounding of the type."""
    T, rng = 300, np.random.default_rng(d)
    c = Plain([(T - new, new)], H=1, grp=2, d=d, g=d, backend=cg.PASSTHROUGH, dtype=dtype, scale=0.5)
    pages = c.kc.B
    v = rng.standard_normal((pages, 64, d)) * 10.0 ** -rng.uniform(0, 8, d)
    v *= 10.0 ** np.where(np.arange(pages) % 2, 1.5, -1.5)[:, None, None]         # a step of small values after large ones
    k = rng.standard_normal((pages, 64, d))
    c.set(np.zeros((c.N, 2, d)), k, v)
    got, _, zv = c.results()
    bf = dtype == torch.bfloat16
    for i in range(new):
        x = zv[: T - new + 1 + i]
        want, a = x.mean(0), x.abs().mean(0)
        lim = a * ((2.0 ** -11 if bf else 2.0 ** -22) + T * 2.0 ** -24 + (2.0 ** -15 if bf else 2.0 ** -22) + 2.0 ** -22) \
            + (0.0 if bf else 2.0 ** -40 * float(x.abs().max())) + (2.0 ** -8 if bf else 2.0 ** -24) * want.abs()
        assert ((got[:, i] - want).abs() <= lim).all(), float(((got[:, i] - want).abs() / lim).max())


def _weights_bound(got, q, zk, zv, scale, unit, floor, planes, step):
    """got [Hq][new][d] against softmax over all positions a token sees; a score is off by A (2 unit + 2^-21) plus `floor`
    (of the queries' sum) where A = |scale| sum |q k|, a weight by a factor within exp(+-2 E) and 2 unit, the rest as
    above; all of it relative to the largest |v|."""
    n, new = zk.shape[0], got.shape[1]
    for j in range(got.shape[0]):
        for i in range(new):
            m = n - new + 1 + i
            s = scale * zk[:m] @ q[j, i]
            want = torch.softmax(s, 0) @ zv[:m]
            E = abs(scale) * (float((zk[:m].abs() @ q[j, i].abs()).max()) * (2 * unit + 2.0 ** -21) + floor * float(q[j, i].abs().sum()))
            lim = (math.expm1(2 * E) + 2 * unit + n * 2.0 ** -24 + planes) * float(zv.abs().max()) + step * want.abs()
            assert E < 0.05 and ((got[j, i] - want).abs() <= lim).all(), (E, float(((got[j, i] - want).abs() / lim).max()))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [1, 3])
def test_error_free_keys_of_small_channels(d, dtype, new):
    """What tells the positions apart lies in a channel of 1e-6, where the query is large, beside channels of 1 where it is
    nought."""
    T, rng = 200, np.random.default_rng(d + 1)
    c = Plain([(T - new, new)], H=1, grp=2, d=d, g=d, backend=cg.PASSTHROUGH, dtype=dtype, scale=1.0)
    k = rng.standard_normal((c.kc.B, 64, d))
    k[..., 7] = 1e-6 * rng.standard_normal(k.shape[:2])
    q = np.zeros((c.N, 2, d))
    q[..., 7] = rng.uniform(1e6, 2e6, q.shape[:2])
    c.set(q, k, rng.standard_normal((c.kc.B, 64, d)))
    got, zk, zv = c.results()
    bf = dtype == torch.bfloat16
    _weights_bound(got, c.q[0, :, :new].double(), zk, zv, 1.0, 2.0 ** -11 if bf else 2.0 ** -22, 0.0 if bf else 2.0 ** -40 * float(zk.abs().max()),
                   2.0 ** -15 if bf else 2.0 ** -22, 2.0 ** -8 if bf else 2.0 ** -24)


@pytest.mark.parametrize("bits,n,d", [(4, 32, 128), (4, 16, 128), (4, 64, 256), (8, 32, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_of_small_channels(bits, n, d, dtype):
    """What tells the positions apart lies in a block of large keys, where the query is 2e-6 of its largest channel; there
    the keys are nought.  Queries keep their bits down to 2^-29 (two planes: 2^-18, and 2^-40 beyond) of the largest."""
    T, new, rng = 200, 3, np.random.default_rng(d + n)
    c = Plain([(T - new, new)], H=1, grp=2, d=d, g=d, bits=bits, n=n, dtype=dtype, scale=40.0)
    side = c.pools[0][1]
    side[...] = 0.0
    side[..., 1, 1] = np.float16(60000.0 / (2 ** bits - 1))
    q = np.zeros((c.N, 2, d))
    q[..., 0] = 1.0
    q[..., n: 2 * n] = 2e-6 / n * rng.uniform(0.5, 1.0, q[..., n: 2 * n].shape)
    c.set(q)
    got, zk, zv = c.results()
    bf = dtype == torch.bfloat16
    floor = 0.0 if bf else 2.0 ** -40 * n * float(zk.max())       # of the largest query, 1
    _weights_bound(got, c.q[0, :, :new].double(), zk, zv, 40.0, 2.0 ** -11 if bf else 2.0 ** -22, floor, 2.0 ** -15 if bf else 2.0 ** -22,
                   2.0 ** -8 if bf else 2.0 ** -24)


def test_a_step_that_ran_out_of_pages_is_begun_again():
    """Rows with a hole are given back whole and begun again after another row is done: every page stands in one place
    throughout, the rows' slots are those of their pages, and rows that had enough keep theirs."""
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    P, total, B, maxp = 64, 9, 4, 6
    pool = cg.PagePool(total)
    pages = torch.full((B, maxp), -1, dtype=torch.int32, device="cuda")
    lens, cu, pos, slots, err = i32([0] * B), i32([0] * (B + 1)), i32([0] * 400), i32([0] * 400), i32([0])

    def step(add):
        err.zero_()
        cg.kv_page_map(lens, i32(add), pool, pages, P, cu, lens, pos, slots, err)
        torch.cuda.synchronize()
        n = int(pool.count.item())
        free, held = pool.free.tolist()[:n], [p for p in pages.flatten().tolist() if p >= 0]
        assert sorted(free + held) == list(range(total))
        table, first = pages.tolist(), cu.tolist()
        for b in range(B):
            for i in range(first[b], first[b + 1]):
                t = int(lens[b]) - (first[b + 1] - i)
                pg = table[b][t // P]
                assert int(pos[i]) == t and int(slots[i]) == (pg * P + t % P if pg >= 0 else -1)
        return int(err.item()), n, table

    assert step([100, 60, 130, 0])[:2] == (0, 3)
    flag, left, table = step([1, 70, 1, 200])                  # row 1 takes two pages, row 3 gets one of four
    assert flag == cg.CG_FLAG_POOL_EMPTY | cg.CG_FLAG_POS_RANGE and left == 0 and table[3].count(-1) == maxp - 1
    assert lens.tolist() == [101, 130, 131, 200]
    kept = table[0], table[2]
    cg.kv_page_release(lens, i32([0, 1, 0, 1]), pool, pages, P, err)   # row 1 is done, row 3 has holes
    torch.cuda.synchronize()
    assert int(pool.count.item()) == 4 and lens.tolist() == [101, 0, 131, 0]
    flag, left, table = step([1, 0, 1, 200])
    assert flag == 0 and left == 0 and lens.tolist() == [102, 0, 132, 200]
    assert (table[0], table[2]) == kept and table[3][:4].count(-1) == 0


LONG = {
    "b2": dict(bits=2), "b3": dict(bits=3), "b4": dict(bits=4), "b6": dict(bits=6), "b8": dict(bits=8),
    "n32": dict(n=32, bits=3), "n16": dict(n=16), "n128": dict(n=128, bits=6), "error_free": dict(backend=cg.PASSTHROUGH),
    "d64": dict(d=64, n=32), "d64_b8": dict(d=64, n=64, bits=8), "d80": dict(d=80, n=80), "d256": dict(d=256, n=64),
    "f32": dict(dtype=torch.float32), "f32_b8_n128": dict(dtype=torch.float32, bits=8, n=128), "f32_n16": dict(dtype=torch.float32, n=16),
    "f32_d64": dict(dtype=torch.float32, d=64, n=32, bits=6), "f32_d256": dict(dtype=torch.float32, d=256, n=128),
    "f32_error_free": dict(dtype=torch.float32, backend=cg.PASSTHROUGH),
}


@pytest.mark.parametrize("rows", [[(6000, 3)], [(5003, 70), (1, 1)], [(6001, 1)], [(4000, 1), (3000, 2), (63, 1)]], ids=lambda r: "+".join(f"{h}_{t}" for h, t in r))
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 300)])
@pytest.mark.parametrize("name", list(LONG))
def test_every_position_of_a_long_row_counts(name, window, sinks, rows):
    """Channel c of a value is 1 at the c-th stretch of its row's positions and 0 elsewhere (identity gauge), so an output
    channel is the weight of its stretch, about 1 / d: sums of positive terms, which do not average away.  A step
    left out, taken twice or read from another page moves a channel by most of itself.

    Bound, relative to the channel: scores of A at most are off by E = A (2 u + d 2^-24), u = 2^-11 or 2^-22 the rounding of an
    operand; all weights by a factor within exp(+-2 E); weights and values by u each, sums over T positions by T 2^-24,
    their planes for the gauge 2^-15 (2^-22), one rounding of the type.  Hidden stretches are nought in chunks.  Single tokens of
    128 channels in blocks of 64 or 128 form a value from its block's offset and the code's distance from it: of each step of 32
    positions one product's and eight offsets' additions round by 2^-24 of a partial sum, at most 2 (a range of 1, the weights'
    sum 1): 9 n / 32 2 2^-24 whatever the channel."""
    kw = dict(dict(d=128, n=64, bits=4, dtype=torch.bfloat16), **LONG[name])
    d = kw["d"]
    c = Plain(rows, H=1, grp=4, g=d, window=window, sinks=sinks, scale=0.08, seed=len(name), **kw)
    rng = np.random.default_rng(11)
    stretch = np.full((c.kc.B, 64), -1)
    for b, n in enumerate(c.held):
        for i in range(-(-n // 64)):
            t = np.arange(64 * i, min(n, 64 * i + 64))
            stretch[c.table[b, i], : len(t)] = t * d // n
    one = (stretch[..., None] == np.arange(d)).astype(np.float32)                # [pages][64][d]
    if c.codec.backend == cg.PASSTHROUGH:
        c.set(None, rng.uniform(-1, 1, one.shape), one)
    else:
        top = 2 ** c.codec.bits - 1
        bit = (top * one[..., None].astype(np.uint8) >> np.arange(c.codec.bits)) & 1
        c.pools[1][0] = np.packbits(bit.reshape(1, c.kc.B, 1, 64, -1), axis=-1, bitorder="little")
        for s, (mn, sc) in enumerate(((-1.0, 2.0 / top), (0.0, 1.0 / top))):
            c.pools[s][1][..., 0], c.pools[s][1][..., 1] = np.float16(mn), np.float16(sc)
        c.set()
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == 0
    got = c.out[0, 0].double().cpu()
    zk, zv = (S.pool_values(c.codec, *p) for p in c.pools)
    bf = c.out.dtype == torch.bfloat16
    u, planes, step = (2.0 ** -11, 2.0 ** -15, 2.0 ** -8) if bf else (2.0 ** -22, 2.0 ** -22, 2.0 ** -24)
    offsets = d == 128 and c.codec.backend == cg.BLOCK_UNIFORM and c.codec.block_c >= 64
    for b, (held, new) in enumerate(rows):
        n = held + new
        floor = 9 * n / 16 * 2.0 ** -24 if offsets and new == 1 else 0.0
        K, V = (torch.from_numpy(z[0, c.table[b][: -(-n // 64)], 0].reshape(-1, d)[:n]) for z in (zk, zv))
        for i in sorted({0, new // 2, new - 1}):
            p = held + i
            seen = S.visible(p, n, window, sinks)
            q = c.q[0, :, int(c.first[b]) + i].double()
            s = (c.scale * q @ K.T).masked_fill(~seen, -math.inf)
            w = torch.softmax(s, -1)
            want = w @ V
            E = abs(c.scale) * float((q.abs() @ K[seen].abs().T).max()) * (2 * u + d * 2.0 ** -24)
            lim = want * (math.expm1(2 * E) + 2 * u + n * 2.0 ** -24 + planes + step) + floor
            err = (got[:, int(c.first[b]) + i] - want).abs()
            assert (err <= lim).all(), (b, i, float((err / lim.clamp(min=1e-30)).max()))
            if n >= 1000:
                # without the first, a middle or the last step that is seen, the same comparison fails
                steps = torch.unique(torch.nonzero(seen)[:, 0] // 64)
                for gone in (steps[0], steps[len(steps) // 2], steps[-2]):
                    x = w.masked_fill((torch.arange(n) // 64 == gone)[None], 0.0)
                    x = x / x.sum(-1, keepdim=True)
                    assert ((x @ V - want).abs() > 3 * lim).any(-1).all()


def test_attend_refuses_a_table_of_other_rows():
    c = Case([(70, 3), (5, 1)], H=1)
    ws = c.workspace()[0]
    for pages in (c.pages[:1], torch.cat((c.pages, c.pages))):
        with pytest.raises(ValueError):
            cg.kv_attend_chunk_paged(0, 1, c.qd, c.cu, c.max_q, c.kc, c.vc, cg.page_table(pages, c.P), c.Gd, c.shp, c.codec, c.lens,
                                     c.scale, c.out, workspace=ws)
    torch.cuda.synchronize()
    assert (c.out == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("what", ["k+", "k-", "v"])
def test_infinities_act_as_in_exp_and_products(what, new, dtype):
    """An infinite key or value at position 130 of an error-free pool, identity gauge, window of 40: a score of +inf makes
    the result NaN, one of -inf weighs nothing, an infinite value its channel infinite or NaN; who does not see it is
    untouched.  The bounds of the others: _weights_bound's, scores of 6 at most."""
    c = Plain([(180 - new, new)], H=1, grp=2, d=64, g=64, backend=cg.PASSTHROUGH, dtype=dtype, scale=0.2, window=40)
    rng = np.random.default_rng(3)
    k, v = (rng.uniform(-1, 1, (c.kc.B, 64, 64)) for _ in (0, 1))
    q = rng.uniform(0.2, 1.0, (c.N, 2, 64))
    (v if what == "v" else k)[c.table[0, 2], 2, 5] = -np.inf if what == "k-" else np.inf
    c.set(q, k, v)
    got, zk, zv = c.results()
    q = c.q[0, :, :new].double()
    bf = dtype == torch.bfloat16
    u, planes, step = (2.0 ** -11, 2.0 ** -15, 2.0 ** -8) if bf else (2.0 ** -22, 2.0 ** -22, 2.0 ** -24)
    for i in range(new):
        p = 180 - new + i
        t = S.visible(p, 180, 40, 0)
        for j in range(2):
            if t[130] and what == "k+":
                assert torch.isnan(got[j, i]).all()
                continue
            if t[130] and what == "v":
                assert not torch.isfinite(got[j, i, 5])
                continue
            w = t.clone()
            if what == "k-":
                w[130] = False
            K, V = zk[w], zv[w]
            want = torch.softmax(c.scale * K @ q[j, i], 0) @ V
            E = c.scale * float((K.abs() @ q[j, i].abs()).max()) * (2 * u + 2.0 ** -21)
            lim = math.expm1(2 * E) + 2 * u + 40 * 2.0 ** -24 + planes + step * want.abs()
            assert ((got[j, i] - want).abs() <= lim).all()


@pytest.mark.parametrize("d,g,bits,n", [(64, 64, 4, 32), (128, 128, 4, 64)])
def test_slots_of_more_tokens_than_one_launch_holds(d, g, bits, n):
    """2^19 + 77 tokens: the same bytes as in two calls (128 channels: one launch of the matrix-core encoder, whose bytes do
    not depend on the tokens beside)."""
    N, P = 2 ** 19 + 77, 256
    pages = N // P + 2
    codec = cg.Codec(cg.BLOCK_UNIFORM, bits, n)
    shp, Gd = S.gauge_dev(S.haar(1, 1, d, g, 2))
    torch.manual_seed(d)
    x = [torch.randn((1, 1, 1, N, d), device="cuda").to(torch.bfloat16) for _ in (0, 1)]
    slots = torch.randperm(pages * P, device="cuda")[:N].to(torch.int32)
    slots[::1001] = -1
    one, two = ([cg.Cache(codec, s, 1, pages, 1, P, d) for s in (0, 1)] for _ in (0, 1))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    cg.kv_append_slots(0, 1, *x, slots, Gd, shp, codec, *one, err)
    for a, b in ((0, 2 ** 18), (2 ** 18, N)):
        cg.kv_append_slots(0, 1, *(t[:, :, :, a:b] for t in x), slots[a:b], Gd, shp, codec, *two, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    for a, b in zip(one, two):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.side, b.side)
        dec = torch.empty((1, pages, 1, P, d), dtype=torch.float32, device="cuda")
        cg.kv_decode(0 if a is one[0] else 1, a, Gd, shp, codec, 0, dec)
        live = torch.nonzero(slots >= 0)[:, 0]
        back = dec.view(-1, d)[slots[live].long()] - x[0 if a is one[0] else 1].view(-1, d)[live].float()
        # half a step of a range of at most 12 deviations, in the 2-norm
        assert float(back.norm(dim=-1).max()) <= 12 / (2 ** bits - 1) / 2 * math.sqrt(d)
