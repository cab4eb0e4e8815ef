"""Attention of packed new tokens over page pools (kv_attend_chunk_paged) against softmax attention in binary64.

Pools hold random codes and ranges written here by the documented byte layout; what lies behind a row's last
position is garbage whose ranges are NaN and infinities, so a position that leaks into a result shows.  The error of
a token is bounded in the 2-norm by the roundings that the kernel makes (tests/_serving.py: attend_ref)."""
import math

import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

import _serving as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


class Case:
    """A batch over random pools: rows (positions held before, new tokens), packed one after the other."""

    def __init__(self, rows, H=2, grp=2, d=128, g=32, bits=4, n=64, P=64, L=1, backend=cg.BLOCK_UNIFORM, pad=3, seed=1,
                 spread=1.0, dtype=torch.bfloat16, out_dtype=None, window=0, sinks=0, scale=None, spare_pages=1,
                 tokens_first=True):
        rng = np.random.default_rng(seed)
        self.codec = cg.Codec(backend, bits, n)
        self.rows, self.P, self.d, self.window, self.sinks = rows, P, d, window, sinks
        self.scale = 1.0 / math.sqrt(d) if scale is None else scale
        self.G = S.haar(L, H, d, g, seed + 1)
        self.shp, self.Gd = S.gauge_dev(self.G)
        need = [-(-(h + t) // P) for h, t in rows]
        maxp = max(1, max(need)) + spare_pages
        pages = sum(need) + 2
        perm = rng.permutation(pages).astype(np.int32)
        self.table = np.full((len(rows), maxp), -1, np.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = perm[at: at + k]
            at += k
        self.pools = [list(S.random_pool(self.codec, L, pages, H, P, d, rng, spread)) for _ in (0, 1)]
        for codes, side in self.pools:
            for b, (h, t) in enumerate(rows):
                last = (h + t) % P
                if last == 0:
                    continue
                pg = self.table[b, need[b] - 1]
                if side is None:
                    codes.view(np.float32)[:, pg, :, last:] = np.nan
                else:
                    side[:, pg, :, last:, :, 0] = np.float16("nan")
                    side[:, pg, :, last:, :, 1] = np.float16("inf")
        N = self.N = sum(t for _, t in rows) + pad
        cu = np.cumsum([0] + [t for _, t in rows]).astype(np.int32)
        self.held = [h + t for h, t in rows]
        self.first = cu
        self.Hq = H * grp
        # projections as a model lays them out, [L][N][heads][d], or heads first
        q = torch.from_numpy(rng.standard_normal((L, N, self.Hq, d) if tokens_first else (L, self.Hq, N, d))).to(dtype)
        self.perm = (0, 2, 1, 3) if tokens_first else (0, 1, 2, 3)
        self.q = q.permute(self.perm)                                   # [L][Hq][N][d] on the host
        self.qd = q.cuda().permute(self.perm).unsqueeze(1)
        self.base = torch.full(q.shape, 7.0, dtype=out_dtype or dtype, device="cuda")
        self.out = self.base.permute(self.perm).unsqueeze(1)
        self.cu = torch.from_numpy(cu).cuda()
        self.lens = torch.tensor(self.held, dtype=torch.int32, device="cuda")
        self.pages = torch.from_numpy(self.table).cuda()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.max_q = max(1, max(t for _, t in rows))
        self.upload()

    def upload(self):
        self.kc, self.vc = (S.pool_dev(self.codec, s, *self.pools[s]) for s in (0, 1))

    def workspace(self, max_q=None):
        n = cg.attend_chunk_workspace_bytes(self.shp, self.shp.L, self.N, len(self.rows), max_q or self.max_q, self.Hq,
                                            self.table.shape[1], self.P, self.window, self.sinks)
        return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda"), n

    def call(self, ws=None, max_q=None, stream=None):
        ws = self.workspace(max_q)[0] if ws is None else ws
        cg.kv_attend_chunk_paged(0, self.shp.L, self.qd, self.cu, max_q or self.max_q, self.kc, self.vc,
                                 cg.page_table(self.pages, self.P), self.Gd, self.shp, self.codec, self.lens, self.scale,
                                 self.out, self.window, self.sinks, ws, self.err, stream)
        return ws

    def ref(self):
        unit = 2.0 ** -11 if self.out.dtype == torch.bfloat16 else 2.0 ** -22
        rows = [(int(self.first[b]), t, self.held[b]) for b, (_, t) in enumerate(self.rows)]
        return S.attend_ref(self.q.double(), self.G, *(S.pool_values(self.codec, *p) for p in self.pools), self.table, rows,
                            self.P, self.scale, self.window, self.sinks, unit)

    def check(self, flag=0):
        torch.cuda.synchronize()
        assert int(self.err.item()) == flag
        got = self.out[:, 0].double().cpu()
        want, bound = self.ref()
        used = int(self.first[-1])
        assert (got[:, :, used:] == 7.0).all(), "rows behind the last sequence were written"
        step = 2.0 ** -8 if self.out.dtype == torch.bfloat16 else 2.0 ** -24
        err = (got - want)[:, :, :used].norm(dim=-1)
        lim = (bound + step * want.norm(dim=-1))[:, :, :used]
        assert torch.isfinite(got).all()
        assert (err <= lim).all(), (float((err / lim).max()), [int(v) for v in np.unravel_index(int((err / lim).argmax()), err.shape)])


RAGGED = [(0, 1), (0, 70), (130, 0), (63, 1), (64, 33), (200, 129), (1, 5)]

ONES = [(700, 1), (0, 1), (64, 1), (130, 0), (63, 1), (131, 1)]

CASES = {
    "b4": dict(rows=RAGGED),
    "b2": dict(rows=RAGGED, bits=2),
    "b3": dict(rows=RAGGED, bits=3),
    "b6": dict(rows=RAGGED, bits=6, g=128),
    "b8": dict(rows=RAGGED, bits=8, g=64),
    "n32": dict(rows=RAGGED, n=32, H=1),
    "n16": dict(rows=RAGGED, n=16, H=1),
    "n8": dict(rows=RAGGED, n=8, H=1, g=8),
    "n4_b8": dict(rows=[(5, 3), (70, 20)], n=4, bits=8, H=1, g=4),
    "pass": dict(rows=RAGGED, backend=cg.PASSTHROUGH, H=1),
    "layers_p128": dict(rows=[(300, 40), (129, 3)], L=2, P=128, grp=4, g=128),
    "p192": dict(rows=[(300, 40), (191, 3)], P=192, grp=1),
    "grp3": dict(rows=[(10, 50), (100, 9)], grp=3),
    "grp5": dict(rows=[(10, 50), (100, 9)], grp=5, H=1),
    "grp40": dict(rows=[(10, 6), (100, 9)], grp=40, H=1),
    "grp130": dict(rows=[(10, 2), (100, 3)], grp=130, H=1),
    "heads_first": dict(rows=RAGGED, tokens_first=False),
    "d64": dict(rows=RAGGED, d=64, g=64, n=32),
    "d32": dict(rows=RAGGED, d=32, g=16, n=32, H=1),
    "d8": dict(rows=[(0, 9), (70, 3)], d=8, g=8, n=8, H=1),
    "d80_g80": dict(rows=[(0, 9), (70, 33)], d=80, g=80, n=80, H=1),
    "d80_g5": dict(rows=[(0, 9), (70, 33)], d=80, g=5, n=16, H=1),
    "d80_g20": dict(rows=[(0, 9), (70, 33)], d=80, g=20, n=80, H=1),
    "d40_g4": dict(rows=[(0, 9), (70, 33)], d=40, g=4, n=8, H=1),
    "d96": dict(rows=[(0, 9), (70, 33)], d=96, g=96, n=32, H=1),
    "d192": dict(rows=[(0, 9), (70, 33)], d=192, g=64, n=64, H=1),
    "d256": dict(rows=[(0, 9), (70, 33)], d=256, g=128, n=128, bits=8, H=1),
    "f32": dict(rows=RAGGED, dtype=torch.float32),
    "f32_b3": dict(rows=RAGGED, dtype=torch.float32, bits=3, g=128, H=1),
    "f32_pass": dict(rows=RAGGED, dtype=torch.float32, backend=cg.PASSTHROUGH, H=1),
    "f32_d64": dict(rows=RAGGED, dtype=torch.float32, d=64, g=16, n=32),
    "f32_d80": dict(rows=[(0, 9), (70, 33)], dtype=torch.float32, d=80, g=80, n=80, H=1),
    "f32_d256": dict(rows=[(0, 9), (70, 33)], dtype=torch.float32, d=256, g=256, n=64, H=1),
    "bf16_in_f32_out": dict(rows=[(0, 9), (70, 33)], out_dtype=torch.float32),
    "f32_in_bf16_out": dict(rows=[(0, 9), (70, 33)], dtype=torch.float32, out_dtype=torch.bfloat16),
    "window": dict(rows=RAGGED, window=50, sinks=4),
    "window_1": dict(rows=[(0, 70), (200, 5)], window=1, sinks=0),
    "window_1_sink": dict(rows=[(0, 70), (200, 5)], window=1, sinks=1),
    "window_long_sinks": dict(rows=[(0, 70), (500, 40)], window=64, sinks=130),
    "window_past_row": dict(rows=[(0, 70), (200, 40)], window=1000, sinks=4),
    "window_f32": dict(rows=[(0, 70), (500, 40)], window=100, sinks=70, dtype=torch.float32, H=1),
    "singles": dict(rows=[(700, 1), (0, 1), (64, 1), (63, 1), (131, 1)], grp=4),
    "singles_window": dict(rows=[(700, 1), (0, 1), (64, 1), (63, 1), (131, 1)], grp=4, window=100, sinks=5),
    "singles_b2": dict(rows=ONES, bits=2, grp=4),
    "singles_b3_window": dict(rows=ONES, bits=3, n=32, grp=3, window=70, sinks=66),
    "singles_b6": dict(rows=ONES, bits=6, g=128, grp=1),
    "singles_b8_window_1": dict(rows=ONES, bits=8, g=64, window=1, grp=9, H=1),
    "singles_n128": dict(rows=ONES, n=128, g=128, grp=4, window=200, sinks=1),
    "singles_n32_window": dict(rows=ONES, n=32, grp=4, window=200, sinks=1),
    "singles_n16": dict(rows=ONES, n=16, bits=6, H=1),
    "singles_pass": dict(rows=ONES, backend=cg.PASSTHROUGH, H=1, window=90, sinks=3),
    "singles_f32": dict(rows=ONES, dtype=torch.float32, window=90, sinks=3, grp=4),
    "singles_f32_n128": dict(rows=ONES, dtype=torch.float32, n=128, bits=3),
    "singles_d64": dict(rows=ONES, d=64, g=64, n=32, window=90, sinks=3),
    "singles_d80": dict(rows=ONES, d=80, g=80, n=80, H=1, window=90, sinks=3),
    "singles_d256": dict(rows=ONES, d=256, g=128, n=128, bits=8, H=1),
    "singles_grp40": dict(rows=ONES, grp=40, H=1),
    "singles_layers_p128": dict(rows=ONES, L=2, P=128, grp=4, g=128, window=300, sinks=5),
    "singles_long": dict(rows=[(9000, 1), (40, 1), (0, 0), (5000, 1)], grp=4, H=1),
    "singles_long_window": dict(rows=[(9000, 1), (40, 1), (0, 0), (5000, 1)], grp=4, H=1, window=2500, sinks=300),
    "singles_heads_first": dict(rows=ONES, tokens_first=False, grp=4),
    "mixed_window": dict(rows=[(700, 1), (40, 90), (0, 1), (300, 33), (64, 1)], grp=4, window=100, sinks=70),
    "mixed_window_f32": dict(rows=[(700, 1), (40, 90), (0, 1), (300, 3)], grp=2, H=1, window=100, sinks=70, dtype=torch.float32),
    "mixed_n128": dict(rows=[(700, 1), (40, 90), (0, 1), (300, 33), (64, 1)], n=128, window=1000),
    "window_largest": dict(rows=[(0, 70), (200, 40), (90, 1)], window=2 ** 31 - 1, sinks=0),
    "window_and_sinks_largest": dict(rows=[(0, 70), (200, 40), (90, 1)], window=2 ** 31 - 1, sinks=2 ** 31 - 1),
    "sinks_largest": dict(rows=[(0, 70), (200, 40), (90, 1)], window=3, sinks=2 ** 31 - 1),
    "many_rows": dict(rows=[(7 * i % 190, 1 + (i % 5 == 0) * (i % 40)) for i in range(130)], H=1),
    "single_long_split": dict(rows=[(6000, 1)], grp=8, H=1),
    "few_long_split": dict(rows=[(5000, 3), (100, 7)], grp=4, H=1, g=128),
    "split_f32": dict(rows=[(3000, 5)], grp=2, H=1, dtype=torch.float32),
    "negative_scale": dict(rows=[(0, 9), (70, 33)], scale=-0.1),
    "zero_scale": dict(rows=[(0, 9), (70, 33)], scale=0.0),
    "large_scores": dict(rows=[(0, 9), (300, 33)], scale=0.5, H=1),
    "tiny_values": dict(rows=[(0, 9), (70, 33)], spread=2.0 ** -11, scale=100.0, H=1, bits=8),
    "pass_tiny_values": dict(rows=[(0, 9), (70, 33)], spread=1e-6, backend=cg.PASSTHROUGH, H=1),
    "pass_huge_values": dict(rows=[(0, 9), (70, 33)], spread=1e6, scale=1e-7, backend=cg.PASSTHROUGH, H=1),
    "huge_values": dict(rows=[(0, 9), (70, 33)], spread=30000.0, scale=1e-5, bits=2, H=1),
}


@pytest.mark.parametrize("name", list(CASES))
def test_chunk_matches_softmax(name):
    c = Case(**CASES[name])
    c.call()
    c.check()


def test_larger_max_q_changes_only_the_plan():
    c = Case(RAGGED)
    c.call(max_q=1000)
    c.check()


def test_wide_ranges_go_past_binary16():
    """A block whose top is beyond 65504 (its side information is finite) and one that is only just inside."""
    c = Case([(100, 40)], H=1, bits=8, scale=2e-7)
    for codes, side in c.pools:
        pg = c.table[0, 0]
        side[:, pg, :, 10, 0] = (-60000.0, 1000.0)
        side[:, pg, :, 11, 1] = (-65504.0, 513.0)
    c.upload()
    c.call()
    c.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("what", ["k", "v"])
def test_non_finite_positions_reach_only_who_sees_them(what, dtype):
    """A NaN range at position 120: tokens before it and those whose window has passed it are exact, the others
    are NaN; an infinity at a sink would reach all."""
    c = Case([(100, 80)], H=1, window=30, sinks=2, dtype=dtype)
    codes, side = c.pools[0 if what == "k" else 1]
    good = side.copy()
    side[:, c.table[0, 120 // 64], :, 120 % 64, 0, 0] = np.float16("nan")
    c.upload()
    c.call()
    torch.cuda.synchronize()
    got = c.out[0, 0].double().cpu()
    side[...] = good
    want, bound = c.ref()
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for i in range(80):
        sees = 120 <= 100 + i < 150
        if sees:
            assert torch.isnan(got[:, i]).any(-1).all(), i
        else:
            err = (got[:, i] - want[0, :, i]).norm(dim=-1)
            assert (err <= bound[0, :, i] + step * want[0, :, i].norm(dim=-1)).all(), i


@pytest.mark.parametrize("kw", [dict(), dict(n=128), dict(d=80, g=80, n=80), dict(dtype=torch.float32)], ids=["b4", "n128", "d80", "f32"])
@pytest.mark.parametrize("what", ["k", "v"])
def test_non_finite_positions_of_single_tokens(what, kw):
    """Behind the window and past the sinks a NaN range is not seen; one inside the window or at a sink is."""
    c = Case([(200, 1), (200, 1), (200, 1)], H=1, window=30, sinks=2, **kw)
    codes, side = c.pools[0 if what == "k" else 1]
    good = side.copy()
    for b, at in enumerate((120, 185, 1)):
        side[:, c.table[b, at // 64], :, at % 64, 0, 0] = np.float16("nan")
    c.upload()
    c.call()
    torch.cuda.synchronize()
    got = c.out[0, 0].double().cpu()
    side[...] = good
    want, bound = c.ref()
    step = 2.0 ** -8 if c.out.dtype == torch.bfloat16 else 2.0 ** -24
    err = (got[:, 0] - want[0, :, 0]).norm(dim=-1)
    assert (err <= bound[0, :, 0] + step * want[0, :, 0].norm(dim=-1)).all()
    assert torch.isnan(got[:, 1]).any(-1).all() and torch.isnan(got[:, 2]).any(-1).all()


@pytest.mark.parametrize("name", ["b4", "singles_window", "mixed_window", "singles_n128"])
def test_general_kernels_agree(monkeypatch, name):
    """With the general kernels asked for the single tokens take theirs; the bounds are the same."""
    monkeypatch.setenv("CG_KERNELS", "generic")
    c = Case(**CASES[name])
    c.call()
    c.check()


@pytest.mark.parametrize("kw", [dict(), dict(d=80, g=80, n=80), dict(dtype=torch.float32, n=128)], ids=["b4", "d80", "f32"])
@pytest.mark.parametrize("long", [90, 6000])
def test_non_finite_query_of_a_single_token(kw, long):
    c = Case([(long, 1), (70, 1), (long, 1)], H=1, grp=2, **kw)
    c.qd[0, 0, 1, 0, 5] = float("nan")
    c.qd[0, 0, 0, 2, 9] = float("inf")
    c.call()
    torch.cuda.synchronize()
    got = c.out[0, 0].double().cpu()
    want, bound = c.ref()
    step = 2.0 ** -8 if c.out.dtype == torch.bfloat16 else 2.0 ** -24
    for j, i in ((0, 0), (0, 1), (1, 1), (1, 2)):
        assert (got[j, i] - want[0, j, i]).norm() <= bound[0, j, i] + step * want[0, j, i].norm()
    assert not torch.isfinite(got[1, 0]).any() and not torch.isfinite(got[0, 2]).all()


def test_lost_pages_of_single_tokens():
    """A page outside the pool contributes nothing; a row with no other page gives zeros."""
    c = Case([(300, 1), (40, 1), (200, 1)], H=1)
    c.pages[0, 1] = c.kc.B
    c.pages[1, 0] = -5
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    got = c.out[0, 0].double().cpu()
    assert (got[:, 1] == 0).all()
    want, bound = c.ref()
    assert ((got[:, 2] - want[0, :, 2]).norm(dim=-1) <= bound[0, :, 2] + 2.0 ** -8 * want[0, :, 2].norm(dim=-1)).all()
    zk, zv = (S.pool_values(c.codec, *p) for p in c.pools)
    pg = c.table[0][:5]
    K, V = (torch.from_numpy(z[0, pg, 0].reshape(-1, 128)[:301].copy()) for z in (zk, zv))
    t = torch.arange(301) // 64 != 1
    for j in range(2):
        s = c.scale * (K[t] @ (S.full_gauge(c.G, 0, 0, 0) @ c.q[0, j, 0].double()))
        o = S.full_gauge(c.G, 0, 1, 0).T @ (torch.softmax(s, 0) @ V[t])
        assert (got[j, 0] - o).norm() <= 0.03 * V[t].norm(dim=1).max()


@pytest.mark.parametrize("kw", [dict(), dict(d=80, g=80, n=80)], ids=["b4", "d80"])
def test_many_single_rows(kw):
    """72000 (row, head) pairs, more than a grid's second dimension holds: rows that share pages, lengths and queries."""
    reps = 3000
    c = Case([(70, 1), (5, 1), (130, 1)], H=8, grp=1, pad=0, **kw)
    c.call()
    c.check()
    one = c.out.clone()
    c.pages = c.pages.repeat(reps, 1)
    c.table = np.tile(c.table, (reps, 1))
    c.lens = c.lens.repeat(reps)
    c.N = 3 * reps
    c.rows = c.rows * reps
    c.cu = torch.arange(c.N + 1, dtype=torch.int32, device="cuda")
    c.qd = c.qd.repeat(1, 1, 1, reps, 1)
    c.out = torch.full((1, 1, 8, c.N, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == 0
    got = c.out.view(1, 1, 8, reps, 3, c.d)
    assert (got == got[:, :, :, :1]).all()
    # the splits may differ: both are within the bound of the same values
    _, bound = Case([(70, 1), (5, 1), (130, 1)], H=8, grp=1, pad=0, **kw).ref()
    err = (got[0, 0, :, 0].double() - one[0, 0].double()).cpu().norm(dim=-1)
    assert (err <= 2 * (bound[0] + 2.0 ** -8 * one[0, 0].double().cpu().norm(dim=-1))).all()


@pytest.mark.parametrize("kw", [dict(), dict(d=80, g=80, n=80), dict(dtype=torch.float32)], ids=["b4", "d80", "f32"])
@pytest.mark.parametrize("new", [40, 1])
def test_window_at_the_end_of_the_longest_table(kw, new):
    """The row's last pages moved to the end of a table of 2^31 - 2^16 positions, its first one (the sinks) left in
    place, nothing between: the same results."""
    c = Case([(600, new)], H=1, P=256, window=100, sinks=4, spare_pages=0, **kw)
    want, bound = c.ref()
    M = (2 ** 31 - 2 ** 16) // 256
    far = torch.full((1, M), -1, dtype=torch.int32, device="cuda")
    far[0, 0] = c.pages[0, 0]
    far[0, M - 2:] = c.pages[0, 1:]
    c.pages, c.table = far, np.zeros((1, M), np.int8)
    c.lens += 256 * (M - 3)
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == 0
    got = c.out[:, 0].double().cpu()[:, :, :new]
    step = 2.0 ** -8 if c.out.dtype == torch.bfloat16 else 2.0 ** -24
    assert ((got - want[:, :, :new]).norm(dim=-1) <= bound[:, :, :new] + step * want[:, :, :new].norm(dim=-1)).all()


def test_two_streams_at_once():
    cs = [Case([(3000, 40), (900, 1)], grp=4, seed=3), Case([(1500, 1), (2000, 17)], grp=4, seed=5, window=900, sinks=4)]
    ws = [c.workspace()[0] for c in cs]
    for c, w in zip(cs, ws):
        c.call(w)
    torch.cuda.synchronize()
    want = [c.out.clone() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        for c in cs:
            c.base.fill_(7.0)
        torch.cuda.synchronize()
        for c, w, st in zip(cs, ws, streams):
            c.call(w, stream=st.cuda_stream)
        torch.cuda.synchronize()
        for c, x in zip(cs, want):
            assert torch.equal(c.out, x)


def test_non_finite_query_stays_in_its_row():
    c = Case([(100, 8)], H=1, grp=2)
    c.qd[0, 0, 1, 3, 5] = float("nan")
    c.qd[0, 0, 0, 6, 9] = float("inf")
    c.call()
    torch.cuda.synchronize()
    got = c.out[0, 0].double().cpu()
    want, bound = c.ref()
    ok = torch.ones(2, c.N, dtype=torch.bool)
    ok[1, 3] = ok[0, 6] = False
    ok[:, 8:] = False
    err = (got - want[0]).norm(dim=-1)
    assert (err <= bound[0] + 2.0 ** -8 * want[0].norm(dim=-1))[ok].all()
    assert not torch.isfinite(got[1, 3]).any() and not torch.isfinite(got[0, 6]).all()


def test_pages_outside_the_pool_contribute_nothing():
    c = Case([(300, 20), (200, 9)], H=1)
    c.pages[0, 1] = c.kc.B
    c.pages[1, 0] = -5
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    got = c.out[0, 0].double().cpu()
    # the same rows with the lost pages' scores at -inf
    zk, zv = (S.pool_values(c.codec, *p) for p in c.pools)
    for b, lost in ((0, 1), (1, 0)):
        n, new, first = c.held[b], c.rows[b][1], int(c.first[b])
        pg = c.table[b][: -(-n // 64)]
        K, V = (torch.from_numpy(z[0, pg, 0].reshape(-1, 128)[:n].copy()) for z in (zk, zv))
        for j in range(2):
            for i in range(new):
                t = S.visible(n - new + i, n, 0, 0) & (torch.arange(n) // 64 != lost)
                s = c.scale * (K[t] @ (S.full_gauge(c.G, 0, 0, 0) @ c.q[0, j, first + i].double()))
                o = S.full_gauge(c.G, 0, 1, 0).T @ (torch.softmax(s, 0) @ V[t])
                assert (got[j, first + i] - o).norm() <= 0.03 * V[t].norm(dim=1).max()


def test_bad_rows_are_flagged_and_leave_the_others():
    c = Case([(100, 9), (50, 7), (64, 5), (10, 4)], H=1)
    c.call()
    torch.cuda.synchronize()
    good = c.out.clone()
    c.lens[1] = 6                              # fewer than its tokens: zeros
    c.lens[2] = c.table.shape[1] * 64 + 1      # beyond the table: zeros
    c.base.fill_(7.0)
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    assert (c.out[:, :, :, 9:21] == 0).all()
    assert torch.equal(c.out[:, :, :, :9], good[:, :, :, :9]) and torch.equal(c.out[:, :, :, 21:], good[:, :, :, 21:])
    # more tokens than max_q, a cu that runs backwards or past the tokens: left as they were
    c.err.zero_()
    c.lens.copy_(torch.tensor(c.held, dtype=torch.int32))
    c.base.fill_(7.0)
    c.call(max_q=7)
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    assert (c.out[:, :, :, :9] == 7).all() and torch.equal(c.out[:, :, :, 9:].float().isfinite(), good[:, :, :, 9:].float().isfinite())
    c.err.zero_()
    c.cu.copy_(torch.tensor([0, 9, 5, 12, c.N + 1], dtype=torch.int32))
    c.base.fill_(7.0)
    c.call()
    torch.cuda.synchronize()
    assert int(c.err.item()) == cg.CG_FLAG_POS_RANGE
    assert (c.out[:, :, :, 12:] == 7).all()


def test_captured_twice_with_two_workspaces_and_on_another_stream():
    a = Case([(2000, 4), (700, 1)], grp=4, seed=3)
    b = Case([(900, 6)], grp=4, seed=5)
    assert a.workspace()[1] > 0 and b.workspace()[1] > 0
    wa, wb = a.workspace()[0], b.workspace()[0]
    a.call(wa)
    b.call(wb)
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    graphs = []
    for c, ws in ((a, wa), (b, wb)):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.call(ws)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(ws)
        graphs.append(g)
    for rep in range(4):
        a.base.fill_(7.0)
        b.base.fill_(7.0)
        for g in graphs:
            g.replay()
        b.call(b.workspace()[0])       # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1]), rep
    # the lengths are read on the device: the captured step follows them
    a.lens[0] = 1500
    graphs[0].replay()
    torch.cuda.synchronize()
    replayed = a.out.clone()
    a.base.fill_(7.0)
    a.call(wa)
    torch.cuda.synchronize()
    assert torch.equal(a.out, replayed) and not torch.equal(a.out, want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.base.fill_(7.0)
    torch.cuda.synchronize()
    a.call(wa, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(a.out, replayed)


def test_same_results_twice():
    c = Case([(2500, 30), (10, 1)], grp=4, g=128)
    c.call()
    torch.cuda.synchronize()
    first = c.out.clone()
    c.base.fill_(7.0)
    c.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out, first)


@pytest.mark.parametrize("new", [10, 1])
def test_positions_past_32_bits_of_bytes(new):
    """The last page of a pool larger than 2^32 bytes of codes (8 bits, 128 channels, 8 heads)."""
    P, H, pages = 256, 8, 17000
    codec = cg.Codec(cg.BLOCK_UNIFORM, 8, 64)
    assert P * H * pages * 128 > 2 ** 32
    c = Case([(70, new)], H=8, grp=1, bits=8, P=256, g=128)
    big = [cg.Cache(codec, s, 1, pages, H, P, 128) for s in (0, 1)]
    for s in (0, 1):
        codes, side = c.pools[s]
        src = c.table[0, 0]
        big[s].codes.view(pages, -1)[pages - 1].copy_(torch.from_numpy(codes[0, src].reshape(-1).copy()))
        big[s].side.view(pages, -1)[pages - 1].copy_(torch.from_numpy(side[0, src].copy().view(np.uint8).reshape(-1)))
    c.pages[0, 0] = pages - 1
    c.kc, c.vc = big
    c.call()
    c.check()
