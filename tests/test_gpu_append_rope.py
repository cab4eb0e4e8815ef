"""Packed tokens turned by their positions and encoded through their slots (kv_append_rope) against the oracle's
encoding of the keys turned in binary64; queries against the same rotation."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2607_20538_amd import codec as cg
from paper_2607_20538_amd import synth

import _serving as S
from _parity import cache_to_host, check_fused_codes, group_rel_err, to_cg, x_dev, x_f64
from test_gpu_append_slots import _pools, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


BU = lambda bits, n: O.Codec(backend=O.BLOCK_UNIFORM, bits=bits, block_c=n)  # noqa: E731
PASS = O.Codec(backend=O.PASSTHROUGH)

CASES = {
    # oracle codec, d, g, dtype, tokens, rotated channels, layout
    "one": (BU(4, 64), 128, 128, "bf16", 1, 128, cg.ROPE_HALF),
    "few": (BU(4, 64), 128, 128, "bf16", 37, 128, cg.ROPE_HALF),
    "b4_g128": (BU(4, 64), 128, 128, "bf16", 1500, 128, cg.ROPE_HALF),
    "b4_g128_pairs": (BU(4, 64), 128, 128, "bf16", 1500, 128, cg.ROPE_PAIRS),
    "b6_g32": (BU(6, 64), 128, 32, "bf16", 1501, 64, cg.ROPE_HALF),
    "b6_g32_pairs": (BU(6, 64), 128, 32, "bf16", 1501, 32, cg.ROPE_PAIRS),
    "b3_g64": (BU(3, 32), 128, 64, "bf16", 1033, 96, cg.ROPE_HALF),
    "b8_g16": (BU(8, 16), 128, 16, "bf16", 1033, 128, cg.ROPE_PAIRS),
    "b8_g128": (BU(8, 32), 128, 128, "bf16", 1700, 128, cg.ROPE_HALF),
    "b2_g8": (BU(2, 32), 128, 8, "bf16", 1033, 2, cg.ROPE_HALF),
    "rot6": (BU(4, 32), 128, 32, "bf16", 1400, 6, cg.ROPE_HALF),
    "rot10_pairs": (BU(4, 32), 128, 32, "bf16", 1400, 10, cg.ROPE_PAIRS),
    "n128": (BU(4, 128), 128, 128, "bf16", 700, 128, cg.ROPE_HALF),
    "d64": (BU(4, 32), 64, 16, "bf16", 700, 64, cg.ROPE_HALF),
    "d96_f32": (BU(4, 32), 96, 32, "f32", 300, 96, cg.ROPE_PAIRS),
    "d128_f32": (BU(8, 32), 128, 128, "f32", 1500, 128, cg.ROPE_HALF),
    "d80": (BU(8, 80), 80, 80, "bf16", 50, 40, cg.ROPE_HALF),
    "d256": (BU(4, 64), 256, 128, "bf16", 90, 256, cg.ROPE_HALF),
    "g5": (BU(8, 80), 80, 5, "bf16", 50, 80, cg.ROPE_PAIRS),
    "pass": (PASS, 128, 128, "bf16", 1100, 128, cg.ROPE_HALF),
    "pass_f32": (PASS, 64, 64, "f32", 33, 64, cg.ROPE_PAIRS),
}

# positions up to 100000: a binary64 angle is off by 2^-37 turns there, the kernel's by 2^-31: nothing beside the
# 2^-22 or so that binary32 sines and two products leave of a channel
FAR = 100000


def _setup(oc, d, g, dtype, N, L=2, H=3, seed=0):
    P = 64
    w = synth.Workload("rope", L=L, B=1, H=H, T=N, d=d, dtype=dtype, g=g, backend="bu", bits=4, data_seed=0x520 + N + seed)
    G = O.gauge_make(O.GAUGE_HAAR, L, H, d, g, seed=9)
    shp = cg.shape(L, H, d, g)
    Gd = cg.alloc_gauge(shp)
    cg.gauge_make(cg.GAUGE_USER, shp, params=G, G_host=None, G_dev=Gd)
    pages = -(-N // P) + 2
    rng = np.random.default_rng(N)
    slots = rng.permutation(pages * P)[:N].astype(np.int64)
    pos = rng.integers(0, FAR, N)
    xs = [synth.kv_tensor(w, s) for s in (0, 1)]
    return P, G, shp, Gd, to_cg(oc), pages, rng, slots, pos, xs


# as many token rows (2 layers x 3 heads) as go through the matrix-core encoder
MANY = {
    "b4_g128": (BU(4, 64), 128, 128, "bf16", 3600, 128, cg.ROPE_HALF),
    "b4_g128_pairs": (BU(4, 64), 128, 128, "bf16", 3501, 128, cg.ROPE_PAIRS),
    "b6_g32": (BU(6, 64), 128, 32, "bf16", 3450, 64, cg.ROPE_HALF),
    "b6_g32_pairs": (BU(6, 16), 128, 32, "bf16", 3450, 32, cg.ROPE_PAIRS),
    "b3_g64": (BU(3, 32), 128, 64, "bf16", 3517, 96, cg.ROPE_HALF),
    "b8_g16": (BU(8, 16), 128, 16, "bf16", 3431, 112, cg.ROPE_PAIRS),
    "b2_g8": (BU(2, 32), 128, 8, "bf16", 3440, 16, cg.ROPE_HALF),
    "rot40": (BU(4, 32), 128, 128, "bf16", 3500, 40, cg.ROPE_HALF),     # not in sixteens: the kernel of few tokens
}


@pytest.mark.parametrize("tokens_first", [True, False])
@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name, tokens_first):
    _check(*CASES[name], tokens_first)


@pytest.mark.parametrize("name", MANY)
def test_many_tokens_against_the_oracle(name):
    _check(*MANY[name], True)


def _check(oc, d, g, dtype, N, rot, layout, tokens_first):
    L, H = 2, 3
    P, G, shp, Gd, c, pages, rng, slots, pos, xs = _setup(oc, d, g, dtype, N)
    if N > 1:
        skipped = rng.random(N) < 0.1
        slots[skipped] = -1 - rng.integers(0, 5, int(skipped.sum()))
        out_of_it = rng.random(N) < 0.1                 # negative positions: neither appended nor turned
        pos[out_of_it] = -1 - rng.integers(0, 5, int(out_of_it.sum()))
    live = (slots >= 0) & (pos >= 0)
    pools = _pools(c, L, pages, H, P, d)
    lay = (lambda t: t.transpose(2, 3).contiguous().transpose(2, 3)) if tokens_first else (lambda t: t)
    dev = [lay(x_dev(x)) for x in xs]
    q = torch.from_numpy(rng.standard_normal((L, 1, 5, N, d))).to(dev[0].dtype)
    qd = lay(q.cuda())
    qo = torch.full_like(qd, 7.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = cg.rope_make(rot, layout, base=500000.0, amplitude=1.25)
    p32, s32 = (torch.from_numpy(v).to(torch.int32).cuda() for v in (pos, slots))
    cg.kv_append_rope(0, L, plan, *dev, p32, s32, Gd, shp, c, *pools, qd, qo, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    turn = lambda t: S.rope_ref(t.double(), torch.from_numpy(pos)[None], rot, layout, base=500000.0, amplitude=1.25)  # noqa: E731
    # queries: as kv_rope turns them, untouched where the position is negative
    other = torch.full_like(qd, 7.0)
    cg.kv_rope(plan, qd, other, p32[None].contiguous())
    torch.cuda.synchronize()
    assert torch.equal(qo, other)
    want, got = turn(q), qo.double().cpu()
    ok = torch.from_numpy(pos >= 0)
    # a rounding, and the binary32 sines and products (2^-21 of the pair's size)
    lim = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * want.abs() + 2.0 ** -21 * 1.25 * 6.0
    assert ((got - want).abs() <= lim)[:, :, :, ok].all() and (got[:, :, :, ~ok] == 7.0).all()
    # keys and values
    keep = np.where(live, slots, -1).tolist()
    for s in (0, 1):
        rows = _rows(cache_to_host(pools[s], oc, s), keep, P)
        x = torch.from_numpy(x_f64(xs[s]))
        x = (turn(x) if s == 0 else x)[:, :, :, torch.from_numpy(live)].float().numpy()
        x = np.ascontiguousarray(x)
        n = int(live.sum())
        z, _ = O.kv_encode(O.Codec(backend=O.PASSTHROUGH), s, x, G, T_cap=n)
        if oc.backend == O.PASSTHROUGH:
            zg = np.ascontiguousarray(rows["codes"]).view(np.float32).reshape(z["codes"].shape)
            assert group_rel_err(z["codes"], zg, g) <= 1e-5
            continue
        code, _ = O.kv_encode(oc, s, x, G, T_cap=n)
        check_fused_codes(rows, code, z["codes"], oc, s, d, n)


@pytest.mark.parametrize("N", [20, 3500])
def test_without_a_turn_it_appends_as_kv_append_slots_does(N):
    """Position 0 and amplitude 1: the keys are what they were.  Values always are."""
    oc = BU(4, 64)
    P, G, shp, Gd, c, pages, _, slots, pos, xs = _setup(oc, 128, 128, "bf16", N)
    a, b = _pools(c, 2, pages, 3, P, 128), _pools(c, 2, pages, 3, P, 128)
    dev = [x_dev(x) for x in xs]
    s32 = torch.from_numpy(slots).to(torch.int32).cuda()
    cg.kv_append_rope(0, 2, cg.rope_make(128), *dev, torch.zeros_like(s32), s32, Gd, shp, c, *a)
    cg.kv_append_slots(0, 2, *dev, s32, Gd, shp, c, *b)
    torch.cuda.synchronize()
    for s in (0, 1):
        x = xs[s]
        z, _ = O.kv_encode(O.Codec(backend=O.PASSTHROUGH), s, x, G, T_cap=N)
        want, _ = O.kv_encode(oc, s, x, G, T_cap=N)
        for pool in (a, b):
            check_fused_codes(_rows(cache_to_host(pool[s], oc, s), slots.tolist(), P), want, z["codes"], oc, s, 128, N)


@pytest.mark.parametrize("N", [20, 1500, 3500])
def test_flags(N):
    """Slots past the pool and non-finite tokens raise their flags; a token left out raises none."""
    oc = BU(4, 64)
    P, G, shp, Gd, c, pages, _, slots, pos, xs = _setup(oc, 128, 128, "bf16", N)
    call = lambda k, v, p, s: cg.kv_append_rope(0, 2, cg.rope_make(128), k, v, p, s, Gd, shp, c, *pools, err_flag=err)  # noqa: E731
    dev = [x_dev(x) for x in xs]
    p32, s32 = (torch.from_numpy(v).to(torch.int32).cuda() for v in (pos, slots))
    for what, flag in (("slot", cg.CG_FLAG_POS_RANGE), ("key", cg.CG_FLAG_NONFINITE), ("value", cg.CG_FLAG_NONFINITE), ("left out", 0)):
        pools, err = _pools(c, 2, pages, 3, P, 128), torch.zeros(1, dtype=torch.int32, device="cuda")
        k, v, p, s = dev[0].clone(), dev[1].clone(), p32.clone(), s32.clone()
        if what == "slot":
            s[7] = pages * P
        elif what == "key":
            k[1, 0, 2, 7, 5] = float("inf")
        elif what == "value":
            v[1, 0, 2, 7, 5] = float("nan")
        else:
            k[1, 0, 2, 7, 5] = v[1, 0, 2, 7, 5] = float("nan")
            p[7], s[7] = -3, pages * P
        call(k, v, p, s)
        torch.cuda.synchronize()
        # (an infinite range is one that binary16 does not hold, too)
        assert int(err.item()) & ~(cg.CG_FLAG_SIDE_OVERFLOW if what in ("key", "value") else 0) == flag, what


def test_queries_in_place_and_far_positions():
    """q_out may be q; positions up to 2^31 - 1."""
    oc = BU(4, 64)
    P, G, shp, Gd, c, pages, rng, slots, _, xs = _setup(oc, 128, 128, "bf16", 70)
    pos = torch.from_numpy(rng.integers(2 ** 30, 2 ** 31 - 1, 70)).to(torch.int32).cuda()
    pos[3] = 2 ** 31 - 1
    dev = [x_dev(x) for x in xs]
    q = torch.randn((2, 1, 6, 70, 128), device="cuda").to(torch.bfloat16)
    want = torch.empty_like(q)
    plan = cg.rope_make(128)
    cg.kv_rope(plan, q, want, pos[None].contiguous())
    pools = _pools(c, 2, pages, 3, P, 128)
    cg.kv_append_rope(0, 2, plan, *dev, pos, torch.from_numpy(slots).to(torch.int32).cuda(), Gd, shp, c, *pools, q, q)
    torch.cuda.synchronize()
    assert torch.equal(q, want)


def test_layers_of_a_pool():
    """Views of one layer go to that cache layer alone."""
    oc = BU(4, 64)
    P, G, shp, Gd, c, pages, _, slots, pos, xs = _setup(oc, 128, 128, "bf16", 40)
    dev = [x_dev(x) for x in xs]
    p32, s32 = (torch.from_numpy(v).to(torch.int32).cuda() for v in (pos, slots))
    plan = cg.rope_make(128)
    both, one = _pools(c, 2, pages, 3, P, 128), _pools(c, 2, pages, 3, P, 128)
    cg.kv_append_rope(0, 2, plan, *dev, p32, s32, Gd, shp, c, *both)
    cg.kv_append_rope(1, 2, plan, *(t[1:] for t in dev), p32, s32, Gd, shp, c, *one)
    torch.cuda.synchronize()
    for a, b in zip(both, one):
        half = a.codes.numel() // 2
        assert torch.equal(a.codes[half:], b.codes[half:]) and (b.codes[:half] == 0xA5).all()


@pytest.mark.parametrize("bits,n,layout", [(4, 64, cg.ROPE_HALF), (6, 16, cg.ROPE_PAIRS), (3, 32, cg.ROPE_HALF)])
def test_long_ranges_and_tokens_that_are_not_finite(monkeypatch, bits, n, layout):
    """The bytes do not depend on how many tiles of tokens a workgroup takes; tokens with an infinity, a NaN or a channel
    near binary32's largest get the bytes that the kernel of few tokens gives them."""
    oc = BU(bits, n)
    N, L, H, P = 12001, 1, 2, 64
    pages = N // P + 2
    shp, Gd = S.gauge_dev(S.haar(L, H, 128, 64, 7))
    torch.manual_seed(N + bits)
    x = [torch.randn((L, 1, N, H, 128), device="cuda").to(torch.bfloat16).transpose(2, 3) for _ in (0, 1)]
    x[0][0, 0, 1, 2200, 5] = float("inf")
    x[0][0, 0, 0, 2201, 100] = float("nan")
    x[0][0, 0, 0, 9000, 64] = 3e38
    x[1][0, 0, 1, 77, 1] = float("-inf")
    odd = [(0, 1, 2200), (0, 0, 2201), (0, 0, 9000), (1, 1, 77)]    # (keys or values, head, token)
    slots = torch.randperm(pages * P, device="cuda")[:N].to(torch.int32)
    slots[5::97] = -1
    pos = torch.randint(0, 100000, (N,), dtype=torch.int32, device="cuda")
    pos[6::97] = -7
    plan = cg.rope_make(128, layout)
    got = []
    for tiles in ("1", "3", "40", "", "generic"):
        if tiles == "generic":
            monkeypatch.delenv("CG_TILES_PER_WG")
            monkeypatch.setenv("CG_KERNELS", "generic")
        else:
            monkeypatch.setenv("CG_TILES_PER_WG", tiles)
        pools = _pools(to_cg(oc), L, pages, H, P, 128)
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        cg.kv_append_rope(0, L, plan, *x, pos, slots, Gd, shp, to_cg(oc), *pools, err_flag=err)
        torch.cuda.synchronize()
        assert int(err.item()) == cg.CG_FLAG_NONFINITE | cg.CG_FLAG_SIDE_OVERFLOW
        got.append([(p.codes.clone(), p.side.clone()) for p in pools])
    for g in got[1:4]:
        for (ca, sa), (cb, sb) in zip(got[0], g):
            assert torch.equal(ca, cb) and torch.equal(sa, sb)
    sl = slots.tolist()
    for kv, h, i in odd:
        page, at = divmod(sl[i], P)
        (ca, sa), (cb, sb) = ([t.reshape(pages, H, P, -1)[page, h, at].contiguous() for t in g[kv]] for g in (got[0], got[4]))
        sa, sb = sa.view(torch.float16), sb.view(torch.float16)     # (a NaN has either sign)
        assert torch.equal(ca, cb) and torch.allclose(sa, sb, rtol=0, atol=0, equal_nan=True)
