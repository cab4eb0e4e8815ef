"""Rotary positions and the tables and slots of a serving step against plain references in binary64 / on the host."""
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


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------
# rotary positions
# ------------------------------------------------------------------------------------------

ROPE = [
    # L, B, Hq, H, T, d, rot, layout, scaling, dtype
    (1, 1, 4, 2, 7, 128, 128, cg.ROPE_HALF, cg.ROPE_NONE, torch.bfloat16),
    (1, 1, 4, 2, 7, 128, 128, cg.ROPE_PAIRS, cg.ROPE_NONE, torch.bfloat16),
    (2, 3, 3, 1, 5, 128, 64, cg.ROPE_HALF, cg.ROPE_LINEAR, torch.float32),
    (2, 3, 3, 1, 5, 128, 64, cg.ROPE_PAIRS, cg.ROPE_RAMP, torch.float32),
    (1, 2, 2, 2, 33, 80, 20, cg.ROPE_HALF, cg.ROPE_NONE, torch.float32),
    (1, 2, 2, 2, 33, 80, 20, cg.ROPE_PAIRS, cg.ROPE_RAMP, torch.bfloat16),
    (1, 1, 1, 1, 300, 64, 24, cg.ROPE_HALF, cg.ROPE_NONE, torch.bfloat16),
    (1, 1, 2, 1, 9, 24, 6, cg.ROPE_HALF, cg.ROPE_NONE, torch.bfloat16),
    (1, 1, 2, 1, 9, 24, 6, cg.ROPE_PAIRS, cg.ROPE_NONE, torch.float32),
    (1, 1, 2, 1, 9, 8, 2, cg.ROPE_PAIRS, cg.ROPE_NONE, torch.float32),
    (1, 1, 16, 4, 1, 256, 256, cg.ROPE_HALF, cg.ROPE_RAMP, torch.bfloat16),
    (1, 1, 8, 8, 2000, 128, 96, cg.ROPE_PAIRS, cg.ROPE_NONE, torch.bfloat16),
]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", ROPE, ids=[str(i) for i in range(len(ROPE))])
def test_rope_matches_binary64(case, inverse):
    """binary32 arithmetic: angle within 2^-30, sine and cosine 2^-22, two products and a sum (3 x 2^-24), the
    plan's frequencies exact to binary64: 2^-21 of the pair's norm; then one rounding of the type."""
    L, B, Hq, H, T, d, rot, layout, scaling, dtype = case
    rng = np.random.default_rng(T + d)
    kw = dict(base=10000.0, scaling=scaling, factor=4.0, low=1.0, high=32.0, train_len=4096, amplitude=1.25)
    plan = cg.rope_make(rot, layout, **kw)
    pos = torch.from_numpy(rng.integers(0, 2 ** 31 - 1, (B, T))).to(torch.int32)
    pos.view(-1)[0] = 0
    pos.view(-1)[-1] = 131071
    if T > 3:
        pos[:, 2] = -1
    xs = [torch.from_numpy(rng.standard_normal((L, B, T, n, d))).to(dtype).cuda().transpose(2, 3) for n in (Hq, H)]
    ys = [torch.full_like(x, 3.0) for x in xs]
    cg.kv_rope(plan, xs[0], ys[0], pos.cuda(), xs[1], ys[1], inverse=inverse)
    alone = torch.full_like(xs[1], 3.0)
    cg.kv_rope(plan, xs[1], alone, pos.cuda(), inverse=inverse)
    inplace = [x.clone() for x in xs]
    cg.kv_rope(plan, inplace[0], inplace[0], pos.cuda(), inplace[1], inplace[1], inverse=inverse)
    torch.cuda.synchronize()
    assert torch.equal(alone, ys[1])
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for x, y, z in zip(xs, ys, inplace):
        xd = x.double().cpu()
        want = S.rope_ref(xd, pos, rot, layout, inverse=inverse, **kw)
        kept = (pos < 0)[None, :, None, :, None].expand_as(want)
        got, got2 = y.double().cpu(), z.double().cpu()
        assert (got[kept] == 3.0).all()
        assert torch.equal(torch.where(kept, want, got), got2)
        norm = 1.25 * xd.abs().amax(-1, keepdim=True) * 1.42
        bad = (torch.where(kept, want, got) - want).abs() > step * want.abs() + 2.0 ** -21 * norm
        assert not bad.any(), float((got - want).abs().max())
        if rot < d:
            assert torch.equal(got2[..., rot:], xd[..., rot:])


def test_rope_inverse_is_the_gradient():
    """<R x, y> = <x, R^T y>, and R^T y against central differences of the loss <R x, y> in binary64 steps."""
    rng = np.random.default_rng(5)
    plan = cg.rope_make(64, cg.ROPE_PAIRS, amplitude=0.75)
    pos = _i32([[5, 1000, 77]])
    x, y = (torch.from_numpy(rng.standard_normal((1, 1, 2, 3, 96))).float().cuda() for _ in range(2))
    f, b = torch.empty_like(x), torch.empty_like(x)
    cg.kv_rope(plan, x, f, pos)
    cg.kv_rope(plan, y, b, pos, inverse=True)
    torch.cuda.synchronize()
    # 576 products with errors of 2^-20 relative to norms of about 24 each
    assert abs((f.double() * y.double()).sum() - (x.double() * b.double()).sum()).item() <= 576 * 2.0 ** -20
    h = 2.0 ** -6
    for ch in (0, 1, 30, 63, 64, 95):
        e = torch.zeros_like(x)
        e[0, 0, 1, 1, ch] = h
        up, dn = torch.empty_like(x), torch.empty_like(x)
        cg.kv_rope(plan, x + e, up, pos)
        cg.kv_rope(plan, x - e, dn, pos)
        torch.cuda.synchronize()
        diff = ((up.double() - dn.double()) * y.double()).sum().item() / (2 * h)
        # linear: the quotient is off by the roundings of three terms, at most 8 * 2^-22 / (2 h), no truncation
        assert abs(diff - b[0, 0, 1, 1, ch].item()) <= 8 * 2.0 ** -22 / h


def test_rope_empty_and_non_finite():
    plan = cg.rope_make(32, cg.ROPE_HALF)
    x = torch.zeros((1, 1, 1, 0, 64), device="cuda")
    cg.kv_rope(plan, x, x, torch.zeros((1, 0), dtype=torch.int32, device="cuda"))
    x = torch.ones((1, 1, 1, 4, 64), device="cuda")
    x[0, 0, 0, 1, 3] = float("inf")
    x[0, 0, 0, 2, 40] = float("nan")
    y = torch.empty_like(x)
    cg.kv_rope(plan, x, y, _i32([[0, 1, 2, 3]]))
    torch.cuda.synchronize()
    bad = ~torch.isfinite(y.cpu())[0, 0, 0]
    assert bad[1].nonzero().flatten().tolist() == [3, 19] and bad[2].nonzero().flatten().tolist() == [40]
    assert not bad[0].any() and not bad[3].any()


# ------------------------------------------------------------------------------------------
# tables and slots
# ------------------------------------------------------------------------------------------

def _step(held, add, P, extra=4, pad=5, seed=0, in_place=False):
    rng = np.random.default_rng(seed)
    need = [-(-(h + n) // P) for h, n in zip(held, add)]
    had = [-(-h // P) for h in held]
    maxp = max(need) + 1
    total = sum(need) + extra
    perm = rng.permutation(total)
    table = np.full((len(held), maxp), -1, np.int32)
    at = 0
    for b, k in enumerate(had):
        table[b, :k] = perm[at: at + k]
        at += k
    free = perm[at:].tolist()
    N = sum(add) + pad
    pool = cg.PagePool(total)
    pool.free[: len(free)] = _i32(free)
    pool.count.fill_(len(free))
    h, a, pages = _i32(held), _i32(add), torch.from_numpy(table.copy()).cuda()
    cu, pos, slots, err = _i32([9] * (len(held) + 1)), _i32([9] * N), _i32([9] * N), _i32([0])
    lens = h if in_place else _i32([9] * len(held))
    cg.kv_page_map(h, a, pool, pages, P, cu, lens, pos, slots, err)
    torch.cuda.synchronize()
    want = S.page_map_ref(held, add, free, table, P, N)
    assert int(err.item()) == 0
    for got, w in zip((cu, lens, pos, slots, pages), want[:5]):
        assert got.cpu().tolist() == w
    assert int(pool.count.item()) == len(want[5])
    return pool, pages, lens, want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("held,add,P", [
    ([0], [1], 64), ([64], [1], 64), ([63], [1], 64), ([63], [2], 64), ([0], [0], 64), ([5, 0, 64, 127, 128], [0, 0, 64, 1, 200], 64),
    ([100] * 64, [1] * 64, 256), ([0] * 3, [5000, 1, 7000], 128), (list(range(1500)), [b % 7 for b in range(1500)], 64),
    (list(range(1024)), [3] * 1024, 64), ([0] * 1025, [5] * 1025, 192)])
def test_page_map_matches_request_by_request(held, add, P, in_place):
    _step(held, add, P, in_place=in_place)


def test_page_release_gives_back_and_is_taken_again():
    held, add = [100, 0, 64, 300], [30, 65, 0, 1]
    pool, pages, lens, want = _step(held, add, 64)
    done = _i32([0, 1, 0, 1])
    err = _i32([0])
    before = pages.cpu().tolist()
    cg.kv_page_release(lens, done, pool, pages, 64, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and lens.cpu().tolist() == [130, 0, 64, 0]
    back = before[1][:2] + before[3][:5]
    stack = pool.free.cpu().tolist()[: int(pool.count.item())]
    assert stack == want[5] + back
    assert pages.cpu().tolist() == [before[0], [-1] * len(before[1]), before[2], [-1] * len(before[3])]
    # the next step takes them from the top
    cu, pos, slots = _i32([0] * 5), _i32([0] * 70), _i32([0] * 70)
    cg.kv_page_map(lens, _i32([0, 70, 0, 0]), pool, pages, 64, cu, lens, pos, slots, err)
    torch.cuda.synchronize()
    assert pages.cpu()[1, :2].tolist() == [back[-1], back[-2]] and int(err.item()) == 0
    assert slots.cpu().tolist() == [back[-1] * 64 + i for i in range(64)] + [back[-2] * 64 + i for i in range(6)]


def test_page_release_of_many_rows_skips_holes():
    B, P = 1300, 64
    table = torch.arange(B * 3, dtype=torch.int32).reshape(B, 3)
    table[5, 1] = -1
    table[7, 0] = 10 ** 6
    pool = cg.PagePool(B * 3)
    pool.count.zero_()
    lens, pages, err = _i32([150] * B), table.cuda(), _i32([0])
    done = _i32([b % 2 for b in range(B)])
    cg.kv_page_release(lens, done, pool, pages, P, err)
    torch.cuda.synchronize()
    want = [int(p) for b in range(1, B, 2) for p in table[b] if 0 <= p < B * 3]
    assert pool.free.cpu().tolist()[: int(pool.count.item())] == want and int(err.item()) == 0
    assert lens.cpu().tolist() == [150 * (1 - b % 2) for b in range(B)]


def test_page_map_flags():
    def run(held, add, maxp=4, total=8, count=8, N=200):
        pool = cg.PagePool(total)
        pool.count.fill_(count)
        B = len(held)
        pages = torch.full((B, maxp), -1, dtype=torch.int32, device="cuda")
        out = [_i32([9] * n) for n in (B + 1, B, N, N)]
        err = _i32([0])
        cg.kv_page_map(_i32(held), _i32(add), pool, pages, 64, *out, err)
        torch.cuda.synchronize()
        return int(err.item()), pages.cpu().tolist(), [t.cpu().tolist() for t in out], int(pool.count.item())

    # the pool runs out: -1 in the table and as slots, the rest as usual
    flag, pages, (cu, lens, pos, slots), left = run([0, 0], [70, 70], count=3)
    assert flag & cg.CG_FLAG_POOL_EMPTY and left == 0 and cu == [0, 70, 140] and lens == [70, 70]
    assert pages[1][1] == -1 and slots[70 + 64: 140] == [-1] * 6 and pos[70 + 64: 140] == list(range(64, 70))
    assert all(s >= 0 for s in slots[: 70 + 64])
    # past the table
    flag, pages, (cu, lens, pos, slots), left = run([250], [20])
    assert flag & cg.CG_FLAG_POS_RANGE and lens == [270] and slots[6:20] == [-1] * 14
    # negative counts
    flag, pages, (cu, lens, pos, slots), left = run([-3, 0], [2, -5])
    assert flag & cg.CG_FLAG_POS_RANGE and cu == [0, 2, 2] and left == 8 and slots[0] == -1
    # more tokens than there is room for
    flag, _, (cu, _, pos, slots), _ = run([0], [100], N=50)
    assert flag & cg.CG_FLAG_POS_RANGE and cu == [0, 100] and pos == list(range(50))
    # sums past 2^31 stick
    flag, _, (cu, lens, _, _), _ = run([2 ** 31 - 1, 0], [2 ** 31 - 1, 5])
    assert flag & cg.CG_FLAG_POS_RANGE and cu == [0, 2 ** 31 - 1, 2 ** 31 - 1] and lens[0] == 2 ** 31 - 1


def test_page_map_captured():
    """A captured step replayed: every replay maps the next token of each row."""
    B, P = 5, 64
    pool = cg.PagePool(40)
    lens, add = _i32([60, 0, 127, 64, 3]), _i32([1] * B)
    table = torch.full((B, 6), -1, dtype=torch.int32)
    held = lens.cpu().tolist()
    free = pool.free.cpu().tolist()
    for b, h in enumerate(held):
        for i in range(-(-h // P)):
            table[b, i] = free.pop()
    pool.count.fill_(len(free))
    pages, cu, pos, slots, err = table.cuda(), _i32([0] * (B + 1)), _i32([0] * B), _i32([0] * B), _i32([0])
    call = lambda: cg.kv_page_map(lens, add, pool, pages, P, cu, lens, pos, slots, err)  # noqa: E731
    saved = [t.clone() for t in (lens, pages, pool.count)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for t, v in zip((lens, pages, pool.count), saved):
        t.copy_(v)
    tab = table.tolist()
    for _ in range(6):
        g.replay()
        torch.cuda.synchronize()
        want = S.page_map_ref(held, [1] * B, free, tab, P, B)
        held, tab, free = want[1], want[4], want[5]
        assert [t.cpu().tolist() for t in (lens, pos, slots, pages)] == [want[1], want[2], want[3], want[4]]
        assert int(pool.count.item()) == len(free) and int(err.item()) == 0
