"""Sizes of a serving step's workspaces, plans of its rotary positions and page tables, on the host."""
import ctypes as C
import gc
import math
import random
from decimal import Decimal, localcontext

import pytest
import torch

from paper_2607_20538_amd import codec as cg


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("H,grp,d,nl,N,B,maxp,P", [
    (8, 4, 128, 1, 4096, 1, 400, 64), (8, 4, 128, 1, 4096, 64, 400, 64), (2, 2, 64, 4, 300, 7, 60, 64),
    (16, 1, 256, 32, 20000, 300, 500, 256), (32, 40, 64, 8, 338, 26, 3696, 256), (1, 130, 128, 1, 5000, 600, 4000, 256),
    (1, 3, 80, 2, 1, 1, 9, 192), (4, 9, 128, 1, 900, 900, 16, 64)])
def test_workspace_limit_covers_every_smaller_call(H, grp, d, nl, N, B, maxp, P):
    """The size of one call does not grow with its tokens (fewer are split into more parts), the limit covers them all."""
    shp, rng = cg.shape(max(nl, 1), H, d, d), random.Random(N + d)
    limit = cg.attend_chunk_workspace_limit(shp, nl, N, B, H * grp, maxp, P)
    for k in range(3000):
        n, b = (N if k % 3 == 0 else _log_int(rng, 1, N)), (B if k % 5 == 0 else _log_int(rng, 1, B))
        mq = rng.choice([1, n, _log_int(rng, 1, n)])
        window, sinks = rng.choice([(0, 0), (_log_int(rng, 1, 9000), rng.choice([0, 4, 3000]))])
        need = cg.attend_chunk_workspace_bytes(shp, _log_int(rng, 1, nl), n, b, mq, H * grp, _log_int(rng, 1, maxp), P, window, sinks)
        assert need <= limit, (n, b, mq, window, sinks)


def test_workspace_of_one_call_is_not_a_limit():
    shp = cg.shape(1, 8, 128, 128)
    need = lambda n: cg.attend_chunk_workspace_bytes(shp, 1, n, 1, n, 32, 400, 64)  # noqa: E731
    assert need(4096) == 0 < need(1024) < need(700)
    limit = cg.attend_chunk_workspace_limit(shp, 1, 4096, 1, 32, 400, 64)
    assert max(need(n) for n in range(1, 4097)) <= limit <= 2 ** 28


def test_workspace_limit_of_nothing_and_of_bad_sizes():
    shp = cg.shape(1, 8, 128, 128)
    lim = lambda *a: cg.attend_chunk_workspace_limit(shp, *a)  # noqa: E731
    assert lim(1, 4096, 1, 32, 4, 64) == 0                         # rows too short to split
    assert lim(0, 1, 1, 32, 400, 64) == lim(1, 1, 1, 31, 400, 64) == lim(1, 1, 1, 32, 400, 63) == lim(1, 0, 1, 32, 400, 64) == 0
    assert lim(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 8, 400, 64) <= 2 ** 30


# ------------------------------------------------------------------------------------------
# turns per position
# ------------------------------------------------------------------------------------------

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899863")


@pytest.mark.parametrize("scaling", [cg.ROPE_NONE, cg.ROPE_LINEAR, cg.ROPE_RAMP])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1000000.5, 1.0, 1e-4])
@pytest.mark.parametrize("d_rot", [2, 6, 20, 64, 96, 128, 256])
def test_rope_steps_are_the_turns_to_64_bits(d_rot, base, scaling):
    """The plan's fractions against 70-digit arithmetic, in units of 2^-64 turns.  A power and a quotient in 64-bit
    significands: 2^-63 f for the power, f |ln f| 2^-65 for its exponent, 3 2^-64 f for two or three more operations (RAMP's
    blend: as many again), over 2 pi, and half a unit: 1 + 2 f in all, of f radians."""
    with localcontext() as ctx:
        ctx.prec = 70
        factor, low, high, train = 8.1, 1.0, 4.0, 8192
        plan = cg.rope_make(d_rot, cg.ROPE_HALF, base=base, scaling=scaling, factor=factor, low=low, high=high, train_len=train)
        for i in range(d_rot // 2):
            f0 = (Decimal(base).ln() * -2 * i / d_rot).exp()
            f = f0
            if scaling == cg.ROPE_LINEAR:
                f = f0 / Decimal(factor)
            if scaling == cg.ROPE_RAMP:
                w = min(Decimal(1), max(Decimal(0), (train * f0 / (2 * PI) - Decimal(low)) / (Decimal(high) - Decimal(low))))
                f = f0 * (1 - w) / Decimal(factor) + f0 * w
            want = f / (2 * PI) % 1 * 2 ** 64
            off = abs(Decimal(plan.step[i]) - want)
            off = min(off, 2 ** 64 - off)
            lim = 1 + 2 * f0 * (1 + abs(f0.ln()) / 16) * (4 if scaling == cg.ROPE_RAMP else 1)
            assert off <= lim, (i, off)
            if base >= 1:
                # at the last position: 2^-32 turns
                assert off * (2 ** 31 - 1) <= 2 ** 32 * (4 if scaling == cg.ROPE_RAMP else 2)


# ------------------------------------------------------------------------------------------
# page tables
# ------------------------------------------------------------------------------------------

def test_page_table_refuses_what_the_kernels_would_misread():
    wide = torch.arange(24, dtype=torch.int32).reshape(4, 6)
    for bad in (wide[:, :3], wide[:, ::2], wide.t(), wide.long(), wide[0]):
        with pytest.raises(ValueError):
            cg.page_table(bad, 64)
    for good in (wide, wide[1:], wide[:1, :3]):
        pt = cg.page_table(good, 64)
        assert (pt.pages, pt.max_pages, pt.page_size) == (good.data_ptr(), good.shape[1], 64)


def test_page_table_keeps_its_tensor():
    pt = cg.page_table(torch.arange(6, dtype=torch.int32).reshape(2, 3).clone(), 64)
    gc.collect()
    assert (C.c_int32 * 6).from_address(pt.pages)[:] == list(range(6))
