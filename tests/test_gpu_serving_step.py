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
