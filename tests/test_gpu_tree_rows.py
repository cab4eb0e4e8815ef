"""Batches whose last rows run backwards: the tokens of the rows before them are those rows' alone, those behind all rows are cleared."""
import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

import _tree as T
from test_gpu_tree import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


# rows of 1000 and 70 nodes, then one that runs backwards; 40000 tokens of padding take longer to clear than the rows to write
@pytest.mark.parametrize("back", [5, 0, -3, 1069])
@pytest.mark.parametrize("more", [0, 1, 130])
def test_masks_and_paths_before_a_row_that_runs_backwards(back, more):
    rng = np.random.default_rng(3)
    trees = [T.tree(1000, "near", rng), T.tree(70, "chain", rng)]
    n, N, words = 1070, 41070, 16
    cu, B = i32([0, 1000, n] + [back] * (1 + more)), 3 + more
    parent = i32(sum(trees, []) + [0] * (N - n))
    pos, mask = torch.full((N,), 77, dtype=torch.int32, device="cuda"), torch.full((N, words), 5, dtype=torch.int64, device="cuda")
    err = i32([0])
    cg.kv_tree_map(parent, cu, i32([1003, 75] + [9] * (1 + more)), pos, mask, err)
    torch.cuda.synchronize()
    (m0, d0), (m1, d1) = (T.closure(t) for t in trees)
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE
    assert pos[:n].tolist() == [3 + k for k in d0] + [5 + k for k in d1]
    assert np.array_equal(mask[:n].cpu().numpy(), T.words_of(m0 + m1, words))
    assert (pos[n:] == -1).all() and (mask[n:] == 0).all()
    draft, target = rng.integers(0, 2, N).tolist(), rng.integers(0, 2, N).tolist()
    path, kept, nxt, err = i32([9] * N), i32([9] * B), i32([9] * B), i32([0])
    cg.kv_tree_accept(parent, cu, i32(draft), i32(target), path, kept, nxt, None, err)
    torch.cuda.synchronize()
    ways = [T.walk(t, draft[a: a + len(t)], target[a: a + len(t)])[0] for t, a in zip(trees, (0, 1000))]
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE
    assert path[:n].tolist() == ways[0] + [-1] * (1000 - len(ways[0])) + ways[1] + [-1] * (70 - len(ways[1]))
    assert kept[:2].tolist() == [len(w) for w in ways] and (path[n:] == -1).all()
