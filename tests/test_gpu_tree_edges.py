"""Attention of trees: units with keys or values beyond binary16 at every code width and tile, calls that stay in the workspace
asked for, steps that run side by side; masks of rows with parents that are none."""
import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

from test_gpu_tree import Step, i32
from test_gpu_tree_attend import Tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


@pytest.mark.parametrize("which", ["keys", "values"])
@pytest.mark.parametrize("grp", [1, 2])                # all of a row's queries in one group of 32, in two
@pytest.mark.parametrize("d,n", [(128, 64), (128, 32), (64, 64)])
@pytest.mark.parametrize("bits", [2, 3, 4, 6, 8])
def test_ranges_beyond_binary16(bits, d, n, grp, which):
    """Ranges up to 60000 times the largest code at every ninth position of a stretch and at a node; the scale takes the keys'
    scores to a few units, so that a wrong channel would show in the weights."""
    top = 60000.0 * (2 ** bits - 1)
    c = Tree([(300, 20), (70, 9), (31, 1)], bits=bits, d=d, n=n, g=32, grp=grp, seed=bits,
             scale=1.0 / (top * d ** 0.5) if which == "keys" else None)
    side = c.pools[0 if which == "keys" else 1][1]
    for b, p in [(0, k) for k in range(100, 260, 9)] + [(0, 303), (1, 5), (1, 71), (2, 31)]:
        at = (slice(None), c.table[b, p // 64], slice(None), p % 64)
        side[at][..., 1] = np.float16(60000.0)
        side[at][..., 0] = np.float16(-30000.0)
    c.upload()
    c.call()
    c.check()


def test_calls_stay_in_the_workspace_asked_for():
    rng = np.random.default_rng(11)
    for k in range(60):
        d, H = int(rng.choice([64, 128])), int(rng.choice([1, 2, 5]))
        grp, L = int(rng.choice([1, 2, 3, 5, 8, 31, 33, 64])), int(rng.choice([1, 1, 2]))
        B = int(rng.integers(1, 9))
        rows = [(int(rng.integers(0, 300)), int(rng.integers(0, max(2, 150 // grp)))) for _ in range(B)]
        rows[0] = (rows[0][0], max(1, rows[0][1]))
        dtype = torch.float32 if k % 6 == 5 else torch.bfloat16
        c = Tree(rows, d=d, H=H, grp=grp, L=L, n=32, bits=int(rng.choice([3, 4])), seed=k, pad=int(rng.integers(0, 4)), dtype=dtype)
        need = c.workspace()[1]
        buf = torch.full((need + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        print(k, d, H, grp, L, rows, dtype, need, flush=True)
        c.call(buf[:max(need, 16)])
        torch.cuda.synchronize()
        assert (buf[max(need, 16):] == 0x5A).all(), (k, need)
        assert int(c.err.item()) == 0 and torch.isfinite(c.out).all()


def test_masks_beside_parents_that_are_none():
    parents = [-1, 0, 5, -7, -1, 0, 1, -1, 0, -1, 0, 1]
    pos, mask, err = i32([77] * 12), torch.full((12, 1), 5, dtype=torch.int64, device="cuda"), i32([0])
    cg.kv_tree_map(i32(parents), i32([0, 2, 4, 7, 12]), i32([10, 12, 13, 15]), pos, mask, err)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE
    assert pos.tolist() == [8, 9, 10, 10, 10, 11, 12, 10, 11, 10, 11, 12]
    assert mask[:, 0].tolist() == [1, 3, 1, 2, 1, 3, 7, 1, 3, 4, 9, 19]


def test_passes_queued_on_two_streams():
    """Four steps of each of two servers, all queued before any is waited for: what they give one after the other."""
    held = (1, 64, 128, 5, 77)
    pairs = [[Step(), Step()], [Step(held=held, window=70, sinks=2), Step(held=held, window=70, sinks=2)]]
    for k, pair in enumerate(pairs):
        for st in pair:
            st.fill(k + 1)
    torch.cuda.synchronize()
    for alone, _ in pairs:
        for _ in range(4):
            alone.run()
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for (_, st), s in zip(pairs, streams):
            with torch.cuda.stream(s):
                st.run()
    torch.cuda.synchronize()
    for alone, beside in pairs:
        assert int(alone.err.item()) == 0 and int(beside.err.item()) == 0
        for x, y in zip(alone.state(), beside.state()):
            assert torch.equal(x, y)
