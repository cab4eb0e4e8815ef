"""Trees deeper than the attention's window: the masks of kv_tree_map with a window, and the step against sequential decoding."""
import math

import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

import _serving as S
import _tree as T
from _tree_window import windowed
from test_gpu_chunk import Case
from test_gpu_tree import KINDS, SIZES, Step, i32, packed
from test_gpu_tree_attend import Tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cg.lib()


@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 3), (16, 0), (50, 120), (64, 1), (65, 10 ** 9), (300, 40), (2 ** 31 - 1, 0), (0, 7)])
def test_masks_under_a_window(sizes, window, sinks):
    rng = np.random.default_rng(window % 1000 + sinks % 1000)
    trees, cu, parents = packed(sizes, KINDS[1:] + KINDS[:1], rng)
    words = max(1, -(-max(sizes) // 64)) + 1
    N = cu[-1] + 3
    held = [int(h) for h in rng.choice([0, 1, 17, 90, 100000], len(sizes))]
    pos, mask = torch.full((N,), 77, dtype=torch.int32, device="cuda"), torch.full((N, words), 5, dtype=torch.int64, device="cuda")
    err = i32([0])
    cg.kv_tree_map(i32(parents + [9] * 3), i32(cu), i32([h + n for h, n in zip(held, sizes)]), pos, mask, err, window=window, sinks=sinks)
    torch.cuda.synchronize()
    want_pos, want = [], []
    for h, t in zip(held, trees):
        m, depth = T.closure(t)
        want_pos += [h + k for k in depth]
        want += windowed(m, depth, h, window, sinks)
    assert int(err.item()) == 0
    assert pos.tolist() == want_pos + [-1] * 3
    assert np.array_equal(mask.cpu().numpy(), np.concatenate([T.words_of(want, words), np.zeros((3, words), np.int64)]))


def test_masks_of_a_row_that_is_shorter_than_its_trees():
    pos, mask, err = i32([7] * 5), torch.full((5, 1), 5, dtype=torch.int64, device="cuda"), i32([0])
    cg.kv_tree_map(i32([-1, 0, 1, 2, 3]), i32([0, 5]), i32([4]), pos, mask, err, window=2, sinks=1)
    torch.cuda.synchronize()
    assert int(err.item()) == cg.CG_FLAG_POS_RANGE and pos.tolist() == [-1] * 5
    assert mask[:, 0].tolist() == [0b1, 0b11, 0b111, 0b1101, 0b11001]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (50, 3), (20, 310)])
def test_chains_behind_a_window_give_what_the_chunk_attention_gives(window, sinks, dtype):
    """Chains up to 100 nodes long, masks from the GPU: the attention of packed tokens in a row, under the same window."""
    rows = [(300, 100), (64, 1), (5, 57), (0, 70)]
    a, b = (K(rows, window=window, sinks=sinks, dtype=dtype, H=1, **kw) for K, kw in ((Tree, dict(kind="chain")), (Case, {})))
    parents = [i - 1 for _, n in rows for i in range(n)] + [-1] * (a.N - int(a.first[-1]))
    cg.kv_tree_map(i32(parents), a.cu, a.lens, a.pos, a.mask, a.err, window=window, sinks=sinks)
    a.call()
    b.call()
    torch.cuda.synchronize()
    assert int(a.err.item()) == 0
    # the nodes' sight as the masks have it, for the bound of either side's error
    for k, ((held, n), m) in enumerate(zip(rows, a.masks)):
        depth = list(range(n))
        a.seen[k] = T.seen_by(windowed(m, depth, held, window, sinks), [held + i for i in depth], held, window, sinks)
    want, bound = a.ref()
    used = int(a.first[-1])
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for t in (a, b):
        err = (t.out[:, 0].double().cpu() - want)[:, :, :used].norm(dim=-1)
        assert (err <= (bound + step * want.norm(dim=-1))[:, :, :used]).all()


class Windowed(Step):
    """The step with masks under its window."""

    def fill(self, seed):
        super().fill(seed)
        self.trees[3] = [i - 1 for i in range(33)]     # a chain: the drafts agree with the model's choices down most of it
        self.parent.copy_(i32(sum(self.trees, []) + [0] * 4))
        a = self.first[3]
        for i in range(30):
            self.hd[a + i + 1] = self.ht[a + i]
        self.draft.copy_(i32(self.hd))

    def run(self):
        saved = cg.kv_tree_map
        try:
            cg.kv_tree_map = lambda *a: saved(*a, window=self.window, sinks=self.sinks)
            super().run()
        finally:
            cg.kv_tree_map = saved


@pytest.mark.parametrize("window,sinks", [(1, 0), (4, 2), (10, 0), (20, 110)])
def test_a_step_under_a_short_window_keeps_what_sequential_decoding_would(window, sinks):
    """Three steps whose kept paths are longer than the window: every kept node's result is that of the chunk attention over pools
    filled with the kept tokens alone."""
    st, ref = Windowed(window=window, sinks=sinks), Windowed(window=window, sinks=sinks)
    for step in range(3):
        st.fill(step)
        before = st.lens.tolist()
        st.run()
        torch.cuda.synchronize()
        assert int(st.err.item()) == 0
        ways = [T.walk(t, st.hd[a:], st.ht[a:])[0] for t, a in zip(st.trees, st.first)]
        assert len(ways[3]) > 30 and st.lens.tolist() == [h + len(w) for h, w in zip(before, ways)]
        idx = [a + i for w, a in zip(ways, st.first) for i in w]
        N = len(idx)
        pos, slots, cu = i32([0] * N), i32([0] * N), i32([0] * 6)
        cg.kv_page_map(ref.lens, i32([len(w) for w in ways]), ref.pool, ref.pages, 64, cu, ref.lens, pos, slots, ref.err)
        take = lambda t: t[:, :, :, idx].contiguous()  # noqa: E731
        q = take(st.q)
        cg.kv_append_rope(0, 1, st.plan, take(st.k), take(st.v), pos, slots, st.Gd, st.shp, st.codec, *ref.dev, q, q, ref.err)
        out = torch.empty_like(q)
        cg.kv_attend_chunk_paged(0, 1, q, cu, 33, *ref.dev, cg.page_table(ref.pages, 64), st.Gd, st.shp, st.codec, ref.lens,
                                 1 / math.sqrt(128), out, window, sinks,
                                 torch.zeros(max(16, cg.attend_chunk_workspace_limit(st.shp, 1, N, 5, 4, 8, 64)), dtype=torch.uint8, device="cuda"),
                                 ref.err)
        torch.cuda.synchronize()
        assert int(ref.err.item()) == 0 and torch.equal(q, st.qo[:, :, :, idx])
        # bf16 results of either kernel: each within one rounding and the operands' 11 bits of the same number
        got, want = st.out[:, :, :, idx].float(), out.float()
        assert (got - want).norm(dim=-1).max() <= 4 * 2.0 ** -8 * want.norm(dim=-1).max()
