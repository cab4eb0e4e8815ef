"""Refusals of the masks under a window, on the host; the masks and the attention's definition against sequential decoding's."""
import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

from test_serving_abi import PTR

import _tree as T
from _tree_window import windowed


def _map(parent=PTR, cu=PTR, lens=PTR, B=2, N=8, words=1, window=4, sinks=1, pos=PTR, mask=PTR, err=None):
    return cg.lib().kv_tree_map_window(parent, cu, lens, B, N, words, window, sinks, pos, mask, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(window=-1), cg.CG_ERR_ARG), (dict(sinks=-1), cg.CG_ERR_ARG), (dict(window=0, sinks=-1), cg.CG_ERR_ARG),
    (dict(parent=None), cg.CG_ERR_ARG), (dict(cu=None), cg.CG_ERR_ARG), (dict(lens=None), cg.CG_ERR_ARG),
    (dict(pos=None), cg.CG_ERR_ARG), (dict(mask=None), cg.CG_ERR_ARG), (dict(B=0), cg.CG_ERR_ARG),
    (dict(N=-1), cg.CG_ERR_ARG), (dict(words=0), cg.CG_ERR_ARG), (dict(mask=PTR + 4), cg.CG_ERR_ALIGN),
    (dict(pos=PTR + 2), cg.CG_ERR_ALIGN), (dict(err=PTR + 2), cg.CG_ERR_ALIGN),
])
def test_tree_map_window_refuses(kw, status):
    assert _map(**kw) == status


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (16, 5), (64, 300), (1000, 0), (7, 12)])
@pytest.mark.parametrize("base", [0, 9, 200])
@pytest.mark.parametrize("kind", ["chain", "near", "forest"])
def test_masks_under_a_window_are_what_sequential_decoding_sees(kind, base, window, sinks):
    """The oracle of the masks: a node sees, of its own path, the positions that a token decoded at its end would see."""
    parents = T.tree(90, kind, np.random.default_rng(base))
    masks, depth = T.closure(parents)
    seen = T.seen_by(windowed(masks, depth, base, window, sinks), [base + k for k in depth], base, window, sinks)
    for i in range(90):
        path, x = [], i
        while x >= 0:
            path.append(x)
            x = parents[x]
        path.reverse()                                 # the row as it would be with this path alone: position base + k is path[k]
        p = base + len(path) - 1
        want = torch.zeros(base + 90, dtype=torch.bool)
        for t in range(p + 1):
            if t > p - window or t < sinks:
                want[t if t < base else base + path[t - base]] = True
        assert torch.equal(seen[i], want)
