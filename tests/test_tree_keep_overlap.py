"""kv_tree_keep writes `held` while other workgroups of the same row read what is kept: buffers that it shares with them are
refused on the host."""
import pytest

from paper_2607_20538_amd import codec as cg

from test_serving_abi import PTR
from test_tree_abi import _keep

B, N = 4, 16


@pytest.mark.parametrize("name,count", [("lens", B), ("kept", B), ("cu", B + 1), ("path", N)])
def test_held_shares_nothing_that_is_read(name, count):
    # (far apart but for `held` and the one named)
    at = dict(path=PTR, kept=2 * PTR, cu=3 * PTR, lens=4 * PTR)
    for first in (0, 1, count - 1, 1 - B):              # held's first element against the other buffer's
        assert _keep(B=B, N=N, held=at[name] + 4 * first, **at) == cg.CG_ERR_ARG, first
