"""attend_tree_workspace_bytes: what a call asks for holds every call of at most its sizes."""
import numpy as np
import pytest

from paper_2607_20538_amd import codec as cg


@pytest.mark.parametrize("d", [64, 80, 128, 256])
def test_no_smaller_call_needs_more(d):
    rng = np.random.default_rng(d)
    for _ in range(400):
        H, grp = int(rng.integers(1, 17)), int(rng.integers(1, 140))
        shp = cg.shape(4, H, d, d)
        big = [int(rng.integers(1, 5)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 10)), int(2 ** rng.uniform(0, 12))]
        small = [int(rng.integers(1, v + 1)) for v in big]
        n = lambda v: cg.attend_tree_workspace_bytes(shp, v[0], v[1], v[2], H * grp, v[3], 64)  # noqa: E731
        assert n(small) <= n(big), (H, grp, small, big)
