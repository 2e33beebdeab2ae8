"""Sizes of microscaled calls: those that no call takes are refused before rows of them are allocated,
and workspaces grow as the header says (CPU)."""
import numpy as np
import pytest


@pytest.mark.parametrize("K,P", [(65537, 1), (0, 1), (-1, 5), (4, -1), (1, (1 << 34) + 1), (65536, 1 << 34),
                                 (32, 1 << 34), (65536, (1 << 23) - 100), (1 << 40, 1 << 40)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_rows_of_sizes_that_no_call_takes(K, P, fmt):
    import paper_2007_06134_amd as A
    with pytest.raises(ValueError, match="must be"):
        A.MxRows.empty(K, P, fmt, device="cpu")       # (before the CPU would be refused, or run out of memory)


def test_the_products_workspace_grows_as_stated():
    import paper_2007_06134_amd as A
    rng = np.random.default_rng(1)
    for _ in range(20_000):
        K, P, T = int(rng.integers(1, 257)), int(2 ** rng.uniform(0, 34)), int(2 ** rng.uniform(0, 24))
        n = A._native.lib.adpsgd_mx_product_workspace(K, P, T)
        assert 4 * T * K * K < n <= 16e6 + P * K * K / 4096 + 4 * T * K * K
