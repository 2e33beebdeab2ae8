"""Sizes that no microscaled call takes are refused before rows of them are allocated (CPU)."""
import pytest


@pytest.mark.parametrize("K,P", [(65537, 1), (0, 1), (-1, 5), (4, -1), (1, (1 << 34) + 1), (65536, 1 << 34),
                                 (32, 1 << 34), (65536, (1 << 23) - 100), (1 << 40, 1 << 40)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_rows_of_sizes_that_no_call_takes(K, P, fmt):
    import paper_2007_06134_amd as A
    with pytest.raises(ValueError, match="must be"):
        A.MxRows.empty(K, P, fmt, device="cpu")       # (before the CPU would be refused, or run out of memory)
