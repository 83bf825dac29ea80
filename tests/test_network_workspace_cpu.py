"""How much workspace the network operators ask for (no GPU)."""
import pytest


@pytest.mark.parametrize("rows,cols", [(912, 8193), (1000, 1 << 20), (100000, 16384), (64, 50000)])
def test_layer_norm_of_long_rows_asks_for_what_it_uses(ndvm, rows, cols):
    """Rows longer than a block's registers hold (8192 elements) have their column sums from 64 ranges of rows at most:
    two binary32 sums a column and range, not those of six blocks an SM."""
    assert ndvm.load().ndvm_layer_norm_workspace_bytes(rows, cols) == min(rows, 64) * cols * 2 * 4


def test_layer_norm_of_other_rows_keeps_its_workspace(ndvm):
    f = ndvm.load().ndvm_layer_norm_workspace_bytes
    assert f(1 << 20, 8192) == f(912, 8192) == 912 * 8192 * 8 and f(5, 8192) == 5 * 8192 * 8
