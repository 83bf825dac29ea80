"""Which layouts the network operators' raw calls read in place (no GPU)."""
import pytest


def test_rows_that_overlap_are_refused(ndvm):
    import torch
    from paper_2607_03574_gb300.network import _rows
    series = torch.empty(100)
    for bad in (series.unfold(0, 10, 1), series.unfold(0, 10, 9), series.unfold(0, 10, 3).unflatten(0, (1, -1))):
        with pytest.raises(ndvm.NdvmError, match="one row stride"):
            _rows(bad, "x")
    assert _rows(series.unfold(0, 10, 10), "x") == (10, 10, 10) and _rows(series.unfold(0, 10, 12), "x") == (8, 10, 12)
    assert _rows(series[:10].unfold(0, 10, 1), "x") == (1, 10, 10)  # one window: nothing overlaps
    assert _rows(series[:1].expand(5, 1), "x") == (5, 1, 0)
