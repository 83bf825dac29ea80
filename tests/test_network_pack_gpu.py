"""Operands that the gated projection copies before it reads them by tiles (GPU): the copies hold what the caller gave
and nothing of what lies around it."""
import pytest

from test_network_gpu import _gated64, _gated_case, _inside, _rounded, _strided

pytestmark = pytest.mark.gpu

AROUND = 7.0  # what _strided leaves between the rows


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", [(2, 1, 3), (3, 7, 5), (6, 9, 17), (40, 64, 72), (65, 333, 130), (300, 136, 50)])
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 1), (6, 3), (9, 8), (15, 7)])
def test_copies_hold_nothing_from_around_the_rows(ndvm, cuda, rows, k, n, pad, shift, t):
    """The workspace of a forward call is the three copies: none of the values between the operands' rows is in it,
    and h has the bits of contiguous operands'."""
    import torch
    x, wg, wu, dh = (v.clamp(-6, 6) for v in _gated_case(rows + k + n, rows, k, n, t))
    xs, gs, us = (_strided(v, pad, shift) for v in (x, wg, wu))
    ws = torch.zeros(ndvm.load().ndvm_gated_workspace_bytes(rows, k, n, 0, 0) // 2, device="cuda", dtype=x.dtype)
    h = ndvm.gated_forward(xs, gs, us, workspace=ws.view(torch.uint8))
    assert not bool((ws == AROUND).any())
    copied = (k + pad) % 8 or shift % 8  # (rows that start on 16 bytes are read where they lie)
    assert int((ws != 0).sum()) == (sum(int((v != 0).sum()) for v in (x, wg, wu)) if copied else 0)
    want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), "silu", t)
    got = (h,) + ndvm.gated_backward(_strided(dh, pad, shift), xs, gs, us)
    for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), got, want, err):
        _inside(a, v, _rounded(v, e, t), name)
    assert torch.equal(h, ndvm.gated_forward(x, wg, wu))
