"""The network operators stay inside the workspace that they ask for (GPU; what lies behind it is part of the test's tensor)."""
import pytest

from test_network_gpu import _gated64, _gated_case, _gen, _inside, _norm64, _randn, _rounded, _strided, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1000, 8193), (100, 16384), (70, 20001), (63, 9000), (1000, 8192), (2000, 4097)])
def test_layer_norm_backward_within_its_workspace(ndvm, cuda, rows, cols, t):
    import torch
    g = _gen(rows + cols)
    x, dy = _randn(g, rows, cols).to(_t(t)), _randn(g, rows, cols).to(_t(t))
    w, b = _randn(g, cols).to(_t(t)), _randn(g, cols).to(_t(t))
    _, stats = ndvm.layer_norm_forward(x, w, b)
    need = ndvm.load().ndvm_layer_norm_workspace_bytes(rows, cols) // 4
    room = torch.full((need + 4 * cols,), 3.0, device="cuda")
    got = ndvm.layer_norm_backward(dy, x, w, stats, workspace=room[:need])
    assert bool((room[need:] == 3).all())
    want, err = _norm64(x.double(), w.double(), b.double(), dy.double(), 1e-5)
    for name, a, v, e in zip(("dx", "dweight", "dbias"), got, want[1:], err[1:]):
        _inside(a, v, _rounded(v, e, t), name)


@pytest.mark.parametrize("rows,k,n", [(1, 40, 1001), (3, 7, 5), (65, 333, 130), (300, 136, 50), (700, 264, 520), (5000, 16, 24)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
@pytest.mark.parametrize("keep", [False, True])
def test_gated_within_its_workspace(ndvm, cuda, rows, k, n, pad, shift, keep):
    import torch
    plain = _gated_case(rows + k + n, rows, k, n, "bf16")
    x, wg, wu, dh = (_strided(v, pad, shift) for v in plain)
    size = ndvm.load().ndvm_gated_workspace_bytes
    kept = ndvm.gated_kept(x, wg) if keep else None
    rooms = [torch.full((size(rows, k, n, back, 0) + 65536,), 3, device="cuda", dtype=torch.uint8) for back in (0, 1)]
    needs = [size(rows, k, n, back, 0) for back in (0, 1)]
    h = ndvm.gated_forward(x, wg, wu, kept=kept, workspace=rooms[0][:needs[0]])
    got = (h,) + ndvm.gated_backward(dh, x, wg, wu, kept=kept, workspace=rooms[1][:needs[1]])
    for room, need in zip(rooms, needs):
        assert bool((room[need:] == 3).all())
    want, err = _gated64(*(v.double() for v in plain), "silu", "bf16")
    for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), got, want, err):
        _inside(a, v, _rounded(v, e, "bf16"), name)
