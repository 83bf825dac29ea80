"""The network operators stay inside the workspace that they ask for (GPU; what lies behind it is part of the test's tensor)."""
import pytest

from test_network_gpu import _gen, _inside, _norm64, _randn, _rounded, _t

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
