"""What the gated projection's differentiable op holds between its passes (GPU)."""
import pytest

from test_network_gpu import _gated_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,k,n", [(300, 1600, 512), (1100, 64, 2048), (40, 72, 136)])
@pytest.mark.parametrize("keep", [None, False, True])
def test_caller_says_what_is_kept(ndvm, cuda, rows, k, n, keep):
    """keep=False holds nothing but the inputs, keep=True the two products; the gradients are those of the raw calls."""
    import torch
    x, wg, wu, dh = _gated_case(rows, rows, k, n, "bf16")
    kept = ndvm.gated_kept(x, wg)
    h = ndvm.gated_forward(x, wg, wu, "gelu", kept=kept)
    want = {w: ndvm.gated_backward(dh, x, wg, wu, "gelu", kept=kept if w else None) for w in (False, True)}
    nbytes, leaves = kept.numel() * 4, [v.requires_grad_(True) for v in (x, wg, wu)]
    before = torch.cuda.memory_allocated()
    y = ndvm.gated(*leaves, "gelu", keep=keep)
    held = torch.cuda.memory_allocated() - before
    by_rule = k >= 1536 or rows * n <= 1 << 21
    holds = by_rule if keep is None else keep
    slack = y.numel() * 2 + 4096
    assert held <= slack if not holds else nbytes <= held <= nbytes + slack + (1 << 21), (held, nbytes)
    assert torch.equal(y.detach(), h)
    for a, b in zip(torch.autograd.grad(y, leaves, dh), want[holds]):
        assert torch.equal(a, b)


def test_keep_without_gradients_holds_nothing(ndvm, cuda):
    import torch
    x, wg, wu, _ = _gated_case(3, 64, 72, 136, "f16")
    assert torch.equal(ndvm.gated(x, wg, wu, keep=True), ndvm.gated_forward(x, wg, wu))
