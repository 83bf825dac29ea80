"""The network operators together: a proposer of parameters that trains through the replay (GPU)."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("amortised_fit", os.path.join(ROOT, "examples", "amortised_fit.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_proposer_learns_through_the_replay(ndvm, cuda):
    """150 steps take the loss of unseen lanes to a twentieth of where it started; no fit is better than
    chance has it (eight readings and three parameters leave 5/8 of the noise's variance)."""
    m = _example()
    before, after, at_truth = m.train(lanes=1000, steps=150, say=lambda s: None)
    assert after < before / 20, (before, after)
    assert after > 0.5 * (5 / 8) * m.NOISE ** 2 and 0.8 * m.NOISE ** 2 < at_truth < 1.2 * m.NOISE ** 2


def test_block_gradients_are_those_of_torch_operations(ndvm, cuda):
    """One block and its weights' gradients against the same block of torch operations in 64 bits.  Each
    bfloat16 rounding on the way (normed, h, its cotangent, dG and dU, down's input and output, x: at most
    8 in a chain, 2^-9 in the root mean square each) adds up as squares: 2^-9 sqrt(8) < 6e-3; 2e-2 leaves
    the reductions' cancellations."""
    import torch
    m = _example()
    torch.manual_seed(3)
    block = m.Block(256, 512, 0.25).cuda()
    x = torch.randn(300, 256, device="cuda").bfloat16().requires_grad_(True)
    dy = torch.randn(300, 256, device="cuda").bfloat16()
    names = ["scale", "shift", "gate", "up", "down"]
    got = torch.autograd.grad(block(x, 7, 64), [x] + [getattr(block, n) for n in names], dy)
    keep = ndvm.dropout_forward(torch.ones(300, 256, device="cuda"), 0.25, 7, 64).double()
    leaves = [x.detach().double().requires_grad_(True)] + [getattr(block, n).detach().double().requires_grad_(True) for n in names]
    xd, scale, shift, gate, up, down = leaves
    h = torch.nn.functional.layer_norm(xd, (256,), scale, shift)
    h = torch.nn.functional.silu(h @ gate.t()) * (h @ up.t())
    want = torch.autograd.grad(xd + (h @ down.t()) * keep, leaves, dy.double())
    for n, a, b in zip(["x"] + names, got, want):
        assert a.shape == b.shape
        assert float((a.double() - b).norm() / b.norm()) <= 2e-2, n
