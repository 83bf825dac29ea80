"""The network operators' autograd nodes (GPU): what is kept for the backward pass, inputs that take no gradient, streams."""
import itertools

import pytest

from test_network_gpu import RMS, _gated64, _gated_case, _inside, _norm64, _randn, _gen, _rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", [(1100, 64, 2048), (4200, 72, 520), (1400, 1600, 1600), (1501, 1537, 1401)])
def test_gated_nodes_of_many_elements(ndvm, cuda, rows, k, n, t):
    """More than 2^21 elements: nothing is kept below a contraction of 1536, G and U are from there on."""
    import torch
    x, wg, wu, dh = _gated_case(rows + k, rows, k, n, t)
    want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), "silu", t)
    leaves = [v.requires_grad_(True) for v in (x, wg, wu)]
    y = ndvm.gated(*leaves)
    for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), (y.detach(),) + torch.autograd.grad(y, leaves, dh), want, err):
        _inside(a, v, _rounded(v, e, t), name)
        assert float((a.double() - v).norm() / v.norm()) <= 3 * RMS[t], name


@pytest.mark.parametrize("wants", [w for w in itertools.product([False, True], repeat=3) if any(w)])
def test_layer_norm_nodes_of_frozen_inputs(ndvm, cuda, wants):
    """Any of x, weight and bias may take no gradient, or be absent: the others' have the bits of the whole."""
    import torch
    g = _gen(8)
    args, dy = [_randn(g, 30, 72), _randn(g, 72), _randn(g, 72)], _randn(g, 30, 72)
    full = [a.clone().requires_grad_(True) for a in args]
    want = torch.autograd.grad(ndvm.layer_norm(*full), full, dy)
    some = [a.clone().requires_grad_(w) for a, w in zip(args, wants)]
    got = torch.autograd.grad(ndvm.layer_norm(*some), [a for a, w in zip(some, wants) if w], dy)
    for a, b in zip(got, [v for v, w in zip(want, wants) if w]):
        assert torch.equal(a, b)
    if wants[2]:  # a bias without a weight
        bias_only = args[2].clone().requires_grad_(True)
        x = args[0].clone().requires_grad_(wants[0])
        grads = torch.autograd.grad(ndvm.layer_norm(x, None, bias_only), [x, bias_only] if wants[0] else [bias_only], dy)
        assert torch.equal(grads[-1], want[2])
        if wants[0]:
            exact, err = _norm64(args[0].double(), torch.ones_like(args[1]).double(), args[2].double(), dy.double(), 1e-5)
            _inside(grads[0], exact[1], _rounded(exact[1], err[1], "f32"), "dx")


@pytest.mark.parametrize("wants", [w for w in itertools.product([False, True], repeat=3) if any(w)])
@pytest.mark.parametrize("rows", [5, 300])
def test_gated_nodes_of_frozen_inputs(ndvm, cuda, wants, rows):
    import torch
    *args, dh = _gated_case(9, rows, 72, 136, "bf16")
    full = [a.clone().requires_grad_(True) for a in args]
    want = torch.autograd.grad(ndvm.gated(*full), full, dh)
    some = [a.clone().requires_grad_(w) for a, w in zip(args, wants)]
    got = torch.autograd.grad(ndvm.gated(*some), [a for a, w in zip(some, wants) if w], dh)
    for a, b in zip(got, [v for v, w in zip(want, wants) if w]):
        assert torch.equal(a, b)


def test_dropout_nodes_of_frozen_inputs(ndvm, cuda):
    import torch
    g = _gen(10)
    x, r, dy = _randn(g, 9, 40), _randn(g, 9, 40), _randn(g, 9, 40)
    xr, rr = x.clone().requires_grad_(True), r.clone().requires_grad_(True)
    want = ndvm.dropout_backward(dy, 0.5, 4, 8)
    assert torch.equal(torch.autograd.grad(ndvm.dropout(xr, 0.5, 4, 8, r), xr, dy)[0], want)
    assert torch.equal(torch.autograd.grad(ndvm.dropout(x, 0.5, 4, 8, rr), rr, dy)[0], dy)


def test_backward_on_the_stream_of_the_forward_pass(ndvm, cuda):
    """Forward on a side stream that is still busy: autograd runs the backward pass there, behind it."""
    import torch
    side = torch.cuda.Stream()
    x, wg, wu, dh = _gated_case(52, 300, 264, 520, "bf16")
    w = torch.ones(264, device="cuda", dtype=torch.bfloat16)

    def step(x, w, wg, wu, dh):
        leaves = [v.detach().requires_grad_(True) for v in (x, w, wg, wu)]
        y = ndvm.dropout(ndvm.gated(ndvm.layer_norm(leaves[0], leaves[1]), leaves[2], leaves[3]), 0.2, 3)
        return torch.autograd.grad(y, leaves, dh)

    want = step(x, w, wg, wu, dh)
    late = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        spin = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            spin = spin @ spin * 1e-3
        late.copy_(x)
        got = step(late, w, wg, wu, dh)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_gated_has_no_second_derivative(ndvm, cuda):
    import torch
    x, wg, wu, dh = _gated_case(61, 9, 24, 40, "bf16")
    x.requires_grad_(True)
    with pytest.raises(ndvm.NdvmError):
        torch.autograd.grad(ndvm.gated(x, wg, wu), x, dh, create_graph=True)
