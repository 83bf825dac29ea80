"""Layouts that the differentiable network operators copy before they read them (GPU): whatever a raw call refuses."""
import pytest

pytestmark = pytest.mark.gpu


def _windows(rows, cols, seed):
    """Overlapping rows: row i is elements i .. i + cols - 1 of one series."""
    import torch
    t = torch.randn(rows + cols - 1, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()
    return t.unfold(0, cols, 1)


def test_overlapping_rows_are_copied(ndvm, cuda):
    """Sliding windows as x, residual, weights and cotangents, forward and backward: the bits of a contiguous copy's."""
    import torch
    x, r, dy, dh = _windows(37, 72, 1), _windows(37, 72, 2), _windows(37, 72, 3), _windows(37, 40, 4)
    wg, wu = _windows(40, 72, 5), _windows(40, 72, 6)
    w = torch.linspace(0.5, 1.5, 72, device="cuda")
    calls = [(lambda x, w: ndvm.layer_norm(x, w), (x, w), dy), (ndvm.gated, (x, wg, wu), dh),
             (lambda x, r: ndvm.dropout(x, 0.25, 9, 0, r), (x, r), dy)]
    for call, args, cot in calls:
        plain = [a.detach().contiguous().requires_grad_(True) for a in args]
        want = call(*plain)
        grads = torch.autograd.grad(want, plain, cot.contiguous())
        with torch.no_grad():
            assert torch.equal(call(*args), want)
        leaves = [a.detach().requires_grad_(True) for a in args]
        y = call(*leaves)
        assert torch.equal(y, want)
        for a, b in zip(torch.autograd.grad(y, leaves, cot), grads):
            assert torch.equal(a, b)


def test_raw_calls_name_the_overlapping_rows(ndvm, cuda):
    x = _windows(8, 24, 1)
    for call in (lambda: ndvm.layer_norm_forward(x), lambda: ndvm.dropout_forward(x, 0.1, 0), lambda: ndvm.gated_forward(x, x, x),
                 lambda: ndvm.gated_forward(x.contiguous(), x, x.contiguous())):
        with pytest.raises(ndvm.NdvmError, match="rows of contiguous elements"):
            call()


def test_strided_weights_and_biases_are_copied(ndvm, cuda):
    """A column of a matrix and a value that all columns share, as layer norm's weight and bias; their gradients go back
    to where the values came from."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    x, dy = (torch.randn(33, 72, generator=g, device="cuda").requires_grad_(True) for _ in range(2))
    both = torch.randn(72, 3, generator=g, device="cuda").requires_grad_(True)
    one = torch.full((1,), 0.25, device="cuda").requires_grad_(True)
    plain = [both.detach()[:, 1].contiguous().requires_grad_(True), one.detach().expand(72).contiguous().requires_grad_(True)]
    want = ndvm.layer_norm(x, *plain)
    dw, db = torch.autograd.grad(want, plain, dy)
    y = ndvm.layer_norm(x, both[:, 1], one.expand(72))
    assert torch.equal(y, want)
    dboth, done = torch.autograd.grad(y, (both, one), dy)
    assert torch.equal(dboth[:, 1], dw) and not dboth[:, ::2].any() and torch.equal(done, db.sum().view(1))
    with torch.no_grad():
        assert torch.equal(ndvm.layer_norm(x, both[:, 1], one.expand(72)), want)


def test_lazily_negated_views(ndvm, cuda):
    """The imaginary part of a conjugate is a view whose memory holds the opposite sign: copied, or refused by a raw call."""
    import torch
    z = torch.randn(9, 1, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda", dtype=torch.complex64)
    x = z.conj().imag
    assert x.is_neg()
    assert torch.equal(ndvm.dropout(x, 0.0, 1), -z.imag) and torch.equal(ndvm.dropout(-z.imag, 0.0, 1, 0, x), -2 * z.imag)
    one, bias = torch.ones(5, 1, device="cuda"), z[0].conj().imag
    assert torch.equal(ndvm.layer_norm(one, None, bias), (-z[0].imag).expand(5, 1))
    y = torch.ones(9, 1, device="cuda", requires_grad=True)
    assert torch.equal(torch.autograd.grad(ndvm.dropout(y, 0.0, 1), y, x)[0], -z.imag)
    with pytest.raises(ndvm.NdvmError, match="resolve_neg"):
        ndvm.dropout_forward(x, 0.0, 1)
