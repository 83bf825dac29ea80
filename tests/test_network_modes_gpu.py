"""What the differentiable network operators do under torch's other ways of running a program (GPU): a mode in which
a launch of theirs would silently be lost is refused."""
import pytest

pytestmark = pytest.mark.gpu


def _ops(ndvm):
    """(name, call, its tensors): every operator with every tensor argument that it takes."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()

    x, r, w, b = randn(12, 24), randn(12, 24), randn(24), randn(24)
    return [("layer_norm", ndvm.layer_norm, (x, w, b)), ("gated", ndvm.gated, (x, randn(40, 24), randn(40, 24))),
            ("dropout", lambda x, r: ndvm.dropout(x, 0.25, 3, 8, r), (x, r))]


@pytest.mark.parametrize("requires_grad", [False, True])
def test_forward_mode_tangents_are_refused(ndvm, cuda, requires_grad):
    """An input with a tangent (of any argument) raises: an output without one would say that the derivative is 0."""
    import torch
    from torch.autograd import forward_ad
    for name, call, args in _ops(ndvm):
        args = [a.clone().requires_grad_(requires_grad) for a in args]
        want = call(*args)
        with forward_ad.dual_level():
            for i in range(len(args)):
                duals = list(args)
                duals[i] = forward_ad.make_dual(args[i], torch.ones_like(args[i]))
                with pytest.raises(ndvm.NdvmError, match="forward-mode"):
                    call(*duals)
                    pytest.fail(f"{name}: argument {i} was not refused")
            assert torch.equal(call(*args), want)  # (a level alone changes nothing)


def test_forward_mode_through_the_backward_pass_is_refused(ndvm, cuda):
    """A cotangent with a tangent (forward over reverse) raises too."""
    import torch
    from torch.autograd import forward_ad
    for name, call, args in _ops(ndvm):
        args = [a.clone().requires_grad_(True) for a in args]
        y = call(*args)
        with forward_ad.dual_level():
            dy = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
            with pytest.raises(ndvm.NdvmError, match="forward-mode"):
                torch.autograd.grad(y, args[0], dy)
                pytest.fail(name)


def test_functional_jvp_raises(ndvm, cuda):
    import torch
    for name, call, args in _ops(ndvm):
        with pytest.raises(RuntimeError):
            torch.func.jvp(lambda x: call(x, *args[1:]), (args[0],), (torch.ones_like(args[0]),))
            pytest.fail(name)


def test_traces_are_refused(ndvm, cuda):
    """A tracer sees the output's allocation and not the launch that fills it, so its program would return memory that
    nothing wrote: the differentiable ops and the raw calls raise under one."""
    import torch
    from torch.fx.experimental.proxy_tensor import make_fx
    raw = [("layer_norm_forward", lambda x, w, b: ndvm.layer_norm_forward(x, w, b)[0], _ops(ndvm)[0][2]),
           ("gated_forward", ndvm.gated_forward, _ops(ndvm)[1][2]),
           ("dropout_forward", lambda x, r: ndvm.dropout_forward(x, 0.25, 3, 8, r), _ops(ndvm)[2][2])]
    for name, op, args in _ops(ndvm) + raw:
        call = (lambda x, r: op(x, r)) if len(args) == 2 else (lambda x, a, b: op(x, a, b))  # (make_fx counts arguments)
        want = call(*args)
        for tracer in (lambda: torch.jit.trace(call, args, check_trace=False), lambda: make_fx(call)(*args),
                       lambda: make_fx(call, pre_dispatch=True)(*args)):
            with pytest.raises(ndvm.NdvmError, match="trace"):
                tracer()
                pytest.fail(f"{name} was traced")
        assert torch.equal(call(*args), want)


def test_traces_of_a_backward_pass_are_refused(ndvm, cuda):
    """Also where the forward pass ran before the tracer came."""
    import torch
    from torch.fx.experimental.proxy_tensor import make_fx
    for name, call, args in _ops(ndvm):
        args = [a.clone().requires_grad_(True) for a in args]
        y = call(*args)
        dy = torch.ones_like(y)

        def back(dy):
            return torch.autograd.grad(y, args[:1], dy, retain_graph=True)[0]

        want = back(dy)
        with pytest.raises(ndvm.NdvmError, match="trace"):
            make_fx(back)(dy)
            pytest.fail(name)
        assert torch.equal(back(dy), want)
