"""What the norm and the dense layers hold for their gradients, as torch's saved-tensor hooks see it (GPU)."""
import pytest

from test_network_gpu import _gen, _randn

pytestmark = pytest.mark.gpu

CASES = [("linear", "silu", None), ("linear", "gelu", "8bit"), ("linear", None, "8bit"), ("linear", None, None), ("rms_norm", None, None), ("rms_norm", "residual", None)]


def _case(ndvm, op, act, keep, rows, k, n, seed=21):
    """(call, its leaves, cotangents of its results)."""
    g = _gen(seed)
    x, w, b = _randn(g, rows, k).bfloat16(), (_randn(g, n, k) * k ** -0.5).bfloat16(), _randn(g, n)
    if op == "linear":
        leaves, call = (x, w, b), lambda x, w, b: (ndvm.linear(x, w, b, act, keep=keep),)
        ds = (_randn(g, rows, n).bfloat16(),)
    else:
        scale = _randn(g, k)
        leaves = (x, scale, _randn(g, rows, k).bfloat16()) if act else (x, scale)
        call = (lambda x, s, r: ndvm.rms_norm(x, s, 1e-6, r)) if act else (lambda x, s: (ndvm.rms_norm(x, s),))
        ds = tuple(_randn(g, rows, k).bfloat16() for _ in range(2 if act else 1))
    return call, [t.requires_grad_(True) for t in leaves], ds


def _grads(call, leaves, ds):
    import torch
    return torch.autograd.grad(call(*leaves), leaves, ds)


@pytest.mark.parametrize("op,act,keep", CASES)
def test_what_is_held_is_freed_by_checkpoints_and_moved_by_hooks(ndvm, cuda, op, act, keep):
    """After a checkpointed forward pass, and after one whose saved tensors go to the host, no more is allocated than the results:
    neither z (4 bytes an element of y), nor blocks, nor the norm's deviations (4 bytes a row, here 1/4 of a result)."""
    import torch
    from torch.utils.checkpoint import checkpoint
    rows, k, n = (1 << 20, 8, 8) if op == "rms_norm" else (4096, 1024, 2048)
    call, leaves, ds = _case(ndvm, op, act, keep, rows, k, n)
    want = _grads(call, leaves, ds)
    torch.cuda.synchronize()
    base = torch.cuda.memory_allocated()
    results = sum(d.numel() * 2 for d in ds)
    y = checkpoint(call, *leaves, use_reentrant=False)
    assert torch.cuda.memory_allocated() - base <= results + 4096
    got = torch.autograd.grad(y, leaves, ds)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del y, got
    with torch.autograd.graph.save_on_cpu():
        y = call(*leaves)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - base <= results + 4096
    got = torch.autograd.grad(y, leaves, ds)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("op,act,keep", CASES)
def test_hooks_may_give_back_other_memory(ndvm, cuda, op, act, keep):
    """Off 16 bytes, strided or transposed: the same bits.  Of another type or shape: refused before it is read."""
    import torch
    call, leaves, ds = _case(ndvm, op, act, keep, 70, 136, 200)
    want = _grads(call, leaves, ds)

    def off(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
        flat[1:].copy_(t.reshape(-1))
        return flat[1:].view(t.shape)

    def gaps(t):
        wide = torch.empty(*t.shape[:-1], 2 * t.shape[-1] + 3, dtype=t.dtype, device=t.device)
        wide[..., 1:2 * t.shape[-1] + 1:2].copy_(t)
        return wide[..., 1:2 * t.shape[-1] + 1:2]

    def turned(t):
        return t.transpose(0, -1).contiguous().transpose(0, -1)

    for change in (off, gaps, turned):
        packed = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: (packed.append(t.shape), change(t.detach()))[1], lambda t: t):
            y = call(*leaves)
        got = torch.autograd.grad(y, leaves, ds)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), change.__name__
        held = {("linear", None): 2 + bool(act), ("linear", "8bit"): 3 + 2 * bool(act)}.get((op, keep), 3)
        assert len(packed) == held
    for index in range(held):
        for change in (lambda t: t.double(), lambda t: t[..., :-1], lambda t: t.cpu(), lambda t: t[None]):
            count = [0]

            def unpack(t):
                count[0] += 1
                return change(t) if count[0] == index + 1 else t

            with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach(), unpack):
                y = call(*leaves)
            with pytest.raises(ndvm.NdvmError, match="hook"):
                torch.autograd.grad(y, leaves, ds)
            assert count[0] > index
    ndvm.check_operators()


def test_no_cotangent_is_no_gradient(ndvm, cuda):
    """A node that is called without one (what read its result had no gradient for it) returns none, or zeros."""
    import torch

    class Nothing(torch.autograd.Function):
        @staticmethod
        def forward(ctx, *ts):
            return ts[0].sum()

        @staticmethod
        def backward(ctx, d):
            return (None,) * 2

    for op, act, keep in CASES:
        call, leaves, _ = _case(ndvm, op, act, keep, 20, 24, 40)
        y = call(*leaves)
        got = torch.autograd.grad(Nothing.apply(y[0], y[-1]), leaves, allow_unused=True)
        assert all(v is None or not v.any() for v in got), op


def test_what_no_gradient_needs_is_not_held(ndvm, cuda):
    """w is held for x's gradient alone, x for w's, the norm's weight for x's and the residual's: a leaf that none of the wanted
    gradients needs may be written to between the passes."""
    import itertools

    import torch
    needs = {"linear": {0: (1,), 1: (0,), 2: (), 3: ()}, "rms_norm": {0: (0, 1), 1: (0,), 2: (0, 1)}}  # (what x's, w's, ... gradients read)
    for op, act, keep in CASES:
        for wanted in itertools.product((False, True), repeat=3 if op == "linear" or act else 2):
            if not any(wanted):
                continue
            call, leaves, ds = _case(ndvm, op, act, keep, 70, 136, 200)
            leaves = [t.detach().clone().requires_grad_(w) for t, w in zip(leaves, wanted)]
            inputs = [t for t in leaves if t.requires_grad]
            want = _grads(lambda *ts: call(*leaves), inputs, ds)
            read = set().union(*(needs[op][i] for i, w in enumerate(wanted) if w))
            if op == "rms_norm" and act:  # (the stream is the call's own sum)
                read.discard(0)
            if keep:  # (x is held as blocks)
                read.discard(0)
            for i, t in enumerate(leaves):
                y = call(*leaves)
                before = t.detach().clone()
                with torch.no_grad():
                    t.mul_(2)
                if i in read:
                    with pytest.raises(RuntimeError, match="inplace"):
                        torch.autograd.grad(y, inputs, ds)
                else:
                    got = torch.autograd.grad(y, inputs, ds)
                    assert all(torch.equal(a, b) for a, b in zip(got, want)), (op, act, keep, wanted, i)
                with torch.no_grad():
                    t.copy_(before)
    ndvm.check_operators()
