"""RMS norm, dense layers and 8-bit blocks under torch's other ways of running a program, in graphs, on other streams and in
threads (GPU)."""
import threading

import pytest

from test_network_gpu import _gen, _randn

pytestmark = pytest.mark.gpu


def _ops(ndvm):
    """(name, call, its tensors): every operator with every tensor argument that it takes."""
    g = _gen(5)
    x, r, w, b, m = (_randn(g, *s).bfloat16() for s in ((12, 24), (12, 24), (24,), (40,), (40, 24)))
    res = _randn(g, 12, 40).bfloat16()
    return [("rms_norm", lambda x, w, r: ndvm.rms_norm(x, w, 1e-6, r), (x, w, r)),
            ("linear", lambda x, m, b, r: ndvm.linear(x, m, b, "silu", r), (x, m, b, res)),
            ("linear, 8 bits", lambda x, m, b, r: ndvm.linear(x, m, b, "silu", r, keep="8bit"), (x, m, b, res))]


def _first(y):
    return y[0] if isinstance(y, tuple) else y


def test_forward_mode_tangents_are_refused(ndvm, cuda):
    import torch
    from torch.autograd import forward_ad
    for name, call, args in _ops(ndvm):
        for requires_grad in (False, True):
            args = [a.clone().requires_grad_(requires_grad) for a in args]
            with forward_ad.dual_level():
                for i in range(len(args)):
                    duals = list(args)
                    duals[i] = forward_ad.make_dual(args[i], torch.ones_like(args[i]))
                    with pytest.raises(ndvm.NdvmError, match="forward-mode"):
                        call(*duals)
                        pytest.fail(f"{name}: argument {i} was not refused")
    x = _ops(ndvm)[0][2][0]
    with forward_ad.dual_level(), torch.no_grad():
        d = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: ndvm.quantize(d), lambda: ndvm.rms_norm_quantized(d)):
            if forward_ad.unpack_dual(d).tangent is not None:
                with pytest.raises(ndvm.NdvmError, match="forward-mode"):
                    with torch.enable_grad():
                        call()


def test_second_derivatives_jvp_and_traces_are_refused(ndvm, cuda):
    import torch
    from torch.fx.experimental.proxy_tensor import make_fx
    for name, call, args in _ops(ndvm):
        plain = [a.clone() for a in args]
        args = [a.clone().requires_grad_(True) for a in args]
        y = _first(call(*args))
        with pytest.raises(ndvm.NdvmError, match="second"):
            torch.autograd.grad(y, args[0], torch.ones_like(y), create_graph=True)
        with pytest.raises(RuntimeError):
            torch.func.jvp(lambda x: _first(call(x, *plain[1:])), (plain[0],), (torch.ones_like(plain[0]),))
        three = (lambda x, a, b: _first(call(x, a, b))) if len(args) == 3 else (lambda x, a, b, c: _first(call(x, a, b, c)))
        for tracer in (lambda: torch.jit.trace(three, tuple(plain), check_trace=False), lambda: make_fx(three)(*plain)):
            with pytest.raises(ndvm.NdvmError, match="trace"):
                tracer()
                pytest.fail(name)
        y = _first(call(*args))
        with pytest.raises(ndvm.NdvmError, match="trace"):
            make_fx(lambda d: torch.autograd.grad(y, args[:1], d, retain_graph=True)[0])(torch.ones_like(y))
    x = args[0].detach()
    with torch.no_grad():
        for call in (lambda x: ndvm.quantize(x).values, lambda x: ndvm.rms_norm_quantized(x).values):
            with pytest.raises(ndvm.NdvmError, match="trace"):
                make_fx(call)(x)


def test_a_graph_runs_backward_once_unless_it_is_kept(ndvm, cuda):
    """A second backward pass over a freed graph, and one over inputs that were written to, raise torch's errors."""
    import torch
    for name, call, args in _ops(ndvm):
        args = [a.clone().requires_grad_(True) for a in args]
        y = _first(call(*args))
        d = torch.ones_like(y)
        a = torch.autograd.grad(y, args, d, retain_graph=True)
        b = torch.autograd.grad(y, args, d)
        assert all(torch.equal(p, q) for p, q in zip(a, b)), name
        with pytest.raises(RuntimeError, match="second time"):
            torch.autograd.grad(y, args, d)
        y = _first(call(*args))
        with torch.no_grad():
            args[1].add_(1)
        with pytest.raises(RuntimeError, match="inplace"):
            torch.autograd.grad(y, args, d)
    x, w, r = _ops(ndvm)[0][2]
    x.requires_grad_(True)
    y, s = ndvm.rms_norm(x, w, 1e-6, r)
    s.detach().add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        torch.autograd.grad(y.sum(), x)


def test_hooks_accumulation_and_checkpoints(ndvm, cuda):
    """Gradients add up in .grad, pass through hooks, and are those of a recomputed forward pass."""
    import torch
    from torch.utils.checkpoint import checkpoint
    for name, call, args in _ops(ndvm):
        args = [a.clone().requires_grad_(True) for a in args]
        y = _first(call(*args))
        d = torch.ones_like(y)
        want = torch.autograd.grad(y, args, d)
        seen = []
        args[0].register_hook(lambda g: seen.append(g.clone()))
        for _ in range(2):
            _first(call(*args)).backward(d)
        assert all(torch.equal(a.grad, g + g) for a, g in zip(args, want)), name
        assert len(seen) == 2 and torch.equal(seen[0], want[0])
        again = torch.autograd.grad(_first(checkpoint(call, *args, use_reentrant=False)), args, d)
        assert all(torch.equal(a, b) for a, b in zip(want, again)), name


def test_graphs_streams_and_threads_give_the_same_bits(ndvm, cuda):
    """Two captured graphs (scoring, and a training step) replayed on new inputs while eager calls run; another stream; four threads
    at once."""
    import torch
    g = _gen(9)
    x, r, scale = _randn(g, 300, 256).bfloat16(), _randn(g, 300, 256).bfloat16(), _randn(g, 256).bfloat16()
    up, b, down = (_randn(g, 512, 256) / 16).bfloat16(), _randn(g, 512), (_randn(g, 256, 512) / 22).bfloat16()
    qu, qd = ndvm.quantize(up), ndvm.quantize(down)
    leaves = [t.requires_grad_(True) for t in (scale, up, b, down)]
    dy = _randn(g, 300, 256).bfloat16()

    @torch.no_grad()
    def score(x, r):
        h, s = ndvm.rms_norm_quantized(x, scale, 1e-6, r)
        return ndvm.linear_quantized(ndvm.quantize(ndvm.linear_quantized(h, qu, b, "gelu")), qd, None, None, s)

    def step(x, r, keep=None):
        h, s = ndvm.rms_norm(x, scale, 1e-6, r)
        y = ndvm.linear(ndvm.linear(h, up, b, "silu", keep=keep), down, None, None, s, keep=keep)
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    def run(x, r):
        return [score(x, r), *step(x, r), *step(x, r, "8bit")]

    want = run(x, r)
    inputs = [torch.zeros_like(x), torch.zeros_like(r)]
    run(*inputs)
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0], stream=side):
        scored = score(*inputs)
    with torch.cuda.graph(graphs[1], stream=side):
        trained = [*step(*inputs), *step(*inputs, "8bit")]
    inputs[0].copy_(x), inputs[1].copy_(r)
    for _ in range(3):
        graphs[0].replay(), graphs[1].replay()
        eager = run(x, r)
        assert all(torch.equal(a, c) for a, c in zip([scored, *trained], want)) and all(torch.equal(a, c) for a, c in zip(eager, want))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run(x, r)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(other, want))
    found, streams = [None] * 4, [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(5):
                found[i] = run(x, r)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads], [t.join() for t in threads]
    torch.cuda.synchronize()
    assert all(f is not None and all(torch.equal(a, c) for a, c in zip(f, want)) for f in found)
    ndvm.check_operators()


def test_raw_calls_on_a_given_stream(ndvm, cuda):
    """Outputs and workspaces that a raw call allocates belong to its stream."""
    import torch
    g = _gen(10)
    x, w, dy = _randn(g, 200, 72).bfloat16(), _randn(g, 136, 72).bfloat16(), _randn(g, 200, 136).bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for s in (None, side):
        y, _, rstd = ndvm.rms_norm_forward(x, stream=s)
        kept = ndvm.linear_kept(y, w, stream=s)
        z = ndvm.linear_forward(y, w, None, "gelu", kept=kept, stream=s)
        back = ndvm.linear_backward(dy, y, w, "gelu", kept=kept, stream=s)
        dx, dw = ndvm.rms_norm_backward(back[0], x, None, rstd, stream=s)
        q = ndvm.quantize_forward(z, stream=s)
        p = ndvm.rms_norm_quantized_forward(x, stream=s)[0]
        got.append([z, *back, dx, dw, q.dequantize(stream=s), ndvm.linear_quantized_forward(p, ndvm.quantize_forward(w, stream=s), stream=s)])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_arguments_are_refused_with_their_reason(ndvm, cuda):
    import torch
    x, w, b = torch.ones(4, 32, device="cuda").bfloat16(), torch.ones(8, 32, device="cuda").bfloat16(), torch.ones(8, device="cuda").bfloat16()
    v = torch.ones(32, device="cuda").bfloat16()
    q = ndvm.quantize(x)
    wrong = [
        (lambda: ndvm.rms_norm(x, b), "weight"), (lambda: ndvm.rms_norm(x, v, 1e-6, x[:2]), "residual"), (lambda: ndvm.rms_norm(x, v, -1.0), "eps"),
        (lambda: ndvm.rms_norm(x, v, 1e-6, x.float()), "residual"), (lambda: ndvm.rms_norm(x.double()), "dtype"), (lambda: ndvm.rms_norm(x, v.half()), "weights"),
        (lambda: ndvm.linear(x.float(), w.float()), "dense layers"), (lambda: ndvm.linear(x, w.t()), "matrix"), (lambda: ndvm.linear(x, w.half()), "dtype"),
        (lambda: ndvm.linear(x, w, v), "bias"), (lambda: ndvm.linear(x, w, b.half()), "bias"), (lambda: ndvm.linear(x, w, b, None, x), "residual"),
        (lambda: ndvm.linear(x, w, b.cpu()), "bias"), (lambda: ndvm.linear(x, w.cpu()), "w"),
        (lambda: ndvm.linear(x, w, b, "tanh"), "activation"), (lambda: ndvm.linear(x, w, b, keep="4bit"), "keep"), (lambda: ndvm.quantize(x.double()), "dtype"),
        (lambda: ndvm.linear_quantized(q, x), "Quantized"), (lambda: ndvm.linear_quantized(q, ndvm.quantize(w[:, :16])), "matrix"),
        (lambda: ndvm.linear_quantized(q, ndvm.quantize(w), dtype=torch.float32), "dense layers"), (lambda: ndvm.Quantized(x, q.scales), "float8"),
        (lambda: ndvm.Quantized(q.values[:, :20], q.scales.view(1, 1, 32, 16)), "scales"), (lambda: ndvm.Quantized(q.values[:, 1:], q.scales), "16 bytes"),
        (lambda: ndvm.rms_norm_forward(x, v, sum=x.clone()), "residual"), (lambda: ndvm.linear_backward(b.expand(4, 8), x, w, "silu"), "kept"),
        (lambda: ndvm.linear_forward(x, w, kept=torch.empty(4, 7, device="cuda")), "kept"), (lambda: ndvm.quantize_forward(x, out=ndvm.quantize(w)), "out")]
    for i, (call, reason) in enumerate(wrong):
        with pytest.raises(ndvm.NdvmError, match=reason):
            call()
            pytest.fail(f"call {i} was not refused")


def test_what_is_held_for_the_gradients(ndvm, cuda):
    """Beside its result a dense layer holds z in binary32, or z and x in 33/32 bytes an element each; nothing without an activation;
    and nothing of it outlives the graph."""
    import torch
    rows, k, n = 4096, 1024, 2048
    g = _gen(11)
    x, w, b = _randn(g, rows, k).bfloat16().requires_grad_(True), _randn(g, n, k).bfloat16().requires_grad_(True), _randn(g, n).requires_grad_(True)
    dy = _randn(g, rows, n).bfloat16()
    torch.autograd.grad(ndvm.linear(x, w, b, "silu", keep="8bit"), (x, w, b), dy)
    base = torch.cuda.memory_allocated()
    for act, keep, want in ((None, None, 0), ("silu", None, 4 * rows * n), (None, "8bit", rows * k * 33 // 32), ("gelu", "8bit", rows * (n + k) * 33 // 32)):
        y = ndvm.linear(x, w, b, act, keep=keep)
        assert 0 <= torch.cuda.memory_allocated() - base - 2 * rows * n - want <= 8192, (act, keep)
        torch.autograd.grad(y, (x, w, b), dy)
        assert torch.cuda.memory_allocated() - base <= 2 * rows * n + 8192
        y = ndvm.linear(x, w, b, act, keep=keep)
        del y
        assert torch.cuda.memory_allocated() == base
    y, s = ndvm.rms_norm(x, None, 1e-6, x)
    assert torch.cuda.memory_allocated() - base <= 4 * rows * k + 4 * rows + 1024
    del y, s
    assert torch.cuda.memory_allocated() == base


def test_gradients_of_some_inputs_alone(ndvm, cuda):
    """Whichever inputs want gradients, they get those of all wanting them."""
    import itertools

    import torch
    for name, call, args in _ops(ndvm):
        every = [a.clone().requires_grad_(True) for a in args]
        y = _first(call(*every))
        d = torch.ones_like(y)
        want = torch.autograd.grad(y, every, d)
        for wanted in itertools.product((False, True), repeat=len(args)):
            if not any(wanted):
                assert not _first(call(*args)).requires_grad
                continue
            some = [a.clone().requires_grad_(w) for a, w in zip(args, wanted)]
            got = torch.autograd.grad(_first(call(*some)), [a for a, w in zip(some, wanted) if w], d)
            assert all(torch.equal(a, c) for a, c in zip(got, [c for c, w in zip(want, wanted) if w])), (name, wanted)


def test_inference_mode_records_nothing(ndvm, cuda):
    """Whatever the gradient mode within it, as torch's own operations; also where the inputs want gradients."""
    import torch
    x = torch.ones(12, 24, device="cuda").bfloat16().requires_grad_(True)
    m = torch.ones(40, 24, device="cuda").bfloat16().requires_grad_(True)
    calls = [(name, lambda call=call, args=[a.clone().requires_grad_(True) for a in args]: call(*args)) for name, call, args in _ops(ndvm)]
    calls += [("layer_norm", lambda: ndvm.layer_norm(x)), ("gated", lambda: ndvm.gated(x, m, m, keep=True)), ("dropout", lambda: ndvm.dropout(x, 0.5, 1)),
              ("rms_norm", lambda: ndvm.rms_norm(x, None, 1e-6, x)), ("linear", lambda: ndvm.linear(x, m, None, "silu")),
              ("linear, 8 bits", lambda: ndvm.linear(x, m, None, "silu", keep="8bit")), ("quantize", lambda: ndvm.quantize(x).dequantize()),
              ("rms_norm_quantized", lambda: ndvm.rms_norm_quantized(x).dequantize())]
    for name, call in calls:
        with torch.no_grad():
            want = _first(call())
        with torch.inference_mode():
            plain = _first(call())
            with torch.enable_grad():
                got = _first(call())
        assert not got.requires_grad and got.grad_fn is None and torch.equal(got, want) and torch.equal(plain, want), name


@pytest.mark.parametrize("k,shift", [(2049, 0), (2048, 1)])
def test_one_row_allocates_its_result_alone(ndvm, cuda, k, shift):
    """Rows off 16 bytes too: no room for copies of the weights that nothing makes."""
    import torch
    g = _gen(31)
    n = 4096
    w = torch.empty(n * k + shift, device="cuda", dtype=torch.bfloat16)[shift:].view(n, k)
    w.copy_(_randn(g, n, k))
    x, b = _randn(g, 1, k).bfloat16(), _randn(g, n)
    want = ndvm.linear(x, w.clone(), b, "silu")
    xg = x.clone().requires_grad_(True)
    ndvm.linear(xg, w, b, "silu")
    for call, most in ((lambda: ndvm.linear(x, w, b, "silu"), 2 * n), (lambda: ndvm.linear_forward(x, w, b, "silu"), 2 * n),
                       (lambda: ndvm.linear(xg, w, b, "silu"), 6 * n)):
        base = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        y = call()
        assert torch.cuda.max_memory_allocated() - base <= most + 1024
        assert torch.equal(y, want) or k % 8 == 0  # (vectors of eight sum in another order than single elements)
        del y
