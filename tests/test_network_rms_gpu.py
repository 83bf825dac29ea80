"""The root-mean-square norm and 8-bit blocks against plain implementations in 64 bits (GPU).

Bounds are derived as the layer norm's: everything in binary32 (unit roundoff U), one rounding to the output's type.  A row's
sum of squares has positive terms, so the mean is off by K U of itself (K: additions a chain at most) and the reciprocal
deviation by half of that and a few U."""
import pytest

from test_network_gpu import U, _gen, _inside, _randn, _rounded, _strided, _t

pytestmark = pytest.mark.gpu

EPS = 1e-6


def _rms64(s, w, dy, ds):
    """y, dx, dw and the bounds of the binary32 evaluation, all in 64 bits."""
    rows, cols = s.shape
    K, KR = cols / 32 + 64, rows + 64
    er = (K / 2 + 8) * U
    r = 1.0 / (s.square().mean(1, keepdim=True) + EPS).sqrt()
    sh = s * r
    y = sh * w
    ey = y.abs() * (er + 4 * U)
    g = dy * w
    m = (g * sh).mean(1, keepdim=True)
    em = (K * U + er + 4 * U) * (g * sh).abs().mean(1, keepdim=True)
    dx = ds + r * (g - sh * m)
    edx = r * ((er + 8 * U) * (g.abs() + 2 * (sh * m).abs()) + sh.abs() * em) + 4 * U * (ds.abs() + dx.abs())
    dw = (dy * sh).sum(0)
    edw = (KR * U + er + 4 * U) * (dy * sh).abs().sum(0)
    return (y, dx, dw), (ey, edx, edw)


SIZES = [(1, 1), (3, 1), (1, 2), (5, 7), (2, 31), (33, 32), (7, 33), (64, 256), (9, 255), (130, 1000), (17, 1024), (40, 1025),
         (300, 1537), (3, 4096), (5, 5001), (2, 8192), (2, 8200), (3, 16384), (2, 16421), (1, 40000), (20000, 24), (4999, 130),
         (3001, 64), (777, 61), (33, 8), (5, 16), (50, 1002), (9, 4098), (21, 514), (301, 66), (2, 8190), (13, 2050), (33000, 600)]


@pytest.mark.parametrize("t,wt", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rms_norm_matches_64_bits(ndvm, cuda, rows, cols, t, wt):
    import torch
    g = _gen(rows * 100003 + cols)
    x, res, dy, ds = ((_randn(g, rows, cols) * 1.5).to(_t(t)) for _ in range(4))
    w = (1 + 0.2 * _randn(g, cols)).to(_t(wt))
    for with_residual in (False, True):
        y, s, rstd = ndvm.rms_norm_forward(x, w, EPS, res if with_residual else None)
        if with_residual:
            assert torch.equal(s, (x.float() + res.float()).to(x.dtype))
        else:
            assert s is None
            s = x
        got = (y,) + ndvm.rms_norm_backward(dy, s, w, rstd, ds if with_residual else None)
        want, err = _rms64(s.double(), w.double(), dy.double(), ds.double() if with_residual else torch.zeros_like(ds, dtype=torch.float64))
        for name, a, v, e, o in zip(("y", "dx", "dweight"), got, want, err, (t, t, wt)):
            assert a.dtype == _t(o)
            _inside(a, v, _rounded(v, e, o), name)


@pytest.mark.parametrize("rows,cols,pad,shift", [(37, 200, 24, 8), (37, 200, 3, 1), (11, 1030, 2, 0), (9, 2048, 8, 0), (6, 9001, 7, 3)])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_rms_norm_strides_alignment_and_in_place(ndvm, cuda, rows, cols, pad, shift, t):
    """Strided and misaligned rows; the gaps are not written; the sum may take the place of x or of the residual."""
    import torch
    g = _gen(rows + cols)
    x, res, dy, ds = (_randn(g, rows, cols).to(_t(t)) for _ in range(4))
    w = _randn(g, cols).to(_t(t))
    outs = [torch.full((rows, cols + pad), 3.0, dtype=x.dtype, device="cuda") for _ in range(3)]
    y, s, dx = (o[:, shift:shift + cols] for o in outs)
    _, _, rstd = ndvm.rms_norm_forward(_strided(x, pad, shift), w, EPS, _strided(res, pad, shift), y=y, sum=s)
    _, dw = ndvm.rms_norm_backward(_strided(dy, pad, shift), s, w, rstd, _strided(ds, pad, shift), dx=dx)
    assert torch.equal(s, (x.float() + res.float()).to(x.dtype))
    want, err = _rms64(s.double(), w.double(), dy.double(), ds.double())
    for name, a, v, e in zip(("y", "dx", "dweight"), (y, dx, dw), want, err):
        _inside(a, v, _rounded(v, e, t), name)
    for o in outs:
        assert bool((o[:, :shift] == 3).all()) and bool((o[:, shift + cols:] == 3).all())
    for k in range(2):
        a = [x.clone(), res.clone()]
        y2, s2, _ = ndvm.rms_norm_forward(a[0], w, EPS, a[1], sum=a[k])
        assert s2 is a[k] and torch.equal(s2, s)
        _inside(y2, want[0], _rounded(want[0], err[0], t), "y, sum in place")
    wide = torch.zeros(2 * cols + 1, dtype=x.dtype, device="cuda")[1:cols + 1]  # weights that start anywhere
    wide.copy_(w)
    y3 = ndvm.rms_norm_forward(s.contiguous(), wide, EPS)[0]
    _inside(y3, want[0], _rounded(want[0], err[0], t), "y, shifted weight")


def test_rms_norm_partial_gradients_no_weights_and_no_rows(ndvm, cuda):
    import torch
    g = _gen(3)
    x, dy = _randn(g, 50, 300), _randn(g, 50, 300)
    one = torch.ones(300, device="cuda")
    y, _, rstd = ndvm.rms_norm_forward(x)
    assert torch.equal(y, ndvm.rms_norm_forward(x, one)[0])
    full = ndvm.rms_norm_backward(dy, x, one, rstd)
    for k in range(2):
        part = ndvm.rms_norm_backward(dy, x, one, rstd, wants=(k == 0, k == 1))
        assert part[1 - k] is None and torch.equal(part[k], full[k])
    assert torch.equal(ndvm.rms_norm_backward(dy, x, None, rstd, wants=(True, False))[0], full[0])
    none = torch.empty(0, 40, device="cuda")
    y, s, rstd = ndvm.rms_norm_forward(none, one[:40], EPS, none)
    dw = torch.full((40,), 5.0, device="cuda")
    ndvm.rms_norm_backward(none, none, one[:40], rstd, dweight=dw)
    assert y.shape == s.shape == (0, 40) and not dw.any()


def test_rms_norm_rows_keep_their_own_values(ndvm, cuda):
    """A row of zeros, one far from zero, rows with an infinity or a NaN: each as the formula has it, no row touches another."""
    import torch
    g = _gen(4)
    x, w = _randn(g, 12, 515), _randn(g, 515)
    clean = ndvm.rms_norm_forward(x, w)[0]
    v = x.clone()
    v[3], v[5, 17], v[8, 514], v[10] = 0.0, float("inf"), float("nan"), x[10] * 1e15
    y = ndvm.rms_norm_forward(v, w)[0]
    for r in (0, 1, 2, 4, 6, 7, 9, 11):
        assert torch.equal(y[r], clean[r]), r
    assert not y[3].any() and y[8].isnan().all() and y[5, 17].isnan() and not y[5, :17].any()
    want = (v[10].double() / (v[10].double().square().mean() + 1e-6).sqrt() * w.double())
    _inside(y[10], want, want.abs() * 200 * U, "far row")


def test_rms_norm_gradient_against_differences(ndvm, cuda):
    """The gradients' product with a direction against a central difference of the 64-bit definition (step 1e-4: its error is
    below 1e-7 of the magnitudes here)."""
    import torch
    g = _gen(6)
    x, res, w, dy, ds = _randn(g, 20, 77), _randn(g, 20, 77), 1 + 0.2 * _randn(g, 77), _randn(g, 20, 77), _randn(g, 20, 77)
    ins = [x.requires_grad_(True), w.requires_grad_(True), res.requires_grad_(True)]
    grads = torch.autograd.grad(ndvm.rms_norm(x, w, EPS, res), ins, (dy, ds))

    def f(x, w, res):
        s = x + res
        return float((s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * w * dy.double()).sum() + (s * ds.double()).sum())

    base = [t.detach().double() for t in ins]
    for k in range(3):
        v = _randn(g, *ins[k].shape).double()
        plus, minus = [list(base) for _ in range(2)]
        plus[k], minus[k] = base[k] + 1e-4 * v, base[k] - 1e-4 * v
        slope = (f(*plus) - f(*minus)) / 2e-4
        got = float((grads[k].double() * v).sum())
        assert abs(got - slope) <= 1e-5 * float((grads[k].double() * v).abs().sum()), (k, got, slope)


def test_rms_norm_op_with_one_cotangent(ndvm, cuda):
    """Either output alone may reach the loss; the same tensor may be x and residual; broadcast rows get their sum."""
    import torch
    g = _gen(7)
    x, w, r = (_randn(g, *n).bfloat16().requires_grad_(True) for n in ((30, 72), (72,), (30, 72)))
    d = _randn(g, 30, 72).bfloat16()
    y, s = ndvm.rms_norm(x, w, EPS, r)
    dx, dr, dw = torch.autograd.grad(s, (x, r, w), d, retain_graph=True)
    assert torch.equal(dx, d) and torch.equal(dr, d) and not dw.any()
    rstd = ndvm.rms_norm_forward(s.detach(), w.detach(), EPS)[2]
    want = ndvm.rms_norm_backward(d, s.detach(), w.detach(), rstd)
    dx, dw = torch.autograd.grad(y, (x, w), d)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    y, s = ndvm.rms_norm(x, w, EPS, x)
    twice, = torch.autograd.grad((y, s), x, (d, d))
    dx, _ = ndvm.rms_norm_backward(d, s.detach(), w.detach(), ndvm.rms_norm_forward(s.detach(), w.detach(), EPS)[2], d)
    assert torch.equal(twice, (dx.float() * 2).bfloat16())
    row = r.detach()[:1].clone().requires_grad_(True)
    y, _ = ndvm.rms_norm(x, w, EPS, row.expand(30, 72))
    a, b = torch.autograd.grad(y, (x, row), d)
    assert b.shape == (1, 72) and float((a.double().sum(0) - b[0].double()).abs().max()) <= 2 ** -8 * float(a.double().abs().sum(0).max())
    one = torch.ones(72, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(ndvm.rms_norm(x.detach(), one.expand(72), EPS), ndvm.rms_norm(x.detach(), None, EPS))
    assert torch.equal(torch.autograd.grad(ndvm.rms_norm(x, None, EPS).sum(), x)[0], torch.autograd.grad(ndvm.rms_norm(x, one, EPS).sum(), x)[0])


def test_rms_norm_past_32_bit_offsets(ndvm, cuda):
    """4.3e9 elements: the last rows are those of a call on them alone."""
    import torch
    rows, cols = 131104, 32768
    x = torch.zeros(rows, cols, dtype=torch.float16, device="cuda")
    tail, w = _randn(_gen(7), 40, cols).half(), _randn(_gen(8), cols).half()
    x[-40:] = tail
    y, _, rstd = ndvm.rms_norm_forward(x, w)
    part, _, prstd = ndvm.rms_norm_forward(tail, w)
    assert torch.equal(y[-40:], part) and torch.equal(rstd[-40:], prstd)
    dx = ndvm.rms_norm_backward(x, x, w, rstd, wants=(True, False), dx=y)[0]
    assert torch.equal(dx[-40:], ndvm.rms_norm_backward(tail, tail, w, prstd, wants=(True, False))[0])
    del y, dx
    q = ndvm.quantize_forward(x)
    part = ndvm.quantize_forward(tail)
    assert torch.equal(q.values[-40:].view(torch.uint8), part.values.view(torch.uint8))
    out = q.dequantize(torch.float16, out=x)
    assert torch.equal(out[-40:], part.dequantize(torch.float16)) and not out[:40].any()


@pytest.mark.parametrize("rows,cols", [(1000, 8193), (100, 16384), (63, 9000), (1000, 8192), (2000, 4097), (5, 300)])
def test_rms_norm_backward_within_its_workspace(ndvm, cuda, rows, cols):
    import torch
    g = _gen(rows + cols)
    x, dy, w = _randn(g, rows, cols), _randn(g, rows, cols), _randn(g, cols)
    _, _, rstd = ndvm.rms_norm_forward(x, w, EPS)
    need = ndvm.load().ndvm_rms_norm_workspace_bytes(rows, cols) // 4
    room = torch.full((need + 4 * cols,), 3.0, device="cuda")
    dx, dw = ndvm.rms_norm_backward(dy, x, w, rstd, workspace=room[:need])
    assert bool((room[need:] == 3).all())
    again = ndvm.rms_norm_backward(dy, x, w, rstd)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


# --------------------------------------------------------------------------------- 8-bit blocks
def _blocks64(v):
    """(what the blocks of v stand for, the exponents [rows, blocks]) by their definition; NaN and 128 where they have none."""
    import torch
    rows, cols = v.shape
    b = torch.nn.functional.pad(v.double(), (0, -cols % 32)).view(rows, -1, 32)
    most = b.abs().amax(2)
    bad = ~most.isfinite()
    most, b = most.masked_fill(bad, 0.0), b.masked_fill(bad[:, :, None], 0.0)
    e = torch.full_like(most, -127.0)
    guess = torch.floor(torch.log2(most.clamp_min(2.0 ** -200))) - 10
    for up in range(4):  # (the least exponent: one too small is stepped up, from below)
        e = torch.where((most > 448 * torch.exp2(e)), torch.maximum(guess + up, torch.full_like(e, -127.0)), e)
    u = b / torch.exp2(e)[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    held = (torch.round(u / step) * step * torch.exp2(e)[:, :, None]).masked_fill(bad[:, :, None], float("nan"))
    return held.reshape(rows, -1)[:, :cols], e.masked_fill(bad, 128.0)


def _same(a, b):
    """Equal, NaN to NaN."""
    import torch
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())


def _exponents(q):
    """The exponents of q's scales [rows, blocks]."""
    import torch
    r, b = torch.arange(q.rows, device="cuda")[:, None], torch.arange(-(-q.cols // 32), device="cuda")[None]
    return q.scales[r // 128, b // 4, r % 32, r // 32 % 4, b % 4].double() - 127


def _decode(q):
    """What q stands for, in 64 bits and from its bytes."""
    import torch
    bits = q.values.reshape(q.rows, q.cols).view(torch.uint8).long()
    e, m = bits >> 3 & 15, (bits & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e.double() - 7)) * torch.where(bits >= 128, -1.0, 1.0)
    e = _exponents(q).repeat_interleave(32, 1)[:, :q.cols]
    return torch.where((e == 128) | (bits & 127 == 127), float("nan"), v * torch.exp2(e))


BLOCK_SIZES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 7), (127, 128), (128, 129), (129, 130), (300, 777), (64, 1000), (33, 16), (7, 4096), (2, 9000), (1000, 2050)]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", BLOCK_SIZES)
def test_blocks_are_those_of_the_definition(ndvm, cuda, rows, cols, t):
    import torch
    g = _gen(rows * 31 + cols)
    x = (_randn(g, rows, cols) * torch.exp2(_randn(g, rows, cols) * 6)).to(_t(t))
    x[0, :] = 0
    want, e = _blocks64(x)
    for given in (x, _strided(x, 8, 0), _strided(x, 3, 1)):
        q = ndvm.quantize_forward(given)
        assert torch.equal(_exponents(q), e) and _same(_decode(q), want)
    raw = q.values.as_strided((rows, q.stride), (q.stride, 1)).view(torch.uint8)
    assert not raw[:, cols:].any()
    full = torch.zeros(-(-rows // 128) * 128, -(-cols // 128) * 4, device="cuda", dtype=torch.uint8)
    full[:rows, :e.shape[1]] = (e + 127).to(torch.uint8)
    assert torch.equal(q.scales, full.view(-1, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4))
    for o in ("f32", "f16", "bf16"):
        back = q.dequantize(_t(o))
        top = torch.finfo(_t(o)).max
        assert _same(back, want.clamp(-top, top).float().to(_t(o)))
    out = torch.full((rows, cols + 5), 3.0, device="cuda", dtype=torch.bfloat16)
    q.dequantize(out=out[:, 1:cols + 1])
    assert _same(out[:, 1:cols + 1], q.dequantize(torch.bfloat16)) and bool((out[:, :1] == 3).all()) and bool((out[:, cols + 1:] == 3).all())


def test_blocks_at_the_ends_of_the_range(ndvm, cuda):
    """Values at 448 2^e and just above, subnormals, the largest; blocks that are not finite are NaN, their neighbours not."""
    import torch
    x = torch.zeros(8, 64, device="cuda")
    x[0, :4] = torch.tensor([448.0, -448.0, 1.0, 2.0 ** -10])
    x[1, :3] = torch.tensor([448.0 * (1 + 2.0 ** -23), 1.0, -1.0])
    x[2, :3] = torch.tensor([2.0 ** -149, 2.0 ** -126, -2.0 ** -130])
    x[3, :2] = torch.tensor([torch.finfo(torch.float32).max, -1e38])
    x[4, 5], x[5, 40], x[6, 63] = float("inf"), float("nan"), -float("inf")
    x[4:7, 10] = 3.0
    q = ndvm.quantize_forward(x)
    want, e = _blocks64(x[:4])
    assert torch.equal(_exponents(q)[:4], e) and torch.equal(_decode(q)[:4], want)
    back = q.dequantize()
    top = torch.finfo(torch.float32).max
    assert torch.equal(back[:4].double(), want.clamp(-top, top)) and not back[7].any()
    bad = torch.tensor([[True, False], [False, True], [False, True]], device="cuda").repeat_interleave(32, 1)
    assert torch.equal(back[4:7].isnan(), bad)
    for t in (torch.float16, torch.bfloat16):
        top = torch.tensor([[torch.finfo(t).max] * 32], device="cuda", dtype=t)  # (its mantissa is rounded up to the next power of two)
        assert torch.equal(ndvm.quantize_forward(top).dequantize(t), top)


@pytest.mark.parametrize("t,wt", [("f32", "f32"), ("f16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,cols", BLOCK_SIZES + [(40, 61), (70, 66), (3, 16390), (200, 1536)])
def test_rms_norm_quantized(ndvm, cuda, rows, cols, t, wt):
    """The blocks of the norm in 64 bits, but where the binary32 norm lies across a border: each element within its own
    half step and the norm's bound, and nearly all equal."""
    import torch
    g = _gen(rows * 7 + cols)
    x, res = ((_randn(g, rows, cols) * 1.5).to(_t(t)) for _ in range(2))
    w = (1 + 0.2 * _randn(g, cols)).to(_t(wt))
    for r in (None, res, _strided(res, 3, 1)):
        q, s = ndvm.rms_norm_quantized_forward(x, w, EPS, r)
        if r is None:
            assert s is None
            s = x
        assert torch.equal(s, x if r is None else (x.float() + res.float()).to(x.dtype))
        (y, *_), (ey, *_) = _rms64(s.double(), w.double(), torch.zeros_like(s, dtype=torch.float64), 0 * s.double())
        want, e = _blocks64(y)
        got = _decode(q)
        # half a step is 2^-4 of an element (2^-10 2^e below 2^-6 2^e); a scale that lies across its border is one step off
        half = y.abs() * 2.0 ** -4 + 2.0 ** -9 * torch.exp2(e).repeat_interleave(32, 1)[:, :cols]
        _inside(got, y, half * (1 + 1e-5) + 2 * ey, "values")
        assert float((_exponents(q) != e).double().mean()) <= 1e-3 + 1.5 / e.numel()
        assert float((got != want).double().mean()) <= 1e-3 + 40.0 / got.numel()


def test_quantized_ops_have_no_gradient(ndvm, cuda):
    import torch
    x = _randn(_gen(1), 10, 64).bfloat16().requires_grad_(True)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    q = ndvm.quantize(x.detach())
    for call in (lambda: ndvm.quantize(x), lambda: ndvm.rms_norm_quantized(x, w), lambda: ndvm.rms_norm_quantized(x.detach(), w.requires_grad_(True)),
                 lambda: ndvm.linear_quantized(q, q, residual=x[:, :10])):
        with pytest.raises(ndvm.NdvmError, match="no gradient"):
            call()
        with torch.no_grad():
            call()


def test_quantized_keeps_leading_dimensions(ndvm, cuda):
    import torch
    x = _randn(_gen(2), 3, 5, 100)
    with torch.no_grad():
        q, flat = ndvm.quantize(x), ndvm.quantize(x.view(15, 100))
        assert q.shape == (3, 5, 100) and torch.equal(q.values.reshape(15, 100).view(torch.uint8), flat.values.view(torch.uint8))
        assert torch.equal(q.dequantize(), flat.dequantize().view(3, 5, 100))
        other = ndvm.Quantized(q.values, q.scales)
        assert torch.equal(other.dequantize(), q.dequantize())
        part = ndvm.quantize(x[:, 1:4])  # (any layout)
        assert torch.equal(part.dequantize(), ndvm.quantize(x[:, 1:4].contiguous()).dequantize())
        assert ndvm.quantize(x[:0]).dequantize().shape == (0, 5, 100)
