"""Dense layers, of 16-bit operands and of 8-bit blocks, against plain implementations in 64 bits (GPU).

Bounds as for the gated projection: sums on the tensor cores may truncate (2 U a term), the activations are off by 16 U,
dz is rounded to the operands' type once (or handed on in two halves, which is less), results once more."""
import math

import pytest

from test_network_gpu import RMS, U, _gen, _inside, _randn, _rounded, _strided, _t
from test_network_rms_gpu import _blocks64, _decode

pytestmark = pytest.mark.gpu

ACTS = [None, "silu", "gelu", "relu", "sigmoid"]


def _act64(name, z, ez):
    """act, act' and the bounds of their errors where z is off by ez (|act'| <= 1.13, |act''| <= 1)."""
    import torch
    if name is None:
        return z, torch.ones_like(z), ez, torch.zeros_like(z)
    if name == "relu":
        return z.clamp_min(0), (z > 0).double(), ez, (z.abs() <= ez).double()
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
        a, da = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        s = torch.sigmoid(z)
        a, da = (z * s, s * (1 + z * (1 - s))) if name == "silu" else (s, s * (1 - s))
    return a, da, 1.13 * ez + 16 * U * (a.abs() + z.abs() * 0.25 + (name == "sigmoid")), ez + 16 * U * (1 + z.abs())


def _forward64(x, w, b, res, act):
    z = x @ w.t() + b
    ez = 2 * U * (x.shape[1] + 8) * (x.abs() @ w.abs().t()) + 2 * U * (b.abs() + z.abs())
    a, _, ea, _ = _act64(act, z, ez)
    y = a + res
    return y, ea + 4 * U * (a.abs() + res.abs()), z, ez


def _backward64(x, w, z, ez, dy, act, t):
    """dx, dw, db and their bounds at x and z as they are held."""
    rows, n = dy.shape
    _, da, _, eda = _act64(act, z, ez)
    dz = dy * da
    edz = dy.abs() * eda + 4 * U * dz.abs()
    db, edb = dz.sum(0), edz.sum(0) + (rows + 64) * U * dz.abs().sum(0)
    ez = _rounded(dz, edz, t) if act else 0 * dz  # (dz is dy where there is no activation)
    size = dz.abs() + ez
    dx, dw = dz @ w, dz.t() @ x
    return (dx, dw, db), (ez @ w.abs() + 2 * U * (n + 8) * (size @ w.abs()), ez.t() @ x.abs() + 2 * U * (2 * rows + 8) * (size.t() @ x.abs()), edb)


def _case(seed, rows, k, n, t, bt):
    g = _gen(seed)
    return (_randn(g, rows, k).to(_t(t)), (_randn(g, n, k) * k ** -0.5).to(_t(t)), (0.3 * _randn(g, n)).to(_t(bt)), _randn(g, rows, n).to(_t(t)),
            _randn(g, rows, n).to(_t(t)))


SIZES = [(1, 1, 1), (1, 8, 16), (1, 2048, 640), (1, 333, 777), (1, 512, 4100), (1, 9, 2500), (2, 64, 64), (3, 100, 257), (4, 512, 130), (5, 7, 9),
         (8, 256, 2000), (9, 264, 72), (16, 4096, 64), (17, 65, 63), (31, 96, 129), (33, 40, 512), (64, 128, 128), (65, 72, 120), (100, 1000, 300),
         (127, 64, 256), (128, 63, 127), (129, 65, 129), (200, 520, 264), (256, 256, 256), (257, 130, 385), (300, 333, 777), (513, 200, 136),
         (1000, 48, 72), (2049, 16, 24), (5000, 120, 56), (70, 5000, 33)]


@pytest.mark.parametrize("t,bt", [("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_linear_matches_64_bits(ndvm, cuda, rows, k, n, t, bt):
    import torch
    x, w, b, res, dy = _case(rows * 7919 + k * 31 + n, rows, k, n, t, bt)
    d = [v.double() for v in (x, w, b, res, dy)]
    for i, act in enumerate(ACTS):
        bias, residual = (None, None) if i == (rows + k) % 5 else (b, res)
        kept = ndvm.linear_kept(x, w) if act else None
        y = ndvm.linear_forward(x, w, bias, act, residual, kept=kept)
        want, err, z, ez = _forward64(d[0], d[1], d[2] * (bias is not None), d[3] * (residual is not None), act)
        _inside(y, want, _rounded(want, err, t), f"y, {act}")
        if act:
            _inside(kept[:, :n], z, ez, "kept")
            assert torch.equal(y, ndvm.linear_forward(x, w, bias, act, residual)) or rows == 1
        got = ndvm.linear_backward(dy, x, w, act, kept=kept, btype=_t(bt))
        want, err = _backward64(d[0], d[1], z, ez, d[4], act, t)
        for name, a, v, e, o in zip(("dx", "dw", "dbias"), got, want, err, (t, t, bt)):
            assert a.dtype == _t(o)
            _inside(a, v, _rounded(v, e, o), f"{name}, {act}")
            # independent roundings (of dz, then of the output) add up as squares: three leaves the scatter of few outputs
            if v.numel() >= 64 and act != "relu" and o != "f32":
                assert float((a.double() - v).norm() / v.norm()) <= 3 * RMS[o], (name, act)
    ndvm.check_operators()


@pytest.mark.parametrize("rows,k,n", [(5003, 2008, 2601), (4999, 2003, 2600), (2300, 1024, 4100)])
def test_linear_of_many_tiles(ndvm, cuda, rows, k, n):
    """Sizes of several rounds of the largest tiles in every product, ragged at every edge."""
    x, w, b, res, dy = _case(rows, rows, k, n, "bf16", "f32")
    d = [v.double() for v in (x, w, b, res, dy)]
    for act, keep in (("silu", None), ("gelu", "8bit"), (None, None)):
        kept = ndvm.linear_kept(x, w, keep) if act else None
        y = ndvm.linear_forward(x, w, b, act, res, kept=kept)
        want, err, z, ez = _forward64(*d[:4], act)
        _inside(y, want, _rounded(want, err, "bf16"), "y")
        xb = x
        if keep:
            z, ez = _decode(kept), 0 * z
            xb = ndvm.quantize_forward(x)
            d[0] = _decode(xb)
        got = ndvm.linear_backward(dy, xb, w, act, kept=kept, btype=b.dtype)
        want, err = _backward64(d[0], d[1], z, ez, d[4], act, "bf16")
        for name, a, v, e, o in zip(("dx", "dw", "dbias"), got, want, err, ("bf16", "bf16", "f32")):
            _inside(a, v, _rounded(v, e, o), f"{name}, {act}")
        d[0] = x.double()
    ndvm.check_operators()


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", SIZES[::2] + [(130, 72, 1001), (300, 1100, 136), (16, 8192, 40)])
def test_linear_held_in_8_bits(ndvm, cuda, rows, k, n, t):
    """z's blocks are those of z but where its binary32 value lies across a border; the gradients are those at what is
    held; the op is the raw calls."""
    import torch
    act = ACTS[1:][(rows + k + n) % 4]
    x, w, b, res, dy = _case(rows * 7919 + k * 31 + n, rows, k, n, t, t)
    d = [v.double() for v in (x, w, b, res, dy)]
    kept, xb = ndvm.linear_kept(x, w, "8bit"), ndvm.quantize_forward(x)
    y = ndvm.linear_forward(x, w, b, act, res, kept=kept)
    want, err, z, ez = _forward64(*d[:4], act)
    _inside(y, want, _rounded(want, err, t), "y")
    blocks, e = _blocks64(z)
    held = _decode(kept)
    half = z.abs() * 2.0 ** -4 + 2.0 ** -9 * torch.exp2(e).repeat_interleave(32, 1)[:, :n]
    _inside(held, z, half * (1 + 1e-5) + 2 * ez, "held z")
    assert float((held != blocks).double().mean()) <= 2e-3 + 40.0 / held.numel()
    got = ndvm.linear_backward(dy, xb, w, act, kept=kept)
    want, err = _backward64(_decode(xb), d[1], held, 0 * held, d[4], act, t)
    for name, a, v, e in zip(("dx", "dw", "dbias"), got, want, err):
        _inside(a, v, _rounded(v, e, t), name)
    leaves = [v.clone().requires_grad_(True) for v in (x, w, b, res)]
    y2 = ndvm.linear(*leaves[:3], act, leaves[3], keep="8bit")
    grads = torch.autograd.grad(y2, leaves, dy)
    assert torch.equal(y, y2) and all(torch.equal(a, g) for a, g in zip(grads, (*got, dy)))
    ndvm.check_operators()


@pytest.mark.parametrize("rows,k,n", [(1, 72, 130), (3, 7, 5), (65, 333, 130), (300, 136, 50), (700, 264, 520), (40, 4100, 70)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)])
def test_linear_strides_alignment_and_workspace(ndvm, cuda, rows, k, n, pad, shift):
    """Strided and misaligned operands, inside the workspace that was asked for, and outputs whose gaps are not written."""
    import torch
    plain = _case(rows + k + n, rows, k, n, "bf16", "bf16")
    d = [v.double() for v in plain]
    x, w, res, dy = (_strided(plain[i], pad, shift) for i in (0, 1, 3, 4))
    size = ndvm.load().ndvm_linear_workspace_bytes
    for act, keep in ((1, None), (1, "8bit"), (0, None)):
        name = "gelu" if act else None
        kept = ndvm.linear_kept(x, w, keep) if act else None
        xb = ndvm.quantize_forward(x) if keep else x
        needs = [size(1 if act else 4, rows, k, n, back, 0, int(bool(keep))) for back in (0, 1)]
        rooms = [torch.full((need + 65536,), 3, device="cuda", dtype=torch.uint8) for need in needs]
        yo, dxo = torch.full((rows, n + pad), 3.0, device="cuda").bfloat16(), torch.full((rows, k + pad), 3.0, device="cuda").bfloat16()
        y = ndvm.linear_forward(x, w, plain[2], name, res, y=yo[:, shift:shift + n], kept=kept, workspace=rooms[0][:needs[0]])
        got = ndvm.linear_backward(dy, xb, w, name, dx=dxo[:, shift:shift + k], kept=kept, workspace=rooms[1][:needs[1]])
        for room, need in zip(rooms, needs):
            assert bool((room[need:] == 3).all())
        for o, c in ((yo, n), (dxo, k)):
            assert bool((o[:, :shift] == 3).all()) and bool((o[:, shift + c:] == 3).all())
        want, err, z, ez = _forward64(*d[:4], name)
        _inside(y, want, _rounded(want, err, "bf16"), "y")
        if keep:
            z, ez = _decode(kept), 0 * z
        want, err = _backward64(_decode(xb) if keep else d[0], d[1], z, ez, d[4], name, "bf16")
        for what, a, v, e in zip(("dx", "dw", "dbias"), got, want, err):
            _inside(a, v, _rounded(v, e, "bf16"), what)
    ndvm.check_operators()


def test_linear_in_place_and_partial_gradients(ndvm, cuda):
    import torch
    x, w, b, res, dy = _case(5, 300, 200, 136, "bf16", "bf16")
    want = ndvm.linear_forward(x, w, b, "silu", res)
    r = res.clone()
    assert ndvm.linear_forward(x, w, b, "silu", r, y=r) is r and torch.equal(r, want)
    kept = ndvm.linear_kept(x, w)
    ndvm.linear_forward(x, w, b, "silu", res, kept=kept)
    full = ndvm.linear_backward(dy, x, w, "silu", kept=kept)
    for i in range(3):
        part = ndvm.linear_backward(dy, x, w, "silu", wants=[i == j for j in range(3)], kept=kept)
        assert [p is None for p in part] == [i != j for j in range(3)] and torch.equal(part[i], full[i])
    leaves = [v.requires_grad_(True) for v in (x, w, b, res)]
    grads = torch.autograd.grad(ndvm.linear(x, w, b, "silu", res), leaves, dy)
    assert all(torch.equal(a, g) for a, g in zip(grads, (*full, dy)))
    for i in range(4):
        alone = [v.detach().requires_grad_(i == j) for j, v in enumerate(leaves)]
        for keep in (None, "8bit"):
            g, = torch.autograd.grad(ndvm.linear(*alone[:3], "silu", alone[3], keep=keep), alone[i], dy)
            assert keep or torch.equal(g, (*full, dy)[i])
    none = x[:0]
    for keep in (None, "8bit"):
        y = ndvm.linear(none, w, b, "silu", res[:0], keep=keep)
        g = torch.autograd.grad(y, (x, w, b), dy[:0])
        assert y.shape == (0, 136) and not any(v.any() for v in g)


def test_linear_of_leading_dimensions_and_broadcast_cotangents(ndvm, cuda):
    import torch
    x, w, b, res, dy = _case(6, 30, 72, 40, "f16", "f16")
    x, w = x.requires_grad_(True), w.requires_grad_(True)
    y = ndvm.linear(x.view(3, 10, 72), w, b, "gelu", res.view(3, 10, 40))
    assert torch.equal(y.view(30, 40), ndvm.linear(x, w, b, "gelu", res))
    got = torch.autograd.grad(y.sum(), (x, w))
    want = torch.autograd.grad(ndvm.linear(x, w, b, "gelu", res), (x, w), torch.ones_like(dy))
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    t = ndvm.linear(x.detach().view(3, 10, 72).transpose(0, 1), w.detach(), b)  # (any layout: it is copied)
    assert torch.equal(t.transpose(0, 1).reshape(30, 40), ndvm.linear(x.detach(), w.detach(), b))
    m = ndvm.linear(x.detach(), w.detach().t().contiguous().t(), b)
    assert torch.equal(m, ndvm.linear(x.detach(), w.detach(), b))


def test_linear_gradient_against_differences(ndvm, cuda):
    """The gradients' product with a direction against a central difference of the 64-bit definition; the gradients' own
    roundings are bf16's: 2^-9 in the root mean square each, at most two in a chain."""
    import torch
    x, w, b, res, dy = _case(8, 60, 90, 50, "bf16", "f32")
    ins = [v.requires_grad_(True) for v in (x, w, b, res)]
    g = _gen(9)
    for act in ACTS[:3] + ACTS[4:]:
        grads = torch.autograd.grad(ndvm.linear(x, w, b, act, res), ins, dy)
        base = [v.detach().double() for v in ins]
        for i in range(4):
            v = _randn(g, *ins[i].shape).double()
            at = [[base[j] + s * 1e-4 * v if i == j else base[j] for j in range(4)] for s in (1, -1)]
            f = [float(((_act64(act, a[0] @ a[1].t() + a[2], 0 * dy.double())[0] + a[3]) * dy.double()).sum()) for a in at]
            slope, terms = (f[0] - f[1]) / 2e-4, grads[i].double() * v
            assert abs(float(terms.sum()) - slope) <= 2 * 2.0 ** -8 * float(terms.norm()) + 1e-6 * float(terms.abs().sum()), (act, i)


def test_linear_of_values_that_are_not_finite(ndvm, cuda):
    """A row with an infinity or a NaN spoils its own results, and no other row's."""
    import torch
    x, w, b, res, _ = _case(11, 200, 136, 72, "bf16", "bf16")
    clean = ndvm.linear_forward(x, w, b, None, res)
    x[3, 5], x[130, 7], res[60, 9] = float("nan"), float("inf"), float("-inf")
    y = ndvm.linear_forward(x, w, b, None, res)
    assert y[3].isnan().all() and not y[130].isfinite().any() and y[60, 9] == float("-inf")
    same = torch.ones_like(y, dtype=torch.bool)
    same[3], same[130], same[60, 9] = False, False, False
    assert torch.equal(y[same], clean[same])


# --------------------------------------------------------------------------------- 8-bit operands
BLOCK_SIZES = [(1, 1, 1), (1, 200, 300), (2, 32, 16), (3, 33, 65), (5, 130, 9), (64, 128, 64), (64, 1024, 192), (100, 96, 200), (127, 160, 257),
               (128, 256, 384), (129, 1000, 130), (200, 31, 64), (256, 64, 1000), (300, 777, 333), (513, 300, 65), (1000, 2000, 500), (40, 8200, 70),
               (2500, 520, 3000), (3000, 1100, 1999)]


@pytest.mark.parametrize("t,bt", [("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,k,n", BLOCK_SIZES)
def test_linear_quantized_matches_64_bits(ndvm, cuda, rows, k, n, t, bt):
    """The products of what the blocks stand for, blocks of very different scales among them."""
    import torch
    x, w, b, res, _ = _case(rows * 31 + k * 7 + n, rows, k, n, "f16" if t == "f16" else "bf16", bt)
    g = _gen(k + n)
    x = x.float() * torch.exp2(torch.randint(-12, 6, (rows, 1), generator=g, device="cuda")) * torch.exp2(torch.randint(-3, 3, (1, k), generator=g, device="cuda"))
    wf = w.float() * torch.exp2(torch.randint(-8, 8, (n, 1), generator=g, device="cuda"))
    act = ACTS[(rows + k + n) % 5]
    q, p = ndvm.quantize_forward(x), ndvm.quantize_forward(wf)
    for bias, r in ((b, res), (None, None), (b, _strided(res, 3, 1))):
        y = ndvm.linear_quantized_forward(q, p, bias, act, r, dtype=_t(t))
        want, err, _, _ = _forward64(_decode(q), _decode(p), b.double() * (bias is not None), res.double() * (r is not None), act)
        assert y.dtype == _t(t)
        if t == "f16":
            want = want.clamp(-65504, 65504)
        ok = y.isfinite() | (want.abs() < 65000)
        _inside(torch.where(ok, y, 0), torch.where(ok, want, 0.0), _rounded(want, err, t), f"y, {act}")
    with torch.no_grad():
        assert torch.equal(ndvm.linear_quantized(q, p, b, act, res, _t(t)), ndvm.linear_quantized_forward(q, p, b, act, res, dtype=_t(t)))
    ndvm.check_operators()


def test_linear_quantized_reads_nothing_behind_the_blocks(ndvm, cuda):
    """Scales of no block may be anything (255 is a NaN), as may the bytes behind the last element; blocks that are NaN spoil their
    own row alone."""
    import torch
    for rows, k, n in ((100, 200, 72), (130, 40, 200), (64, 130, 330)):
        g = _gen(rows)
        x, w = _randn(g, rows, k), _randn(g, n, k)
        q, p = ndvm.quantize_forward(x), ndvm.quantize_forward(w)
        want = ndvm.linear_quantized_forward(q, p)
        for v in (q, p):
            e = v.scales.clone()
            r, b = torch.arange(v.rows, device="cuda")[:, None], torch.arange(-(-v.cols // 32), device="cuda")[None]
            v.scales.fill_(255)
            at = (r // 128, b // 4, r % 32, r // 32 % 4, b % 4)
            v.scales[at] = e[at]
            v.values.as_strided((v.rows, v.stride), (v.stride, 1)).view(torch.uint8)[:, v.cols:] = 0x7f
        assert torch.equal(ndvm.linear_quantized_forward(q, p), want)
        x[7, 3] = float("nan")
        y = ndvm.linear_quantized_forward(ndvm.quantize_forward(x), p)
        assert y[7].isnan().all() and torch.equal(y[:7], want[:7]) and torch.equal(y[8:], want[8:])


def test_scored_block_together(ndvm, cuda):
    """The norm of the stream's sum, a layer up and one back into the stream, in 8 bits: against the same steps in 64 bits.
    Rounding to e4m3 is off by 2^-4 at most, its root mean square below 2^-5; the three operands of each product that are
    rounded (x, h and two weights in all) add up as squares: sqrt(4) 2^-5 < 0.07 of the layer's part of the stream."""
    import torch
    g = _gen(12)
    x, add = _randn(g, 500, 256).bfloat16(), _randn(g, 500, 256).bfloat16()
    scale = (1 + 0.2 * _randn(g, 256)).bfloat16()
    up, down, b = _randn(g, 600, 256) / 16, _randn(g, 256, 600) / 24, 0.1 * _randn(g, 600)
    with torch.no_grad():
        h, s = ndvm.rms_norm_quantized(x, scale, 1e-6, add)
        h = ndvm.linear_quantized(h, ndvm.quantize(up), b, "gelu")
        y = ndvm.linear_quantized(ndvm.quantize(h), ndvm.quantize(down), None, None, s)
    sd = (x.float() + add.float()).bfloat16().double()
    n = sd / (sd.square().mean(1, keepdim=True) + 1e-6).sqrt() * scale.double()
    part = torch.nn.functional.gelu(n @ up.double().t() + b.double()) @ down.double().t()
    assert torch.equal(s.double(), sd)
    assert float((y.double() - sd - part).norm() / part.norm()) <= 0.07 + 2.0 ** -8 * float(sd.norm() / part.norm())


def test_trained_block_together(ndvm, cuda):
    """The pre-norm block as it is trained, its activations held as they are and in 8 bits, against torch's operations in 64
    bits.  Each bf16 rounding in a chain (at most 8) is off by 2^-9 in the root mean square: sqrt(8) 2^-9 < 6e-3, and 2e-2
    leaves cancellation; held in 8 bits, gradients see x and z off by 2^-5: 0.1."""
    import torch
    g = _gen(13)
    x, add = (_randn(g, 400, 256).bfloat16().requires_grad_(True) for _ in range(2))
    scale = (1 + 0.2 * _randn(g, 256)).requires_grad_(True)
    up = (_randn(g, 512, 256) / 16).bfloat16().requires_grad_(True)
    down = (_randn(g, 256, 512) / 22).bfloat16().requires_grad_(True)
    b = (0.1 * _randn(g, 512)).requires_grad_(True)
    leaves = [x, add, scale, up, down, b]
    dy = _randn(g, 400, 256).bfloat16()
    d = [v.detach().double().requires_grad_(True) for v in leaves]
    s = d[0] + d[1]
    n = s / (s.square().mean(1, keepdim=True) + 1e-6).sqrt() * d[2]
    want_y = torch.nn.functional.silu(n @ d[3].t() + d[5]) @ d[4].t() + s
    want = torch.autograd.grad(want_y, d, dy.double())
    for keep, most in ((None, 2e-2), ("8bit", 0.1)):
        h, s = ndvm.rms_norm(x, scale, 1e-6, add)
        y = ndvm.linear(ndvm.linear(h, up, b, "silu", keep=keep), down, None, None, s, keep=keep)
        assert float((y.double() - want_y).detach().norm() / want_y.detach().norm()) <= 2e-2
        for i, (a, c) in enumerate(zip(torch.autograd.grad(y, leaves, dy), want)):
            assert float((a.double() - c).norm() / c.norm()) <= most, (keep, i)
    ndvm.check_operators()


@pytest.mark.parametrize("act,keep", [("silu", None), ("gelu", "8bit"), (None, None)])
def test_linear_past_32_bit_offsets(ndvm, cuda, act, keep):
    """4.3e9 elements of the result: its last rows, and gradients that only they and the first ones make."""
    import torch
    rows, k, n = 131200, 16, 33000
    some = torch.cat((torch.arange(40), torch.arange(rows - 60, rows))).cuda()
    x, w, b, res, dy = _case(14, 100, k, n, "bf16", "f32")
    d = [v.double() for v in (x, w, b, res, dy)]
    big = torch.zeros(rows, k, device="cuda", dtype=torch.bfloat16)
    big[some] = x
    y = torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16)
    y[some] = res
    kept = ndvm.linear_kept(big, w, keep) if act else None
    ndvm.linear_forward(big, w, b, act, y, y=y, kept=kept)
    want, err, z, ez = _forward64(*d[:4], act)
    _inside(y[some], want, _rounded(want, err, "bf16"), "y")
    held = ndvm.quantize_forward(big) if keep else big
    if keep:
        part = ndvm.linear_kept(x, w, keep)
        ndvm.linear_forward(x, w, b, act, res, kept=part)
        assert torch.equal(kept.values.view(torch.uint8)[some], part.values.view(torch.uint8))
        z, ez, d[0] = _decode(part), 0 * z, _decode(ndvm.quantize_forward(x))
    elif act:
        _inside(kept[some][:, :n], z, ez, "kept")
    y.zero_()
    y[some] = dy
    got = ndvm.linear_backward(y, held, w, act, kept=kept, btype=torch.float32)
    want, err = _backward64(d[0], d[1], z, ez, d[4], act, "bf16")
    for name, a, v, e, o in zip(("dx", "dw", "dbias"), (got[0][some], *got[1:]), want, err, ("bf16", "bf16", "f32")):
        _inside(a, v, _rounded(v, e, o), name)
    assert not got[0][40:rows - 60].any()
    ndvm.check_operators()


def test_linear_quantized_past_32_bit_offsets(ndvm, cuda):
    import torch
    rows, k, n = 131200, 40, 33000
    x, w, b, res, _ = _case(15, 60, k, n, "bf16", "f32")
    q = ndvm.quantize_forward(w)
    big = torch.zeros(rows, k, device="cuda", dtype=torch.bfloat16)
    big[-60:] = x
    y = torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16)
    y[-60:] = res
    ndvm.linear_quantized_forward(ndvm.quantize_forward(big), q, b, "relu", y, y=y)
    assert torch.equal(y[-60:], ndvm.linear_quantized_forward(ndvm.quantize_forward(x), q, b, "relu", res))
    assert torch.equal(y[70000], torch.relu(b).bfloat16())


def test_inputs_whose_rows_are_one(ndvm, cuda):
    """Rows of stride 0 (an expanded row) as x, residual and cotangent; blocks of such rows; a part of other blocks."""
    import torch
    x, w, b, res, dy = _case(16, 200, 136, 72, "bf16", "bf16")
    for i, act in enumerate(ACTS):
        one = [v[:1].expand(200, v.shape[1]) for v in (x, res, dy)]
        full = [v.contiguous() for v in one]
        keep = "8bit" if act and i % 2 else None
        results = []
        for xi, ri, di in (one, full):
            kept = ndvm.linear_kept(xi, w, keep) if act else None
            y = ndvm.linear_forward(xi, w, b, act, ri, kept=kept)
            results.append((y, *ndvm.linear_backward(di, ndvm.quantize_forward(xi) if keep else xi, w, act, kept=kept)))
        assert all(torch.equal(a, c) for a, c in zip(*results)), act
    one, full = x[:1].expand(200, 136), x[:1].repeat(200, 1)
    assert all(torch.equal(a, c) for a, c in zip(ndvm.rms_norm_forward(one, None, 1e-6, one), ndvm.rms_norm_forward(full, None, 1e-6, full)))
    q = ndvm.quantize_forward(x.repeat(2, 1))
    part = ndvm.Quantized(q.values[128:], q.scales[1:])
    assert torch.equal(part.dequantize(), q.dequantize()[128:])
    p = ndvm.quantize_forward(w)
    assert torch.equal(ndvm.linear_quantized_forward(part, p, b), ndvm.linear_quantized_forward(q, p, b)[128:])
