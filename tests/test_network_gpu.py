"""Layer norm, dropout and the gated projection against plain implementations in 64 bits (GPU).

Bounds are derived, element by element, from the arithmetic that the operators state: everything in
binary32 (unit roundoff U = 2^-24) with one rounding to the output's type (to nearest with 8, 11 and 24
significant bits: off by at most 2^-8, 2^-11 and 2^-24 of the value), dG and dU rounded to the operands'
type in between.  A binary32 sum of n terms in any order is off by at most (n - 1) U times the
sum of their magnitudes; the layer norm's row sums go over at most C/32 + 64 additions a chain, its
column sums over at most R + 64.  The bounds hold for any order, so they do not depend on a kernel's split.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
RMS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -9}  # bounds of one rounding's root mean square
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}  # half a subnormal step and underflow in 32 bits


def _t(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _inside(got, want, bound, what):
    err = (got.double() - want).abs()
    over = err > bound
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {over.numel()} outside, worst {float((err / bound).max()):.3g} "
                                  f"times the bound")
    assert bool(got.isfinite().all()), what


def _gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    import torch
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _strided(x, pad, shift):
    """The same values in rows that are `pad` elements longer, `shift` elements into their memory."""
    import torch
    base = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=x.dtype, device=x.device)
    view = base[:, shift:shift + x.shape[1]]
    view.copy_(x)
    return view


# ------------------------------------------------------------------------------- layer norm
def _norm64(x, w, b, dy, eps):
    """y, dx, dw, db and the bounds of the binary32 evaluation, all in 64 bits."""
    rows, cols = x.shape
    K, KR = cols / 32 + 64, rows + 64
    m = x.mean(1, keepdim=True)
    r = 1.0 / ((x - m).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (x - m) * r
    # the mean is off by K U mean|x|, differences by another U, the deviation by K U relative (and the
    # mean's error does not count in it to first order, but is allowed for)
    dm = K * U * x.abs().mean(1, keepdim=True)
    dxh = r * dm * 2 + xh.abs() * (3 * K * U + r * r * dm * dm) + 4 * U * xh.abs()
    y = xh * w + b
    ey = w.abs() * dxh + 4 * U * ((xh * w).abs() + b.abs())
    g = dy * w
    mg, mgx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - mg - xh * mgx)
    e_mg = K * U * g.abs().mean(1, keepdim=True)
    e_mgx = K * U * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * dxh).mean(1, keepdim=True)
    edx = r * (e_mg + xh.abs() * e_mgx + mgx.abs() * dxh + 8 * U * (g.abs() + mg.abs() + (xh * mgx).abs()))
    edx = edx + dx.abs() * (3 * K * U + r * r * dm * dm)
    dw, db = (dy * xh).sum(0), dy.sum(0)
    edw = KR * U * (dy * xh).abs().sum(0) + (dy.abs() * dxh).sum(0)
    edb = KR * U * dy.abs().sum(0)
    return (y, dx, dw, db), (ey, edx, edw, edb)


def _rounded(want, err, t):
    return err + ROUND[t] * (want.abs() + err) + TINY[t]


NORM_SIZES = [(1, 1), (3, 1), (1, 2), (5, 7), (2, 31), (33, 32), (7, 33), (64, 256), (9, 255), (130, 1000), (17, 1024),
              (40, 1025), (300, 1537), (3, 4096), (5, 5001), (2, 8192), (2, 8200), (3, 16384), (2, 16421), (1, 40000),
              (2, 70001), (20000, 24), (4999, 130), (3001, 64), (1003, 128), (777, 61), (33, 8), (5, 16), (50, 1002), (9, 4098), (21, 514), (301, 66), (2, 8190),
              (13, 2050), (6, 250), (33000, 1104), (33000, 600)]


@pytest.mark.parametrize("t,wt", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_layer_norm_matches_64_bits(ndvm, cuda, rows, cols, t, wt):
    g = _gen(rows * 100003 + cols)
    x = (_randn(g, rows, cols) * 1.5 + 0.5 * _randn(g, cols)).to(_t(t))
    w, b = (1 + 0.2 * _randn(g, cols)).to(_t(wt)), (0.2 * _randn(g, cols)).to(_t(wt))
    dy = _randn(g, rows, cols).to(_t(t))
    y, stats = ndvm.layer_norm_forward(x, w, b)
    got = (y,) + ndvm.layer_norm_backward(dy, x, w, stats)
    want, err = _norm64(x.double(), w.double(), b.double(), dy.double(), 1e-5)
    for name, a, v, e, o in zip(("y", "dx", "dweight", "dbias"), got, want, err, (t, t, wt, wt)):
        assert a.dtype == _t(o)
        _inside(a, v, _rounded(v, e, o), name)


@pytest.mark.parametrize("rows,cols,pad,shift", [(37, 200, 24, 8), (37, 200, 3, 1), (11, 1030, 2, 0), (64, 64, 64, 32),
                                                 (9, 2048, 8, 0), (6, 9001, 7, 3)])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_layer_norm_strides_and_alignment(ndvm, cuda, rows, cols, pad, shift, t):
    """Strided and misaligned rows give the bits of contiguous ones; the gaps are not written."""
    import torch
    g = _gen(rows + cols)
    x, dy = _randn(g, rows, cols).to(_t(t)), _randn(g, rows, cols).to(_t(t))
    w, b = _randn(g, cols).to(_t(t)), _randn(g, cols).to(_t(t))
    y, stats = ndvm.layer_norm_forward(x, w, b)
    want, err = _norm64(x.double(), w.double(), b.double(), dy.double(), 1e-5)
    out, dxo = (torch.full((rows, cols + pad), 3.0, dtype=x.dtype, device="cuda") for _ in range(2))
    ys, st = ndvm.layer_norm_forward(_strided(x, pad, shift), w, b, y=out[:, shift:shift + cols])
    got = ndvm.layer_norm_backward(_strided(dy, pad, shift), _strided(x, pad, shift), w, st, dx=dxo[:, shift:shift + cols])
    for name, a, v, e in zip(("y", "dx", "dweight", "dbias"), (ys,) + got, want, err):
        _inside(a, v, _rounded(v, e, t), name)
    for o in (out, dxo):
        assert bool((o[:, :shift] == 3).all()) and bool((o[:, shift + cols:] == 3).all())
    wide = torch.zeros(2 * cols + 1, dtype=x.dtype, device="cuda")[1:cols + 1]  # weights that start anywhere
    wide.copy_(w)
    y2, _ = ndvm.layer_norm_forward(x, wide, b)
    _inside(y2, want[0], _rounded(want[0], err[0], t), "y, shifted weight")


def test_layer_norm_without_weights_and_partial_gradients(ndvm, cuda):
    import torch
    g = _gen(3)
    x, dy = _randn(g, 50, 300), _randn(g, 50, 300)
    one, zero = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    want, err = _norm64(x.double(), one.double(), zero.double(), dy.double(), 0.25)
    y, stats = ndvm.layer_norm_forward(x, eps=0.25)
    _inside(y, want[0], _rounded(want[0], err[0], "f32"), "y")
    full = ndvm.layer_norm_backward(dy, x, one, stats)
    for k in range(3):
        part = ndvm.layer_norm_backward(dy, x, one, stats, wants=tuple(i == k for i in range(3)))
        assert [p is None for p in part] == [i != k for i in range(3)]
        assert torch.equal(part[k], full[k])
    assert torch.equal(ndvm.layer_norm_backward(dy, x, None, stats, wants=(True, False, False))[0], full[0])


def test_layer_norm_of_no_rows_clears_the_weight_gradients(ndvm, cuda):
    import torch
    x = torch.empty(0, 40, device="cuda")
    y, stats = ndvm.layer_norm_forward(x, torch.ones(40, device="cuda"))
    assert y.shape == (0, 40) and stats.shape == (2, 0)
    dw, db = torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
    ndvm.layer_norm_backward(x, x, torch.ones(40, device="cuda"), stats, dweight=dw, dbias=db)
    assert not dw.any() and not db.any()


def test_layer_norm_rows_keep_their_own_values(ndvm, cuda):
    """A constant row, a row far from zero, rows with an infinity or a NaN: each as the formula has it,
    and no row touches another."""
    import torch
    g = _gen(4)
    x = _randn(g, 12, 515)
    w, b = _randn(g, 515), _randn(g, 515)
    clean, _ = ndvm.layer_norm_forward(x, w, b)
    y0 = x.clone()
    y0[3], y0[5, 17], y0[8, 514], y0[10] = 2.5, float("inf"), float("nan"), x[10] + 3000.0
    y, stats = ndvm.layer_norm_forward(y0, w, b)
    for r in (0, 1, 2, 4, 6, 7, 9, 11):
        assert torch.equal(y[r], clean[r]), r
    assert torch.equal(y[3], b) and y[5].isnan().all() and y[8].isnan().all()
    want, err = _norm64(y0[10:11].double(), w.double(), b.double(), w.double().view(1, -1), 1e-5)
    _inside(y[10:11], want[0], _rounded(want[0], err[0], "f32"), "far row")


def test_layer_norm_gradient_against_differences(ndvm, cuda):
    """sum(y dy) along random directions: the gradients' product with the direction against a central
    difference of the 64-bit definition (step 1e-4: its error is below 1e-7 of the magnitudes here)."""
    import torch
    g = _gen(6)
    x, w, b, dy = _randn(g, 20, 77), 1 + 0.2 * _randn(g, 77), _randn(g, 77), _randn(g, 20, 77)
    ins = [x.requires_grad_(True), w.requires_grad_(True), b.requires_grad_(True)]
    grads = torch.autograd.grad(ndvm.layer_norm(*ins), ins, dy)

    def f(x, w, b):
        xc = x - x.mean(1, keepdim=True)
        return float(((xc / (xc.square().mean(1, keepdim=True) + 1e-5).sqrt() * w + b) * dy.double()).sum())

    base = [t.detach().double() for t in ins]
    for k in range(3):
        v = _randn(g, *ins[k].shape).double()
        plus, minus = [list(base) for _ in range(2)]
        plus[k], minus[k] = base[k] + 1e-4 * v, base[k] - 1e-4 * v
        slope = (f(*plus) - f(*minus)) / 2e-4
        got = float((grads[k].double() * v).sum())
        assert abs(got - slope) <= 1e-5 * float((grads[k].double() * v).abs().sum()), (k, got, slope)


def test_layer_norm_past_32_bit_offsets(ndvm, cuda):
    """4.3e9 elements: the last rows are those of a call on them alone."""
    import torch
    rows, cols = 131104, 32768
    x = torch.empty(rows, cols, dtype=torch.float16, device="cuda")
    tail = _randn(_gen(7), 40, cols).half()
    x[:40], x[-40:] = tail, tail
    x[40:-40] = 0
    w = _randn(_gen(8), cols).half()
    y, stats = ndvm.layer_norm_forward(x, w, w)
    part, pstats = ndvm.layer_norm_forward(tail, w, w)
    assert torch.equal(y[-40:], part) and torch.equal(y[:40], part) and torch.equal(stats[:, -40:], pstats)
    dx = ndvm.layer_norm_backward(x, x, w, stats, wants=(True, False, False), dx=y)[0]
    assert torch.equal(dx[-40:], ndvm.layer_norm_backward(tail, tail, w, pstats, wants=(True, False, False))[0])


# ---------------------------------------------------------------------------------- dropout
def _philox(block, seed):
    """One block of Philox4x32 with 10 rounds on Python integers."""
    mask = 0xFFFFFFFF
    c, k = [block & mask, block >> 32 & mask, 0, 0], [seed & mask, seed >> 32]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & mask, (p >> 32) ^ c[3] ^ k[1], p & mask]
        k = [(k[0] + 0x9E3779B9) & mask, (k[1] + 0xBB67AE85) & mask]
    return c


def _words(seed, offset, n):
    out = []
    for b in range(offset // 4, (offset + n + 3) // 4):
        out += _philox(b % (1 << 64), seed)
    return np.array(out[:n], dtype=np.uint64)


def test_generator_is_the_published_one():
    """The paper's test vector for a zero counter and key."""
    assert _philox(0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]


@pytest.mark.parametrize("seed,offset", [(0, 0), (12345, 4), (2 ** 64 - 1, 2 ** 34 - 8), (0xDEADBEEF00000001, 2 ** 64 - 4 * 200)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (1, 4), (3, 5), (7, 33), (4, 64), (2, 250), (16, 48)])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_dropout_draws_the_sequence(ndvm, cuda, rows, cols, seed, offset, t):
    import torch
    n = rows * cols
    g = _gen(n + 1)
    x, r = _randn(g, rows, cols).to(_t(t)), _randn(g, rows, cols).to(_t(t))
    keep_all = _words(seed, offset, n)
    for p in (0.0, 0.1, 0.5, 0.93, 1 - 2.0 ** -32):
        keep = torch.from_numpy(keep_all >= np.uint64(round(p * 2 ** 32))).to("cuda").view(rows, cols)
        scale = 1.0 / (1.0 - p)
        want = torch.where(keep, x.double() * scale, 0.0)
        big = want.abs() > torch.finfo(_t(t)).max * 0.99  # (p = 1 - 2^-32 leaves half's range)
        for res in (None, r):
            y = ndvm.dropout_forward(x, p, seed, offset, res)
            v = want if res is None else want + res.double()
            e = 3 * U * (want.abs() + v.abs())
            _inside(y[~big], v[~big], _rounded(v, e, t)[~big], f"p = {p}")
            assert torch.equal(y == 0, ~keep | (x == 0)) if res is None else torch.equal(y[~keep], res[~keep])


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1000, 1001), (4096, 513), (313, 4096)])
def test_dropout_strides_alignment_and_inplace(ndvm, cuda, rows, cols, t):
    """The mask goes by the row-major index whatever the layout; y may be x or the residual."""
    import torch
    g = _gen(rows)
    x, r = _randn(g, rows, cols).to(_t(t)), _randn(g, rows, cols).to(_t(t))
    want = ndvm.dropout_forward(x, 0.3, 77, 1 << 20, r)
    kept = (ndvm.dropout_forward(torch.ones_like(x), 0.3, 77, 1 << 20) != 0).float().mean()
    assert abs(float(kept) - 0.7) < 6 * math.sqrt(0.21 / (rows * cols))  # six standard deviations
    for pad, shift in ((8, 0), (3, 1), (5, 2)):
        out = torch.full((rows, cols + pad), 3.0, dtype=x.dtype, device="cuda")
        y = ndvm.dropout_forward(_strided(x, pad, shift), 0.3, 77, 1 << 20, _strided(r, 2 * pad, shift), out[:, shift:shift + cols])
        assert torch.equal(y, want)
        assert bool((out[:, :shift] == 3).all()) and bool((out[:, shift + cols:] == 3).all())
    flat = torch.empty(rows * cols + 1, dtype=x.dtype, device="cuda")[1:].view(rows, cols)
    flat.copy_(x)
    assert torch.equal(ndvm.dropout_forward(flat, 0.3, 77, 1 << 20, r), want)
    a, b = x.clone(), r.clone()
    assert torch.equal(ndvm.dropout_forward(a, 0.3, 77, 1 << 20, r, a), want)
    assert torch.equal(ndvm.dropout_forward(x, 0.3, 77, 1 << 20, b, b), want)
    # parts of a tensor with their own offsets draw what the whole draws
    half = rows // 4 * 4 // 2
    parts = [ndvm.dropout_forward(x[:half], 0.3, 77, 1 << 20, r[:half])]
    if half * cols % 4 == 0:
        parts.append(ndvm.dropout_forward(x[half:], 0.3, 77, (1 << 20) + half * cols, r[half:]))
    assert torch.equal(torch.cat(parts), want[:sum(p.shape[0] for p in parts)])


def test_dropout_of_values_that_are_not_finite(ndvm, cuda):
    import torch
    x = torch.full((64, 64), float("nan"), device="cuda", dtype=torch.bfloat16)
    x[::2] = float("inf")
    r = torch.ones_like(x)
    y = ndvm.dropout_forward(x, 0.5, 9, 0, r)
    keep = ndvm.dropout_forward(torch.ones_like(x), 0.5, 9) != 0
    assert bool((y[~keep] == 1).all()) and not bool(y[keep].isfinite().any())


def test_dropout_gradient(ndvm, cuda):
    """Linear in x and the residual, so a difference of two calls is the slope: exact powers of two."""
    import torch
    x = torch.ones(100, 37, device="cuda", requires_grad=True)
    r = torch.zeros(100, 37, device="cuda", requires_grad=True)
    y = ndvm.dropout(x, 0.5, 5, 400, r)
    dy = _randn(_gen(2), 100, 37)
    dx, dr = torch.autograd.grad(y, (x, r), dy)
    slope = ndvm.dropout_forward(2 * x.detach(), 0.5, 5, 400) - ndvm.dropout_forward(x.detach(), 0.5, 5, 400)
    assert torch.equal(dx, slope * dy) and torch.equal(dr, dy)
    assert torch.equal(dx, ndvm.dropout_backward(dy, 0.5, 5, 400))
    only = torch.autograd.grad(ndvm.dropout(x, 0.5, 5, 400), x, dy.new_ones(()).expand(100, 37))[0]  # cotangent of stride 0
    assert torch.equal(only, slope)


def test_dropout_past_32_bit_offsets(ndvm, cuda):
    import torch
    rows, cols = 65537, 65540
    x = torch.ones(rows, cols, dtype=torch.float16, device="cuda")
    ndvm.dropout_forward(x, 0.25, 31, 16, None, x)
    tail = ndvm.dropout_forward(torch.ones(9, cols, dtype=torch.float16, device="cuda"), 0.25, 31, 16 + (rows - 9) * cols)
    assert torch.equal(x[-9:], tail)


# ------------------------------------------------------------------------- gated projection
def _act64(name, g, eg):
    """act, act' and bounds of their errors when g is off by eg (|act'| <= 1.13, |act''| <= 1; the
    functions themselves to 16 U)."""
    import torch
    if name == "relu":
        a, da = g.clamp_min(0), (g > 0).double()
        return a, da, eg, (g.abs() <= eg).double()
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        a, da = g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        s = torch.sigmoid(g)
        a, da = (g * s, s * (1 + g * (1 - s))) if name == "silu" else (s, s * (1 - s))
    return a, da, 1.13 * eg + 16 * U * (a.abs() + g.abs() * 0.25 + (name == "sigmoid")), eg + 16 * U * (1 + g.abs())


def _gated64(x, wg, wu, dh, act, t):
    """h, dx, dw_gate, dw_up and their bounds.  Tensor-core sums may truncate: 2 U a term."""
    rows, k = x.shape
    n = wg.shape[0]
    ax = x.abs()
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = (2 * U * (k + 8) * (ax @ w.abs().t()) for w in (wg, wu))
    a, da, ea, eda = _act64(act, g, eg)
    h = a * u
    eh = ea * (u.abs() + eu) + a.abs() * eu + 4 * U * h.abs()
    dg, du = dh * u * da, dh * a
    edg = dh.abs() * (u.abs() * eda + eu * (da.abs() + eda)) + 4 * U * dg.abs()
    edu = dh.abs() * ea + 4 * U * du.abs()
    edg, edu = (_rounded(v, e, t) for v, e in ((dg, edg), (du, edu)))
    adg, adu = dg.abs() + edg, du.abs() + edu
    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + 2 * U * (2 * n + 8) * (adg @ wg.abs() + adu @ wu.abs())
    dws = [v.t() @ x for v in (dg, du)]
    ews = [e.t() @ ax + 2 * U * (rows + 8) * (s.t() @ ax) for e, s in ((edg, adg), (edu, adu))]
    return (h, dx, *dws), (eh, edx, *ews)


def _gated_case(seed, rows, k, n, t):
    g = _gen(seed)
    return (_randn(g, rows, k).to(_t(t)), (_randn(g, n, k) * k ** -0.5).to(_t(t)), (_randn(g, n, k) * k ** -0.5).to(_t(t)),
            _randn(g, rows, n).to(_t(t)))


GATED_SIZES = [(1, 1, 1), (1, 8, 16), (1, 2048, 640), (1, 333, 777), (2, 64, 64), (3, 100, 257), (4, 512, 130), (5, 7, 9),
               (8, 256, 2000), (9, 264, 72), (16, 1024, 512), (17, 65, 63), (31, 96, 129), (33, 40, 512), (64, 128, 128),
               (65, 72, 120), (100, 1000, 300), (127, 64, 256), (128, 63, 127), (129, 65, 129), (200, 520, 264),
               (256, 256, 256), (257, 130, 385), (300, 333, 777), (513, 200, 136), (1000, 48, 72), (2049, 16, 24),
               (5000, 120, 56)]


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", GATED_SIZES)
def test_gated_matches_64_bits(ndvm, cuda, rows, k, n, t):
    act = ["silu", "gelu", "relu", "sigmoid"][(rows + k + n) % 4]
    x, wg, wu, dh = _gated_case(rows * 7919 + k * 31 + n, rows, k, n, t)
    got = (ndvm.gated_forward(x, wg, wu, act),) + ndvm.gated_backward(dh, x, wg, wu, act)
    want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), act, t)
    for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), got, want, err):
        _inside(a, v, _rounded(v, e, t), name)
        # independent roundings (of dG or dU, then of the output) add up as squares: twice RMS would hold
        # them, three leaves the scatter of small outputs
        if v.numel() >= 64 and act != "relu":
            rel = float((a.double() - v).norm() / v.norm())
            assert rel <= 3 * RMS[t], (name, rel)


@pytest.mark.parametrize("rows,k,n", [(5003, 2008, 2601), (4999, 2003, 2600), (2300, 1024, 4100)])
def test_gated_of_many_tiles(ndvm, cuda, rows, k, n):
    """Sizes of several rounds of the largest tiles in every product, ragged at every edge."""
    import torch
    x, wg, wu, dh = _gated_case(rows, rows, k, n, "bf16")
    want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), "silu", "bf16")
    bounds = [_rounded(v, e, "bf16") for v, e in zip(want, err)]
    for kept in (None, ndvm.gated_kept(x, wg)):
        got = (ndvm.gated_forward(x, wg, wu, kept=kept),) + ndvm.gated_backward(dh, x, wg, wu, kept=kept)
        for name, a, v, b in zip(("h", "dx", "dw_gate", "dw_up"), got, want, bounds):
            _inside(a, v, b, name)
            assert float((a.double() - v).norm() / v.norm()) <= 3 * RMS["bf16"], name
    ndvm.check_operators()


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", GATED_SIZES[::2] + [(1, 40, 1001), (130, 72, 1001), (300, 1100, 136)])
def test_gated_with_kept_products(ndvm, cuda, rows, k, n, t):
    """The same bounds with the products kept; h has the bits of the call that keeps nothing."""
    import torch
    act = ["silu", "gelu", "relu", "sigmoid"][(rows + k + n) % 4]
    x, wg, wu, dh = _gated_case(rows * 7919 + k * 31 + n, rows, k, n, t)
    kept = ndvm.gated_kept(x, wg)
    h = ndvm.gated_forward(x, wg, wu, act, kept=kept)
    assert torch.equal(h, ndvm.gated_forward(x, wg, wu, act))
    for i, w in enumerate((wg, wu)):  # G and U themselves, in binary32
        exact = x.double() @ w.double().t()
        _inside(kept[i, :, :n], exact, 2 * U * (k + 8) * (x.double().abs() @ w.double().abs().t()), "kept")
    for d in (dh, _strided(dh, 3, 1)):
        got = (h,) + ndvm.gated_backward(d, x, wg, wu, act, kept=kept)
        want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), act, t)
        for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), got, want, err):
            _inside(a, v, _rounded(v, e, t), name)


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,k,n", [(1, 64, 16), (1, 48, 1000), (2, 2048, 640), (5, 33, 77), (64, 64, 64), (200, 80, 81), (900, 40, 50)])
def test_gated_gradients_of_few_elements_are_rounded_once(ndvm, cuda, rows, k, n, t):
    """Over few elements dG and dU are handed on in two halves (together 2^-15 or closer): the gradients are those
    of the binary32 chain with one rounding, so no further from the exact ones than half a unit in the last place and
    the small bounds of the halves and sums."""
    import torch
    x, wg, wu, dh = _gated_case(rows + 17 * n, rows, k, n, t)
    want, _ = _gated64(*(v.double() for v in (x, wg, wu, dh)), "silu", t)
    _, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), "silu", "f32")  # bounds without the 16-bit rounding between
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    a, da, _, _ = _act64("silu", g, 0)
    left = {"bf16": 2.0 ** -16, "f16": 2.0 ** -22}[t]  # of dG and dU; and half's smallest step
    dg, du = ((dh.double() * v).abs() * left + (2.0 ** -24 if t == "f16" else 0) for v in (u * da, a))
    more = (dg @ wg.double().abs() + du @ wu.double().abs(), dg.t() @ x.double().abs(), du.t() @ x.double().abs())
    for kept in (None, ndvm.gated_kept(x, wg)):
        ndvm.gated_forward(x, wg, wu, kept=kept)
        got = ndvm.gated_backward(dh, x, wg, wu, kept=kept)
        for name, b, v, e, m in zip(("dx", "dw_gate", "dw_up"), got, want[1:], err[1:], more):
            _inside(b, v, _rounded(v, e + m, t), name)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "sigmoid"])
@pytest.mark.parametrize("rows", [1, 6, 200])
def test_gated_activations(ndvm, cuda, act, rows):
    """Pre-activations from far below to far above zero (the functions' tails)."""
    x, wg, wu, dh = _gated_case(5, rows, 96, 264, "bf16")
    x = x * 12
    got = (ndvm.gated_forward(x, wg, wu, act),) + ndvm.gated_backward(dh, x, wg, wu, act)
    want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), act, "bf16")
    for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), got, want, err):
        _inside(a, v, _rounded(v, e, "bf16"), name)


@pytest.mark.parametrize("rows", [1, 7, 150])
@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 8), (3, 1), (1, 0)])
def test_gated_strides_and_alignment(ndvm, cuda, rows, pad, shift):
    import torch
    k, n, t = 136, 200, "bf16"
    x, wg, wu, dh = _gated_case(11, rows, k, n, t)
    want, err = _gated64(*(v.double() for v in (x, wg, wu, dh)), "silu", t)
    ho = torch.full((rows, n + pad), 3.0, dtype=x.dtype, device="cuda")
    dxo = torch.full((rows, k + pad), 3.0, dtype=x.dtype, device="cuda")
    xs, gs, us, ds = (_strided(v, pad, shift) for v in (x, wg, wu, dh))
    h = ndvm.gated_forward(xs, gs, us, "silu", h=ho[:, shift:shift + n])
    got = (h,) + ndvm.gated_backward(ds, xs, gs, us, "silu", dx=dxo[:, shift:shift + k])
    for name, a, v, e in zip(("h", "dx", "dw_gate", "dw_up"), got, want, err):
        _inside(a, v, _rounded(v, e, t), name)
    for o, m in ((ho, n), (dxo, k)):
        assert bool((o[:, :shift] == 3).all()) and bool((o[:, shift + m:] == 3).all())
    # a pair of weights that are one matrix, and inputs whose rows are all the same memory
    both = torch.cat((wg, wu))
    assert torch.equal(ndvm.gated_forward(x, both[:n], both[n:]), ndvm.gated_forward(x, wg, wu))
    same = x[:1].expand(rows, k)
    assert torch.equal(ndvm.gated_forward(same, wg, wu), ndvm.gated_forward(same.contiguous(), wg, wu))


@pytest.mark.parametrize("rows", [1, 5, 140])
def test_gated_partial_gradients(ndvm, cuda, rows):
    import torch
    x, wg, wu, dh = _gated_case(21, rows, 72, 136, "f16")
    full = ndvm.gated_backward(dh, x, wg, wu)
    for k in range(3):
        part = ndvm.gated_backward(dh, x, wg, wu, wants=tuple(i == k for i in range(3)))
        assert [p is None for p in part] == [i != k for i in range(3)]
        assert torch.equal(part[k], full[k])


def test_gated_of_no_rows(ndvm, cuda):
    import torch
    x, wg, wu, dh = _gated_case(22, 0, 24, 40, "bf16")
    assert ndvm.gated_forward(x, wg, wu).shape == (0, 40)
    dx, dg, du = ndvm.gated_backward(dh, x, wg, wu, dw_gate=torch.ones_like(wg), dw_up=torch.ones_like(wu))
    assert dx.shape == (0, 24) and not dg.any() and not du.any()


@pytest.mark.parametrize("rows", [4, 200])
def test_gated_rows_keep_their_own_values(ndvm, cuda, rows):
    """A row with an infinity or a NaN stays alone in h and dx; a weight row with one stays in its column."""
    import torch
    x, wg, wu, dh = _gated_case(23, rows, 80, 150, "bf16")
    h, (dx, _, _) = ndvm.gated_forward(x, wg, wu), ndvm.gated_backward(dh, x, wg, wu)
    bad = x.clone()
    bad[1, 3], bad[2, 79] = float("nan"), float("inf")
    rest = [i for i in range(rows) if i not in (1, 2)]
    hb, (dxb, _, _) = ndvm.gated_forward(bad, wg, wu), ndvm.gated_backward(dh, bad, wg, wu)
    assert torch.equal(hb[rest], h[rest]) and torch.equal(dxb[rest], dx[rest])
    assert bool(hb[1].isnan().all())
    wb = wg.clone()
    wb[149, 79] = float("nan")
    hw = ndvm.gated_forward(x, wb, wu)
    assert torch.equal(hw[:, :149], h[:, :149]) and bool(hw[:, 149].isnan().all())


def test_gated_gradient_against_differences(ndvm, cuda):
    """Directional slopes of the 64-bit definition (central differences) against the gradients' products
    with the direction: off by no more than the gradients' bounds along it."""
    import torch
    x, wg, wu, dh = _gated_case(31, 70, 90, 110, "f16")
    ins = [v.requires_grad_(True) for v in (x, wg, wu)]
    grads = torch.autograd.grad(ndvm.gated(*ins, "gelu"), ins, dh)
    base = [v.detach().double() for v in ins]
    want, err = _gated64(*base, dh.double(), "gelu", "f16")

    def f(x, wg, wu):
        return float((_act64("gelu", x @ wg.t(), 0)[0] * (x @ wu.t()) * dh.double()).sum())

    for k in range(3):
        v = _randn(_gen(40 + k), *ins[k].shape).double()
        plus, minus = [list(base) for _ in range(2)]
        plus[k], minus[k] = base[k] + 1e-4 * v, base[k] - 1e-4 * v
        slope, got = (f(*plus) - f(*minus)) / 2e-4, float((grads[k].double() * v).sum())
        bound = float((_rounded(want[k + 1], err[k + 1], "f16") * v.abs()).sum())
        assert abs(got - slope) <= bound + 1e-6 * float((want[k + 1] * v).abs().sum())
        assert abs(got - slope) <= 20 * ROUND["f16"] * float((want[k + 1] * v).norm())  # (and as independent roundings)


# ---------------------------------------------------------------------- calls and streams
def test_same_call_same_bits(ndvm, cuda):
    import torch
    x, wg, wu, dh = _gated_case(51, 700, 264, 520, "bf16")
    w = torch.ones(264, device="cuda")

    def once():
        y, stats = ndvm.layer_norm_forward(x, w, w)
        return (ndvm.gated_forward(x, wg, wu), *ndvm.gated_backward(dh, x, wg, wu), y, *ndvm.layer_norm_backward(x, x, w, stats))

    first = once()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, once()))


def test_another_stream_than_the_current_one(ndvm, cuda):
    """Calls on a side stream are ordered after the work queued there, and outputs belong to it."""
    import torch
    side = torch.cuda.Stream()
    x, wg, wu, dh = _gated_case(52, 300, 264, 520, "bf16")
    w = torch.ones(264, device="cuda", dtype=torch.bfloat16)
    want = ndvm.gated_forward(x, wg, wu), *ndvm.gated_backward(dh, x, wg, wu)
    yw, sw = ndvm.layer_norm_forward(x, w, w)
    dw = ndvm.dropout_forward(x, 0.2, 3)
    nw = ndvm.layer_norm_backward(x, x, w, sw)
    late = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        spin = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            spin = spin @ spin * 1e-3
        late.copy_(x)
    got = ndvm.gated_forward(late, wg, wu, stream=side), *ndvm.gated_backward(dh, late, wg, wu, stream=side)
    ys, ss = ndvm.layer_norm_forward(late, w, w, stream=side)
    ds = ndvm.dropout_forward(late, 0.2, 3, stream=side)
    ns = ndvm.layer_norm_backward(late, late, w, ss, stream=side)
    side.synchronize()
    for a, b in zip((*want, yw, dw, *nw), (*got, ys, ds, *ns)):
        assert torch.equal(a, b)


def test_graph_capture(ndvm, cuda):
    import torch
    x, wg, wu, dh = _gated_case(53, 150, 264, 136, "bf16")
    w = torch.ones(264, device="cuda", dtype=torch.bfloat16)

    def step():
        y, stats = ndvm.layer_norm_forward(x, w, w)
        h = ndvm.gated_forward(y, wg, wu)
        dx, dg, du = ndvm.gated_backward(ndvm.dropout_backward(dh, 0.1, 8), y, wg, wu)
        return (h, dg, du, *ndvm.layer_norm_backward(dx, x, w, stats))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, step()):
        assert torch.equal(a, b)


def test_differentiable_ops_take_any_layout(ndvm, cuda):
    """Leading dimensions, transposed inputs and broadcast cotangents give the raw calls' results."""
    import torch
    g = _gen(61)
    x = _randn(g, 5, 72, 6).bfloat16().permute(0, 2, 1).requires_grad_(True)  # (5, 6, 72), last dimension strided
    wg, wu = (_randn(g, 40, 72) * 0.1).bfloat16(), (_randn(g, 72, 40) * 0.1).bfloat16().t()
    w = _randn(g, 72).requires_grad_(True)
    y = ndvm.layer_norm(x, w)
    h = ndvm.gated(y, wg, wu, "sigmoid")
    z = ndvm.dropout(h, 0.0, 1, 0, h)
    z.sum().backward()
    x2 = x.detach().contiguous().view(30, 72)
    y2, stats = ndvm.layer_norm_forward(x2, w.detach())
    h2 = ndvm.gated_forward(y2, wg, wu.contiguous(), "sigmoid")
    assert torch.equal(z.detach().view(30, 40), h2 + h2)
    dy2 = ndvm.gated_backward(torch.full_like(h2, 2.0), y2, wg, wu.contiguous(), "sigmoid")[0]
    dx2, dw2, _ = ndvm.layer_norm_backward(dy2, x2, w.detach(), stats)
    assert torch.equal(x.grad.reshape(30, 72), dx2) and torch.equal(w.grad, dw2)


def test_empty_inputs_through_autograd(ndvm, cuda):
    import torch
    x = torch.empty(0, 24, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    w = torch.ones(24, device="cuda", requires_grad=True)
    g, u = (torch.ones(40, 24, device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(2))
    h = ndvm.dropout(ndvm.gated(ndvm.layer_norm(x, w), g, u), 0.1, 1)
    dx, dw, dg, du = torch.autograd.grad(h, (x, w, g, u), torch.empty_like(h))
    assert dx.shape == (0, 24) and not dw.any() and not dg.any() and not du.any()


def test_no_second_derivatives(ndvm, cuda):
    import torch
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    for y in (ndvm.layer_norm(x), ndvm.dropout(x, 0.5, 1)):
        with pytest.raises(ndvm.NdvmError):
            torch.autograd.grad(y, x, torch.ones_like(y), create_graph=True)


def test_refusals(ndvm, cuda):
    """Wrong types, shapes, layouts and values raise before any launch."""
    import torch
    x, wg, wu, dh = _gated_case(71, 8, 24, 40, "bf16")
    f = torch.ones(24, device="cuda")
    E = ndvm.NdvmError
    calls = [
        lambda: ndvm.layer_norm(x.double()),
        lambda: ndvm.layer_norm(x.cpu()),
        lambda: ndvm.layer_norm(torch.ones((), device="cuda")),
        lambda: ndvm.layer_norm(x, f[:23]),
        lambda: ndvm.layer_norm(x, f, f.bfloat16()),
        lambda: ndvm.layer_norm(x, f.half()),
        lambda: ndvm.layer_norm(x.float(), f.bfloat16()),
        lambda: ndvm.layer_norm(x, f.cpu()),
        lambda: ndvm.layer_norm(x, f, eps=-1e-3),
        lambda: ndvm.layer_norm(x, f, eps=float("nan")),
        lambda: ndvm.layer_norm(torch.empty(3, 0, device="cuda")),
        lambda: ndvm.layer_norm_forward(x.t()),
        lambda: ndvm.layer_norm_forward(x, y=torch.empty(8, 23, device="cuda", dtype=x.dtype)),
        lambda: ndvm.layer_norm_forward(x, y=x.new_empty(24).expand(8, 24)),
        lambda: ndvm.layer_norm_forward(x, stats=torch.empty(2, 7, device="cuda")),
        lambda: ndvm.layer_norm_backward(x[:7], x, f, torch.empty(2, 8, device="cuda")),
        lambda: ndvm.layer_norm_backward(x, x, f, torch.empty(2, 8, device="cuda"), dweight=f[:3]),
        lambda: ndvm.layer_norm_backward(x, x, f, torch.empty(2, 8, device="cuda"), workspace=f[:4]),
        lambda: ndvm.dropout(x, 1.0, 0),
        lambda: ndvm.dropout(x, -0.1, 0),
        lambda: ndvm.dropout(x, float("nan"), 0),
        lambda: ndvm.dropout(x, 0.1, -1),
        lambda: ndvm.dropout(x, 0.1, 1 << 64),
        lambda: ndvm.dropout(x, 0.1, 0, 2),
        lambda: ndvm.dropout(x, 0.1, 0, -4),
        lambda: ndvm.dropout(x, 0.1, 0, 0, x[:7]),
        lambda: ndvm.dropout(x, 0.1, 0, 0, x.float()),
        lambda: ndvm.dropout(x.double(), 0.1, 0),
        lambda: ndvm.dropout_forward(x, 0.1, 0, y=x.new_empty(24).expand(8, 24)),
        lambda: ndvm.gated(x, wg, wu, "tanh"),
        lambda: ndvm.gated(x.float(), wg.float(), wu.float()),
        lambda: ndvm.gated(x, wg, wu.half()),
        lambda: ndvm.gated(x, wg, wu[:39]),
        lambda: ndvm.gated(x[:, :23], wg, wu),
        lambda: ndvm.gated(x, wg, wu.cpu()),
        lambda: ndvm.gated_forward(x, wg.t().contiguous().t(), wu),
        lambda: ndvm.gated_forward(x, wg, wu, h=torch.empty(8, 41, device="cuda", dtype=x.dtype)),
        lambda: ndvm.gated_backward(dh[:, :39], x, wg, wu),
        lambda: ndvm.gated_backward(dh, x, wg, wu, workspace=f[:4]),
        lambda: ndvm.gated_backward(dh, x, wg, wu, dw_gate=wg[:, :23]),
        lambda: ndvm.gated_forward(x, wg, wu, kept=torch.empty(2, 8, 39, device="cuda")),
        lambda: ndvm.gated_backward(dh, x, wg, wu, kept=torch.empty(2, 8, 40, device="cuda").half()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(E):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
