"""The network operators give the same bits every time (GPU): a piece of an operand that is overwritten while it is read shows as
a few elements that differ once in some ten calls."""
import pytest

from test_network_gpu import _gated_case, _inside, _randn, _rounded, _gen
from test_network_linear_gpu import _backward64

pytestmark = pytest.mark.gpu


def _repeat(call, times):
    import torch
    first = [t.clone() for t in call()]
    for i in range(times):
        other = torch.empty(1 << (16 + i % 6), device="cuda")  # (the next outputs lie elsewhere)
        for k, (a, b) in enumerate(zip(first, call())):
            assert torch.equal(a, b), f"call {i}, output {k}: {int((a != b).sum())} elements differ"
        del other


@pytest.mark.parametrize("rows,k,n", [(2300, 1024, 4100), (4096, 1024, 4096), (5003, 2008, 2601), (513, 200, 136)])
def test_gated_same_bits(ndvm, cuda, rows, k, n):
    x, wg, wu, dh = _gated_case(rows, rows, k, n, "bf16")
    kept = ndvm.gated_kept(x, wg)
    _repeat(lambda: (ndvm.gated_forward(x, wg, wu), *ndvm.gated_backward(dh, x, wg, wu)), 200)
    _repeat(lambda: (ndvm.gated_forward(x, wg, wu, kept=kept), *ndvm.gated_backward(dh, x, wg, wu, kept=kept)), 100)
    ndvm.check_operators()


@pytest.mark.parametrize("rows,k,n", [(2300, 1024, 4100), (4096, 1024, 4096), (16384, 256, 2048), (3000, 64, 6000), (513, 200, 136)])
def test_linear_same_bits(ndvm, cuda, rows, k, n):
    x, w, b, res = (_randn(_gen(rows + i), *s).bfloat16() for i, s in enumerate(((rows, k), (n, k), (n,), (rows, n))))
    q, p = ndvm.quantize_forward(x), ndvm.quantize_forward(w)

    def step(act, keep):
        kept = ndvm.linear_kept(x, w, keep) if act else None
        y = ndvm.linear_forward(x, w, b, act, res, kept=kept)
        return (y, *ndvm.linear_backward(res, q if keep else x, w, act, kept=kept))

    for act, keep in (("silu", None), ("gelu", "8bit"), (None, None)):
        _repeat(lambda: step(act, keep), 100)
    _repeat(lambda: (ndvm.linear_quantized_forward(q, p, b, "gelu", res), ndvm.quantize_forward(x).dequantize()), 100)
    ndvm.check_operators()


@pytest.mark.parametrize("rows,cols", [(16384, 1024), (5000, 2048), (3001, 1537), (777, 8200)])
def test_rms_norm_same_bits(ndvm, cuda, rows, cols):
    x, res, dy, ds = (_randn(_gen(rows + i), rows, cols).bfloat16() for i in range(4))
    w = _randn(_gen(cols), cols)

    def step():
        y, s, rstd = ndvm.rms_norm_forward(x, w, 1e-6, res)
        return (y, s, *ndvm.rms_norm_backward(dy, s, w, rstd, ds), ndvm.rms_norm_quantized_forward(x, w, 1e-6, res)[0].dequantize())

    _repeat(step, 100)


# Sizes whose two gradients share units, one with binary32 sums that are split (dw, or of few rows dx) and, right after them, the
# other's 16-bit results: the staging of the one must have been read when it takes the other.  By the rule that cuts them
# (parts of dw, parts of dx; how many units go from sums to results): 16384 x 1024 -> 64 (8, 1; 32), 16384 x 3357 -> 264 (2, 1; 84),
# 150 x 1001 -> 4096 (1, 8; 64), 3 x 2000 -> 4096 in halves (1, 4; 32).
SHARED = [(16384, 1024, 64, None), (16384, 3357, 264, "silu"), (150, 1001, 4096, None), (3, 2000, 4096, "gelu")]


@pytest.mark.parametrize("rows,k,n,act", SHARED)
def test_linear_gradients_of_shared_units(ndvm, cuda, rows, k, n, act):
    """Against 64 bits, against each gradient alone, and again and again; into rows off 16 bytes too, which are not stored by copies."""
    import torch
    g = _gen(rows + k + n)
    x, w, dy = _randn(g, rows, k).bfloat16(), (_randn(g, n, k) * k ** -0.5).bfloat16(), _randn(g, rows, n).bfloat16()
    kept = ndvm.linear_kept(x, w) if act else None
    ndvm.linear_forward(x, w, None, act, kept=kept)
    got = ndvm.linear_backward(dy, x, w, act, kept=kept)
    z = kept[:, :n].double() if act else dy.double()
    want, err = _backward64(x.double(), w.double(), z, 0 * z, dy.double(), act, "bf16")
    for name, a, v, e in zip(("dx", "dw", "dbias"), got, want, err):
        _inside(a, v, _rounded(v, e, "bf16"), name)
    for i in range(3):
        assert torch.equal(ndvm.linear_backward(dy, x, w, act, wants=[i == j for j in range(3)], kept=kept)[i], got[i])
    wide = torch.full((rows, k + 3), 7.0, device="cuda").bfloat16()
    again = ndvm.linear_backward(dy, x, w, act, dx=wide[:, 1:1 + k], kept=kept)
    assert all(torch.equal(a, b) for a, b in zip(again, got)) and bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + k:] == 7).all())
    _repeat(lambda: ndvm.linear_backward(dy, x, w, act, kept=kept), 100)
    _repeat(lambda: ndvm.linear_backward(dy, x, w, act, dx=wide[:, 1:1 + k], kept=kept), 100)
    ndvm.check_operators()
