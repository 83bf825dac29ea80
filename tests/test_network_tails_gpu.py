"""The gated projection's activations and their derivatives far from zero (GPU), where a formula that is right to a few
units near zero can lose every digit.

x holds a pre-activation g and a 1 in each row, the first row of w_gate picks the one and that of w_up the other, so G = g
and U = 1 exactly, h = act(g), dU = act(g) and dG = act'(g) (dh = 1), and dx = (dG, dU).

Bounds, derived from binary32 arithmetic (U = 2^-24): e^-|g| is the power of two of a product that is off by 1.3 U |g| in
all, itself off by up to 4 U; a sum, a reciprocal and a product or two follow, a few U each: 16 U (1 + |g|) of the value.
The normal distribution's density and tail: their logarithm moves by g^2 times the argument's 1.3 U; the tail itself
is off by 8 U: 16 U (1 + g^2).  Steps of 2^-149 (below 2^-126) are allowed for, times |g|; in dx, which a tensor core
adds up, anything below 2^-125.  Then one rounding to bfloat16 for h and two for dx.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16 = 2.0 ** -8


def _act(name, g):
    """act, act' and their bounds in binary32, in 64 bits."""
    import torch
    if name == "gelu":
        rel = 16 * U * (1 + g * g)
        cdf, bell = 0.5 * torch.erfc(-g / math.sqrt(2)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * cdf, cdf + g * bell, rel * (g * cdf).abs(), 2 * rel * (cdf + (g * bell).abs())
    rel = 16 * U * (1 + g.abs())
    s, rest = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    if name == "sigmoid":
        return s, s * rest, rel * s, 2 * rel * s * rest
    return g * s, s + g * s * rest, rel * (g * s).abs(), 2 * rel * (s + (g * s).abs() * rest)


def _check(got, want, err, tiny, roundings, what, g):
    for _ in range(roundings):
        err = err + BF16 * (want.abs() + err)
    over = (got.double() - want).abs() > err + tiny
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {over.numel()} outside; first at g = {float(g[over][0])}: "
                                  f"{float(got[over][0])}, not {float(want[over][0])}")


def _run(ndvm, act, values, n, keep):
    import torch
    g = torch.tensor(values, device="cuda", dtype=torch.bfloat16)
    x = torch.zeros(len(values), 8, device="cuda", dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = g, 1
    wg, wu = (torch.zeros(n, 8, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    wg[0, 0] = wu[0, 1] = 1
    kept = ndvm.gated_kept(x, wg) if keep else None
    h = ndvm.gated_forward(x, wg, wu, act, kept=kept)[:, 0]
    dx = ndvm.gated_backward(torch.ones(len(values), n, device="cuda", dtype=torch.bfloat16), x, wg, wu, act, kept=kept)[0]
    g = g.double()
    a, da, ea, eda = _act(act, g)
    step = (1 + g.abs()) * 2.0 ** -148
    _check(h, a, ea, step + 2.0 ** -133, 1, "h", g)
    _check(dx[:, 1], a, ea, step + 2.0 ** -125, 2, "dU", g)
    _check(dx[:, 0], da, eda, step + 2.0 ** -125, 2, "dG", g)


RANGES = {"gelu": [i / 16 for i in range(-13 * 16, 13 * 16 + 1)], "silu": [i / 2 for i in range(-200, 201)],
          "sigmoid": [i / 2 for i in range(-174, 201)]}


def _tails(act, n, repeat, keep, ndvm):
    _run(ndvm, act, [g for g in RANGES[act] for _ in range(repeat)], n, keep)


# n = 1: few elements, whose dG and dU go in halves; n = 264: rounded in between, G and U computed again or kept
SHAPES = [(1, 1), (264, 50)]


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("n,repeat", SHAPES)
def test_gelu_tails(ndvm, cuda, n, repeat, keep):
    _tails("gelu", n, repeat, keep, ndvm)


@pytest.mark.parametrize("g", [-12.0, -8.0, -5.0, 4.0])
def test_gelu_tails_of_one_row(ndvm, cuda, g):
    _run(ndvm, "gelu", [g], 1, False)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("n,repeat", SHAPES)
@pytest.mark.parametrize("act", ["silu", "sigmoid"])
def test_logistic_tails(ndvm, cuda, act, n, repeat, keep):
    _tails(act, n, repeat, keep, ndvm)


@pytest.mark.parametrize("act,g", [("silu", -95.0), ("silu", -88.0), ("silu", 30.0), ("sigmoid", -80.0), ("sigmoid", 25.0)])
def test_logistic_tails_of_one_row(ndvm, cuda, act, g):
    _run(ndvm, act, [g], 1, False)
