"""Error bounds of the gates and of the softmax exponentials from the
instructions that the kernels use, held against the bounds of seq_ref (stated
there for __expf and a 2-ulp division, and a little wider).

u = 2^-24.  Published errors: ex2.approx 2^-22 of the value (4 u), rcp.approx
2^-23 (2 u), products, sums and differences u each; log2(e) as a float is off by
0.23 u.

Gate: y = -z log2(e) carries 1.23 u |y|, so e = 2^y is off by (4 + 1.23 |z|) u;
r = 1 / (1 + e) adds u and 2 u, f = r - 2^-126 and 1 - f = e r one u more.  So f
and 1 - f are relatively accurate to (8 + 1.23 |z|) u, as long as 2^-126 is
nothing beside them: f from z = -70 on (f = 2^-101), 1 - f up to z = 87, where
exponentials below 2^-126 are flushed.  Beyond that the error is 2^-126 itself.

Softmax: (s - m) k with k = (1 / tau) log2(e) carries 4.23 u of itself (the
difference, the reciprocal, two products and the constant), its exponential 4 u."""
import math

import torch

import seq_ref as R

GATE = lambda z: (8 + 1.23 * z.abs()) * R.U  # noqa: E731
LEAST = 2.0 ** -126


def exponent(y):
    return (4 + 4.23 * y.abs()) * R.U


def test_the_constant():
    c = torch.tensor(math.log2(math.e), dtype=torch.float64)
    assert abs(float(c.float().double() / c - 1)) <= 0.23 * R.U


def test_seq_ref_covers_the_kernels_arithmetic():
    z = torch.linspace(-100, 100, 4001, dtype=torch.float64)
    assert bool((GATE(z) <= R.gate_error(z)).all()) and LEAST < R.TINY
    y = torch.linspace(0, 200, 4001, dtype=torch.float64)
    assert bool((exponent(y) <= (3 + 1.16 * y) * R.ULP + 4 * R.U * y).all())  # of each entry in seq_ref.distill


def test_gates_in_fp32_steps():
    """The kernel's steps in fp32 with a correctly rounded exponential and reciprocal stay within the bound."""
    z = torch.linspace(-100, 100, 200001, dtype=torch.float64).float()
    y = (z * torch.tensor(-math.log2(math.e)).float()).clamp(max=126.0)
    e = torch.exp2(y.double()).float()
    e = torch.where(e < LEAST, 0.0, e)
    r = (1 / (1 + e).double()).float()
    f, g = r - LEAST, e * r
    ef, eg = 1 / (1 + torch.exp(-z.double())), 1 / (1 + torch.exp(z.double()))
    zd = z.double()
    for got, exact, accurate in ((f, ef, zd >= -70), (g, eg, zd <= 87)):
        lim = GATE(zd) * exact + torch.where(accurate, 0.0, LEAST)
        assert bool(((got.double() - exact).abs() <= lim).all())
