"""The dense layer in fp32: short contractions, numbers next to the smallest, and GELU."""
import math

import numpy as np
import pytest
import torch

from paper_2412_12218_amd import binding as B
from transformer_reference import S, check, f64

pytestmark = pytest.mark.gpu


def randn(n, d, seed, scale=1.0):
    return (torch.randn((n, d), generator=torch.Generator().manual_seed(seed)) * scale).cuda()


@pytest.mark.parametrize("few", [1, 2, 3, 4])
@pytest.mark.parametrize("rows,cols", [(70, 40), (300, 129), (2000, 1030)])
def test_sums_of_up_to_four_products(few, rows, cols):
    """Z of up to four features, dX of up to four results and dW of up to four rows: a rounding for each product (one: the product itself)."""
    def compare(name, got, x, y):
        want, ab = f64(x) @ f64(y), np.abs(f64(x)) @ np.abs(f64(y))
        check(f"{name} {few} {rows} {cols}", got, want, few * S * ab)
        if few == 1:
            assert torch.equal(got, x * y), name
    for odd in (0, 1):
        cols_ = cols + odd
        X, W = randn(rows, few, 1), randn(few, cols_, 2)
        compare("Z", B.ftc_linear(X, W), X, W)
        G, W = randn(rows, few, 3), randn(cols_, few, 4)
        compare("dX", B.ftc_linear_backward(randn(rows, cols_, 5), W, G, want_dW=False, want_db=False)[0], G, W.t())
        X, G = randn(few, rows, 6), randn(few, cols_, 7)
        compare("dW", B.ftc_linear_backward(X, randn(rows, cols_, 8), G, want_dX=False, want_db=False)[1], X.t(), G)


@pytest.mark.parametrize("n,d_in,d_out", [(70, 64, 128), (300, 33, 65), (2900, 72, 1028), (2561, 35, 1537), (5, 5000, 70)])
def test_small_numbers(n, d_in, d_out):
    """Numbers below 2^-110 against others of 2^100: held to 2^-134, half a step of the smallest bf16 numbers, in every row or in some of them.  Those of
    2^-108 are held in 24 bits."""
    def sized(n, d, seed):
        t = randn(n, d, seed)
        return torch.sign(t) * (t.abs() % 1.0 + 0.5)    # no number far below the others
    for least, every in ((-118, 1), (-118, 37), (-124, 1), (-108, 1)):
        X, W, G = sized(n, d_in, 1), sized(d_in, d_out, 2) * 2.0 ** 100, sized(n, d_out, 3)
        small = torch.where(torch.arange(n, device="cuda") % every == 0, 2.0 ** least, 2.0 ** -100)[:, None]
        X, G = X * small, G * small
        dX = B.ftc_linear_backward(X, W, G, want_dW=False, want_db=False)[0]
        dW = B.ftc_linear_backward(X * 2.0 ** 100 * 2.0 ** 100, W, G, want_dX=False, want_db=False)[1]
        x, w, g = f64(X), f64(W), f64(G)
        for name, got, a, b in (("Z", B.ftc_linear(X, W), x, w), ("dX", dX, g, w.T), ("dW", dW, x.T * 2.0 ** 200, g)):
            held = 2.0 ** -134 * (np.abs(a) < 2.0 ** -109) if name != "dW" else np.zeros_like(a)
            other = 2.0 ** -134 * (np.abs(b) < 2.0 ** -109) if name == "dW" else np.zeros_like(b)
            bound = np.abs(a) @ np.abs(b) * (a.shape[1] + 8) * S + held @ np.abs(b) + np.abs(a) @ other
            check(f"{name} {n} {d_in} {d_out} 2^{least} every {every}", got, a @ b, bound)


def test_gelu():
    """GELU and its slope at numbers between -9 and 9 in fp32.  z = p Phi(p): Phi(-a) = erfc(a / sqrt 2) / 2 is off by some steps (given eight) and by
    that of its argument, whose rounding (half a step, twice) moves it by a^2 half steps; Phi(a) = 1 - Phi(-a).  The slope adds p phi(p), off by a few steps and, by its
    exponent's rounding, by p^2 / 2."""
    p = torch.linspace(-9, 9, 65_536 + 7)
    n, few = 5, p.numel()
    X, W, slope = torch.zeros((n, 3), device="cuda"), torch.zeros((3, few), device="cuda"), torch.empty((n, few), device="cuda")
    out = B.ftc_linear(X, W, bias=p.cuda(), act=B.FTC_ACT_GELU, slope=slope)
    one = B.ftc_linear(X[:1], W, bias=p.cuda(), act=B.FTC_ACT_GELU)
    q = p.double()
    cdf, pdf = 0.5 * torch.erfc(-q / math.sqrt(2)), torch.exp(-0.5 * q * q) / math.sqrt(2 * math.pi)
    small = 0.5 * torch.erfc(q.abs() / math.sqrt(2))
    off_cdf = (8 + 2 * q * q) * S * small + torch.where(q > 0, 2 * S, 0.0)
    bound = q.abs() * off_cdf + 4 * S * (q * cdf).abs() + 2.0 ** -140
    for got in (out, one):
        check("GELU", got, (q * cdf).expand(got.shape).numpy(), bound.expand(got.shape).numpy())
    steep = off_cdf + q.abs() * pdf * (8 + 2 * q * q) * S + 4 * S * (cdf + q * pdf).abs() + 2.0 ** -140
    check("slope", slope, (cdf + q * pdf).expand(slope.shape).numpy(), steep.expand(slope.shape).numpy())
