"""The dense layer in fp32: short contractions."""
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
