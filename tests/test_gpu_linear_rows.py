"""The dense layer of one to four rows on either side of what sends them to kernels of their own (csrc/dense_plan.hpp: dense_few_rows)."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from test_gpu_linear import ACTS, DTYPES, layer, matrix
from transformer_reference import check, linear, linear_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", [(1, 4096, 1024), (1, 4096, 1025), (1, 4097, 40), (2, 2048, 48), (2, 2049, 48), (1, 1024, 16_384), (1, 1025, 16_384), (3, 64, 64),
                                          (1, 5000, 4096), (1, 5000, 4090), (2, 3000, 4096), (1, 20_000, 17)])
def test_forward(dtype, n, d_in, d_out):
    for act in ("none", "gelu"):
        X, W, b, R = layer(n, d_in, d_out, dtype, act, seed=n, bias=True, residual=act != "none")
        out = B.ftc_linear(X, W, bias=b, act=ACTS[act], residual=R)
        z, dz = linear(X, W, b, act, R, dtype)[:2]
        check(f"Z {dtype} {n} x {d_in} -> {d_out} {act}", out, z, dz)
        assert torch.equal(out, B.ftc_linear(X, W, bias=b, act=ACTS[act], residual=R))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", [(1, 40, 8192), (1, 40, 8193), (2, 2048, 8192), (2, 2049, 8192), (3, 40, 4096), (4, 40, 4097), (4, 4096, 4096), (4, 4097, 4096), (5, 64, 64),
                                          (4, 1000, 8192), (4, 1000, 8200), (3, 1100, 8300), (2, 17, 20_000)])
def test_input_gradient(dtype, n, d_in, d_out):
    X, W, _, _ = layer(n, d_in, d_out, dtype, "none", seed=n, bias=False, residual=False)
    G, add = matrix(n, d_out, dtype, 9), matrix(n, d_in, dtype, 10)
    only = dict(want_dW=False, want_db=False)
    want, bound = linear_backward(X, W, G, None, dtype, dtype)[0]
    check(f"dX {dtype} {n} x {d_in} <- {d_out}", B.ftc_linear_backward(X, W, G, **only)[0], want, bound)
    there = add.clone()
    B.ftc_linear_backward(X, W, G, dX_add=there, dX=there, **only)
    assert torch.equal(there, B.ftc_linear_backward(X, W, G, dX_add=add, **only)[0])
