"""Grouped dense layers whose last tiles of 256 come in parts of the contraction, beyond 512 groups too, and whose weight gradients are joined from parts (that these layers
do: test_grouped_tail_host.py), against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from block_reference import grouped, grouped_backward
from grouped_tail_layers import JOINED, MANY, TAILS, many_lengths
from paper_2412_12218_amd import binding as B
from test_gpu_grouped_linear import DTYPES, layer, matrix, offsets
from transformer_reference import HALF_STEP, S, TINY, check, slope_values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens,d_in,d_out", TAILS, ids=str)
def test_last_tiles_in_parts(dtype, lens, d_in, d_out):
    ptr = np.cumsum([0] + lens).tolist()
    n = ptr[-1]
    X, W, b, R = layer(n, len(lens), d_in, d_out, dtype)
    slope = B.slope_like(R[:, :d_out].contiguous())
    ws = B._workspace(max(f(n, len(lens), d_in, d_out) for f in (B.lib().ftc_grouped_linear_workspace_bytes, B.lib().ftc_grouped_linear_backward_workspace_bytes)), "cuda")
    ws.fill_(255)      # NaN wherever a part would be read that nobody wrote
    out = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_SILU, residual=R, slope=slope, ws=ws)
    dZ, add = matrix(n, d_out, dtype, 5), matrix(n, d_in, dtype, 6)
    ws.fill_(255)
    dX = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, want_dW=False, want_db=False, ws=ws)[0]
    assert bool(out.isfinite().all()) and bool(dX.isfinite().all())
    assert torch.equal(out, B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_SILU, residual=R, ws=ws))
    wide = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dX_add=add, dx_dtype=torch.float32, want_dW=False, want_db=False)[0]
    B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dX_add=add, dX=add, want_dW=False, want_db=False)
    assert torch.equal(add, wide.to(dtype))
    # both sides of every border of a group, and rows in all tiles
    rows = torch.cat([torch.arange(max(0, p - 5), min(n, p + 5)) for p in ptr] + [torch.arange(13, n, 61)]).unique()
    for g, (a, e) in enumerate(zip(ptr, ptr[1:])):
        at = rows[(rows >= a) & (rows < e)].cuda()
        if len(at):
            (z, dz), (s, ds), _ = grouped(X[at], W[g:g + 1], [0, len(at)], b[g:g + 1], "silu", R[at], dtype)
            check(f"Z {g}", out[at], z, dz)
            assert np.all(np.abs(slope_values(slope[at]) - s) <= ds)
            want, bound = grouped_backward(X[at], W[g:g + 1], [0, len(at)], dZ[at], slope[at], dtype, dtype)[0]
            check(f"dX {g}", dX[at], want, bound)


@pytest.mark.parametrize("n,groups,d_in,d_out", MANY)
def test_many_groups_with_a_tail(n, groups, d_in, d_out):
    """Every row: sums of products of 16-bit numbers, off by at most (terms + 8) half steps of fp32 of their absolute sum, and a rounding."""
    dtype, lens = torch.bfloat16, many_lengths(n, groups)
    ptr = np.cumsum([0] + lens).tolist()
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    X, dZ, W = new(n, d_in), new(n, d_out), (new(groups, d_in, d_out) * d_in ** -0.5)
    b = new(groups, d_out)
    out = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b)
    dX = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, want_dW=False, want_db=False)[0]
    worst = 0.0
    for g, (a, e) in enumerate(zip(ptr, ptr[1:])):
        if a == e:
            continue
        w = W[g].double()
        for got, x, m, c in ((out, X, w, b[g].double()), (dX, dZ, w.t().contiguous(), 0.0)):
            x = x[a:e].double()
            want, size = x @ m + c, x.abs() @ m.abs() + (c.abs() if torch.is_tensor(c) else 0.0)
            bound = (m.shape[0] + 8) * S * size
            worst = max(worst, float(((got[a:e].double() - want).abs() / (bound + (want.abs() + bound) * HALF_STEP[dtype] + TINY[dtype])).max()))
            assert worst <= 1, (g, worst)
    print(worst)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,d_in,d_out", JOINED, ids=str)
def test_joined_weight_gradients(dtype, lens, d_in, d_out):
    ptr = np.cumsum([0] + lens).tolist()
    X, W, b, _ = layer(ptr[-1], len(lens), d_in, d_out, dtype, residual=False)
    slope = B.slope_like(X.new_empty((ptr[-1], d_out)))
    B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_GELU, slope=slope)
    dZ = matrix(ptr[-1], d_out, dtype, 5)
    for dt in {dtype, torch.float32}:
        for s in (slope, None):
            want = grouped_backward(X, W, ptr, dZ, s, dtype, dt)
            around = torch.full((2 + len(lens) * d_in * d_out,), 7.0, dtype=dt, device="cuda")
            dW = around[1:-1].view(len(lens), d_in, d_out)
            dX, _, db = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=s, dW=dW)
            for name, got, (value, bound) in zip(("dX", "dW", "db"), (dX, dW, db), want):
                check(f"{name} {dtype} -> {dt}", got, value, bound)
            assert around[0].item() == 7 and around[-1].item() == 7
