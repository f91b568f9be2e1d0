"""Norms of rows whose mean is large beside their spread, of equal numbers, and of numbers at the ends of fp32, with bounds that are small beside the results."""
import numpy as np
import pytest
import torch

from block_rows import block, tight
from paper_2412_12218_amd import binding as B
from test_gpu_block_norm import DTYPES, KINDS, matrix, vector
from transformer_reference import check

pytestmark = pytest.mark.gpu
WIDTHS = [3, 20, 96, 250, 300, 768, 1100, 2052, 3077, 5000, 9000, 16384]


def layer_norm(X, w=None, b=None, eps=1e-5, **k):
    stats = torch.empty((X.shape[0], 4), device="cuda")
    _, U = B.ftc_block_norm(X, pre=B.FTC_NORM_LAYER, pre_w=w, pre_b=b, eps=eps, stats=stats, **k)
    return U, stats


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_equal_numbers(dtype, d):
    """Their mean is one of them: the first step is off by at most 40 roundings of it, the second by as many of that, so their sum rounds to the mean itself, all
    distances are zeros and what comes out is the bias, whatever eps is."""
    w, b = vector(d, dtype, 1, 1.0), vector(d, dtype, 2, 0.0)
    values = torch.tensor([3.5, 1000.0, -0.1, 6e4, 1e-3, 0.0, -333.25, 7e-6], device="cuda")
    X = values[:, None].expand(-1, d).to(dtype).contiguous()
    for eps in (1e-5, 1e-12, 1e-30):
        U, stats = layer_norm(X, w, b, eps)
        assert torch.equal(U, b.expand(8, d)), (U - b).abs().max(1).values.tolist()
        assert torch.equal(stats[:, 2], X[:, 0].float())
        want = 1 / np.sqrt(np.float64(np.float32(eps)))
        check(f"factor {dtype} {d} {eps}", stats[:, 3], np.full(8, want), np.full(8, want * 2.0 ** -22))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_mean_beside_a_small_spread(monkeypatch, dtype, d):
    means = [(1000.0, 0.5), (-30000.0, 30.0), (3.0, 1e-3), (0.3, 1.0)] + ([(1e5, 1.0), (1e30, 1e26)] if dtype == torch.float32 else [])
    X = torch.stack([matrix(1, d, torch.float32, i, scale=spread, mean=mean)[0] for i, (mean, spread) in enumerate(means)]).to(dtype)
    n = len(means)
    w, b = vector(d, dtype, 1, 1.0), vector(d, dtype, 2, 0.0)
    want = block(monkeypatch, X, None, 1.0, "none", None, None, None, "layer", w, b)
    U, stats = layer_norm(X, w, b)
    check(f"U {dtype} {d}", U, *want["U"])
    check(f"stats {dtype} {d}", stats, *want["stats"])
    for i in range(n if d >= 20 else 0):
        tight(f"row {i}", want["U"][0][i], want["U"][1][i], 0.15)
    if dtype == torch.float32:
        return
    # through a block: h has the mean, in fp32
    F, x_scale = matrix(n, d, dtype, 9, scale=0.3), 0.875
    dU = matrix(n, d, dtype, 10)
    want = block(monkeypatch, X, F, x_scale, "none", None, None, None, "layer", w, b, dU=dU)
    H, U = B.ftc_block_norm(X, F=F, x_scale=x_scale, pre=B.FTC_NORM_LAYER, pre_w=w, pre_b=b, stats=stats)
    check(f"H {dtype} {d}", H, *want["H"])
    check(f"U of a block {dtype} {d}", U, *want["U"])


@pytest.mark.parametrize("d", WIDTHS)
def test_gradient_beside_a_mean(monkeypatch, d):
    X = torch.stack([matrix(1, d, torch.float32, i, scale=spread, mean=mean)[0] for i, (mean, spread) in enumerate([(1000.0, 0.5), (-50.0, 1.0), (3.0, 0.01)] * 7)])
    w, dU = vector(d, torch.float32, 1, 1.0), matrix(21, d, torch.float32, 2)
    want = block(monkeypatch, X, None, 1.0, "none", None, None, None, "layer", w, None, dU=dU)
    _, stats = layer_norm(X, w)
    g = B.ftc_block_norm_backward(X, stats, dU=dU, pre=B.FTC_NORM_LAYER, pre_w=w)
    check(f"dX {d}", g.dX, *want["dX"])
    check(f"dw {d}", g.dpre_w, *want["dpre_w"])


def test_the_row_beside_it_does_not_matter():
    """Rows that need another sum (equal numbers, beyond 1e19, NaN) share a wave with rows that do not."""
    for d in (20, 96, 250, 500, 1100):
        X = matrix(40, d, torch.float32, 1, mean=0.5)
        alone = layer_norm(X)[0]
        for i, row in enumerate((7.0, 0.1, float("nan"), float("inf"))):
            X[3 + 9 * i] = row
        X[39] *= 1e25
        U, _ = layer_norm(X)
        keep = [i for i in range(39) if i not in (3, 12, 21, 30)]
        assert torch.equal(U[keep], alone[keep]) and bool((U[[3, 12]] == 0).all()) and bool(U[[21, 30]].isnan().all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_large_eps(kind):
    """Squares beyond fp32 beside an eps that counts: 1 / sqrt(v + eps) is as the formula has it."""
    X = torch.tensor([[1.5e19, -1.5e19, 1e19, -1e19], [3e19, -3e19, 2e19, -2e19], [1.0, 2.0, 3.0, 4.0], [1e19, -1e19, 0.0, 0.0]], device="cuda")
    for eps in (3e38, 1e38, 1e36):
        x, e = X.double().cpu().numpy(), float(np.float32(eps))
        mean = x.mean(1, keepdims=True) if kind == "layer" else 0.0
        r = 1 / np.sqrt(((x - mean) ** 2).mean(1) + e)
        stats = torch.empty((4, 4), device="cuda")
        _, U = B.ftc_block_norm(X, pre=KINDS[kind], eps=eps, stats=stats)
        check(f"factor {kind} {eps}", stats[:, 3], r, r * 2.0 ** -20)     # 1 / sqrt of a sum of five: ten roundings at most
        check(f"U {kind} {eps}", U, (x - mean) * r[:, None], np.abs((x - mean) * r[:, None]) * 2.0 ** -19 + 2.0 ** -40)
