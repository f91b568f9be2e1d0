"""The dense layer with bias, activation and residual, and its gradients, against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2412_12218_amd import binding as B
from transformer_reference import check, f64, linear, linear_backward, slope_values

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = dict(none=B.FTC_ACT_NONE, relu=B.FTC_ACT_RELU, gelu=B.FTC_ACT_GELU, silu=B.FTC_ACT_SILU)


def matrix(n, d, dtype, seed, ld=None, shift=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    ld = ld or d
    whole = (torch.randn(n * ld + shift, generator=gen) * scale).to(dtype).cuda()
    return whole[shift:].view(n, ld)[:, :d]


def layer(n, d_in, d_out, dtype, act, seed=0, bias=True, residual=True, ldx=None, shift=0):
    X = matrix(n, d_in, dtype, seed, ldx, shift)
    W = matrix(d_in, d_out, dtype, seed + 1, scale=d_in ** -0.5)
    b = matrix(1, d_out, dtype, seed + 2)[0].contiguous() if bias else None
    R = matrix(n, d_out, dtype, seed + 3, d_out + 1) if residual else None
    return X, W, b, R


SIZES = [(1, 1, 1), (1, 1024, 300), (2, 5001, 33), (4, 700, 90), (2, 40, 17000), (3, 8, 5), (17, 33, 65), (64, 64, 64), (65, 63, 67), (130, 100, 129), (200, 129, 40), (257, 520, 264), (5, 2000, 70),
         (1500, 16, 9), (2, 7, 1030)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_forward_and_slope(dtype, n, d_in, d_out):
    for i, act in enumerate(ACTS):
        X, W, b, R = layer(n, d_in, d_out, dtype, act, seed=i, bias=i % 2 == 0, residual=i >= 2, ldx=d_in + 3 * (i % 2), shift=i % 3)
        for out_dtype in {dtype, torch.float32}:
            slope = torch.full((n, d_out + 2), 7, device="cuda", dtype=B.slope_like(X).dtype)[:, :d_out]
            out = torch.full((n, d_out + 3), 7.0, device="cuda", dtype=out_dtype)[:, :d_out]
            B.ftc_linear(X, W, bias=b, act=ACTS[act], residual=R, out=out, slope=slope)
            z, dz, s, ds, dp, p = linear(X, W, b, act, R, out_dtype)
            check(f"Z {dtype} {n} {d_in} {d_out} {act} -> {out_dtype}", out, z, dz)
            got = slope_values(slope)
            sure = np.abs(p) > dp if act == "relu" else np.ones_like(p, bool)   # a sum next to zero may fall to either side
            assert np.all(np.abs(got - s)[sure] <= ds[sure])
            assert bool((out.as_strided((n, d_out + 3), (d_out + 3, 1))[:, d_out:] == 7).all())
            assert bool((slope.as_strided((n, d_out + 2), (d_out + 2, 1))[:, d_out:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES + [(9000, 24, 40), (3000, 257, 12)])
def test_backward(dtype, n, d_in, d_out):
    for act in ("none", "gelu"):
        X, W, b, _ = layer(n, d_in, d_out, dtype, act, seed=7, residual=False, ldx=d_in + 1)
        dZ = matrix(n, d_out, dtype, 99, d_out + 3, 1)
        slope = None
        if act != "none":
            slope = B.slope_like(dZ)
            B.ftc_linear(X, W, bias=b, act=ACTS[act], slope=slope)
        for wide in (False, True):
            dt = torch.float32 if wide else dtype
            dX = torch.full((n, d_in + 5), 7.0, device="cuda", dtype=dt)[:, :d_in]
            dX, dW, db = B.ftc_linear_backward(X, W, dZ, slope=slope, dX=dX, dw_dtype=dt)
            for name, got, (want, bound) in zip(("dX", "dW", "db"), (dX, dW, db), linear_backward(X, W, dZ, slope, dt, dt)):
                check(f"{name} {dtype} {n} {d_in} {d_out} {act} -> {dt}", got, want, bound)
            assert bool((dX.as_strided((n, d_in + 5), (d_in + 5, 1))[:, d_in:] == 7).all())
            again = B.ftc_linear_backward(X, W, dZ, slope=slope, dx_dtype=dt, dw_dtype=dt)
            assert all(torch.equal(x, y) for x, y in zip(again, (dX, dW, db)))


def test_parts_of_the_gradient():
    X, W, b, _ = layer(70, 40, 50, torch.float16, "silu", residual=False)
    slope = torch.empty((70, 50), dtype=torch.int16, device="cuda")
    B.ftc_linear(X, W, bias=b, act=B.FTC_ACT_SILU, slope=slope)
    dZ = matrix(70, 50, torch.float16, 5)
    dX, dW, db = B.ftc_linear_backward(X, W, dZ, slope=slope)
    only = lambda **k: B.ftc_linear_backward(X, W, dZ, slope=slope, **{**dict(want_dX=False, want_dW=False, want_db=False), **k})
    assert torch.equal(only(want_dX=True)[0], dX) and torch.equal(only(want_dW=True)[1], dW) and torch.equal(only(want_db=True)[2], db)
    assert only() == (None, None, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 3, 70])
def test_gradient_beside_a_residual_connection(dtype, n):
    """dX_add, apart from dX and in place: as the sum, which has one rounding more than the product."""
    X, W, b, _ = layer(n, 40, 50, dtype, "none", residual=False)
    dZ, add = matrix(n, 50, dtype, 5), matrix(n, 40, dtype, 6, ld=43)
    only = dict(want_dW=False, want_db=False)
    alone, bound = linear_backward(X, W, dZ, None, torch.float32, torch.float32)[0]
    got = B.ftc_linear_backward(X, W, dZ, dX_add=add, dx_dtype=torch.float32, **only)[0]
    want = alone + f64(add)
    check(f"dX + residual {dtype} {n}", got, want, bound + 2 * 2.0 ** -24 * np.abs(want))
    there = add.clone()
    B.ftc_linear_backward(X, W, dZ, dX_add=there, dX=there, **only)
    assert torch.equal(there, B.ftc_linear_backward(X, W, dZ, dX_add=add, **only)[0])


@pytest.mark.parametrize("act", list(ACTS))
def test_gradient_against_differences(act):
    """Central differences of <Z, G> along random directions, in fp32: h = 2^-7, off by the third derivative (below 2) times h^2 / 6
    of the direction's size and by rounding of Z over h."""
    n, d_in, d_out = 20, 12, 16
    X, W, b, _ = layer(n, d_in, d_out, torch.float32, act, seed=3, residual=False)
    if act == "relu":
        b = b + 10.0 * torch.sign(b)      # no sum within a step of the corner
    G = matrix(n, d_out, torch.float32, 8)
    slope = B.slope_like(G)
    B.ftc_linear(X, W, bias=b, act=ACTS[act], slope=slope)
    grads = B.ftc_linear_backward(X, W, G, slope=slope)
    f = lambda X, W, b: float((B.ftc_linear(X, W, bias=b, act=ACTS[act]).double() * G.double()).sum())
    h = 2.0 ** -7
    for i, grad in enumerate(grads):
        at = [X, W, b]
        d = torch.sign(matrix(1, grad.numel(), torch.float32, 11 + i)).view(grad.shape).contiguous()
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * d, at[i] - h * d
        got = (f(*up) - f(*down)) / (2 * h)
        # of an entry of P: |x| (or |w|) summed, 1 for the bias
        step = [np.abs(W.cpu().numpy()).sum(0).max(), np.abs(X.cpu().numpy()).sum(1).max(), 1.0][i]
        size = float(G.double().abs().sum())
        z = float(B.ftc_linear(X, W, bias=b, act=ACTS[act]).abs().max())
        assert abs(got - float((grad.double() * d.double()).sum())) <= size * (2 * step ** 3 * h * h / 6 + 32 * 2.0 ** -24 * (z + 1) / h)


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan(dtype):
    """A NaN or infinite input reaches the rows (columns) it belongs to and no others; slopes at infinity are the limits."""
    n, d_in, d_out = 40, 24, 70
    X, W, b, _ = layer(n, d_in, d_out, dtype, "gelu", residual=False)
    clean = B.ftc_linear(X, W, bias=b, act=B.FTC_ACT_GELU)
    Y = X.clone()
    Y[3, 5] = float("nan")
    out = B.ftc_linear(Y, W, bias=b, act=B.FTC_ACT_GELU)
    assert bool(out[3].isnan().all())
    keep = torch.arange(n, device="cuda") != 3
    assert torch.equal(out[keep], clean[keep])
    for act in ("gelu", "silu", "relu"):
        ends = torch.tensor([float("inf"), float("-inf"), float("nan"), 0.0], dtype=dtype, device="cuda")
        slope = B.slope_like(ends[None])
        z = B.ftc_linear(torch.zeros((1, 3), dtype=dtype, device="cuda"), torch.zeros((3, 4), dtype=dtype, device="cuda"), bias=ends, act=ACTS[act],
                         slope=slope)
        assert z[0, 0] == float("inf") and z[0, 1] == 0 and bool(z[0, 2].isnan()) and z[0, 3] == 0, (act, z)
        s = slope_values(slope)[0]
        assert s[0] == 1 and abs(s[1]) < 1e-6 and np.isnan(s[2]) and abs(s[3] - (0.0 if act == "relu" else 0.5)) < 1e-6, (act, s)


@pytest.mark.parametrize("n,d_in,d_out", [(70, 64, 130), (300, 33, 65)])
def test_fp32_numbers_that_bf16_pieces_do_not_hold(n, d_in, d_out):
    """Infinities, the largest numbers, sums that overflow, and tiny numbers, in fp32: as a product in fp32 gives them.  A number below 2^-110
    may be off by 2^-126."""
    X, W, _, _ = layer(n, d_in, d_out, torch.float32, "none", residual=False, bias=False)
    big = torch.finfo(torch.float32).max
    X[1, 2], X[5, 7], X[9, 0], X[40, 3] = float("inf"), float("-inf"), big, -big * 0.999
    W[5, 11], W[0, 3] = float("inf"), 0.5
    W[2, 20] = 0.0                                             # inf * 0
    X[50] = 0.0
    X[50, 4] = 2.0 ** -140
    X[51] *= 2.0 ** -120
    x, w = f64(X), f64(W)
    with np.errstate(invalid="ignore", over="ignore"):
        want = x @ w
        want[np.abs(want) > big] = np.inf * np.sign(want[np.abs(want) > big])
        bound = (np.abs(x) @ np.abs(w)) * (d_in + 8) * 2.0 ** -24 + 2.0 ** -125 * np.abs(w).sum(0)
    bound[~np.isfinite(want)] = 0
    check("large and small numbers", B.ftc_linear(X, W), want, bound)
    with np.errstate(invalid="ignore", over="ignore"):
        dZ = matrix(n, d_out, torch.float32, 3)
        dZ[2, 9] = float("inf")
        g = f64(dZ)
        wantX, wantW = g @ w.T, x.T @ g
        for m in (wantX, wantW):
            m[np.abs(m) > big] = np.inf * np.sign(m[np.abs(m) > big])
        finite = np.isfinite(wantW)
        boundW = (np.abs(x).T @ np.abs(g)) * (n + 8) * 2.0 ** -24 + 2.0 ** -125 * np.abs(g).sum(0)
        boundX = (np.abs(g) @ np.abs(w.T)) * (d_out + 8) * 2.0 ** -24 + 2.0 ** -125 * np.abs(g).sum(1)[:, None]
    boundW[~finite] = 0
    boundX[~np.isfinite(wantX)] = 0
    dX, dW, _ = B.ftc_linear_backward(X, W, dZ, want_db=False)
    check("dX", dX, wantX, np.nan_to_num(boundX, nan=0.0, posinf=0.0))
    check("dW", dW, wantW, np.nan_to_num(boundW, nan=0.0, posinf=0.0))


def test_residual_in_place_and_empty():
    X, W, b, _ = layer(50, 30, 44, torch.bfloat16, "silu", residual=False)
    R = matrix(50, 44, torch.bfloat16, 5)
    want = B.ftc_linear(X, W, bias=b, act=B.FTC_ACT_SILU, residual=R)
    B.ftc_linear(X, W, bias=b, act=B.FTC_ACT_SILU, residual=R, out=R)
    assert torch.equal(R, want)
    assert B.ftc_linear(X[:0], W, bias=b).shape == (0, 44)
    dX, dW, db = B.ftc_linear_backward(X[:0], W, R[:0])
    assert dX.shape == (0, 30) and bool((dW == 0).all()) and bool((db == 0).all())


def test_parts_added_up_in_place():
    """Few rows and a long contraction: the second kernel reads the residual that it writes over."""
    X, W, b, _ = layer(3, 3001, 40, torch.float16, "none", residual=False)
    R = matrix(3, 40, torch.float16, 5)
    want = B.ftc_linear(X, W, bias=b, residual=R.clone())
    B.ftc_linear(X, W, bias=b, residual=R, out=R)
    assert torch.equal(R, want)


def test_captured_and_on_another_stream():
    n, d_in, d_out = 300, 700, 130
    X, W, b, R = layer(n, d_in, d_out, torch.bfloat16, "gelu")
    dZ = matrix(n, d_out, torch.bfloat16, 9)
    L = B.lib()
    ws = B._workspace(max(L.ftc_linear_workspace_bytes(n, d_in, d_out), L.ftc_linear_backward_workspace_bytes(n, d_in, d_out)), "cuda")
    new = lambda: [torch.full((n, d_out), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((n, d_out), 7, dtype=torch.int16, device="cuda"),
                   torch.full((n, d_in), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((d_in, d_out), 7.0, device="cuda"),
                   torch.full((d_out,), 7.0, device="cuda")]

    def both(t):
        B.ftc_linear(X, W, bias=b, act=B.FTC_ACT_GELU, residual=R, out=t[0], slope=t[1], ws=ws)
        B.ftc_linear_backward(X, W, dZ, slope=t[1], dX=t[2], dW=t[3], db=t[4], ws=ws)

    want, got = new(), new()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(want)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(got)
    for _ in range(3):
        for t in got:
            t.fill_(3)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        X.float().sum().item()
