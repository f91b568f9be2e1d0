"""The dense layer and its gradients in the larger tiles (128 and 256, one to ten parts, whole pieces and others), against the formulas in
64 bits, every element.  The bounds are those of transformer_reference.py, the 64-bit products torch's on the GPU."""
import math

import pytest
import torch

from dense_tiles import CASES
from paper_2412_12218_amd import binding as B
from transformer_reference import HALF_STEP, S, TINY

pytestmark = pytest.mark.gpu
ACTS = dict(none=B.FTC_ACT_NONE, relu=B.FTC_ACT_RELU, gelu=B.FTC_ACT_GELU, silu=B.FTC_ACT_SILU)
ALL = [pytest.param(c, t, id=f"{c[0]}-{c[1]}-{c[2]}-{'whole' if c[4] else 'odd'}-{str(t)[6:]}") for c in CASES
       for t in ([torch.float32] if c[3] else [torch.float16, torch.bfloat16])]


def rows(n, d, dtype, seed, ld, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((n, ld), generator=gen, device="cuda") * scale).to(dtype)[:, :d]


def layer(n, d_in, d_out, dtype, whole):
    """X, W, bias, residual, dZ; whole: rows of whole pieces, the same with a gap of 16 bytes behind them."""
    gap = 16 // torch.empty(0, dtype=dtype).element_size() if whole else 3
    X, G, R = rows(n, d_in, dtype, 1, d_in + gap), rows(n, d_out, dtype, 2, d_out + gap), rows(n, d_out, dtype, 3, d_out + 1)
    W, b = rows(d_in, d_out, dtype, 4, d_out, d_in ** -0.5).contiguous(), rows(1, d_out, dtype, 5, d_out)[0].contiguous()
    for t, w in ((X, d_in), (W, d_out), (G, d_out)):
        e = t.element_size()
        assert (t.data_ptr() % 16 == 0 and t.stride(0) * e % 16 == 0 and w * e % 16 == 0) == whole
    return X, W, b, R, G


def check(name, got, want, bound):
    assert got.shape == want.shape
    off = (got.double() - want).abs()
    finite = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan()), f"{name}: NaN elsewhere"
    assert torch.equal(got[want.isinf()].double(), want[want.isinf()]), f"{name}: infinities elsewhere"
    share = (off / bound.clamp(min=1e-300))[finite].max().item()
    print(f"{name}: {share:.3f} of the bound", flush=True)
    assert share <= 1.0, f"{name}: {share:.3f} times the bound"


def activation(p, act):
    if act == "relu":
        return p.clamp(min=0), (p > 0).double(), 1.0, 0.0
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-p / math.sqrt(2))
        return p * cdf, cdf + p * torch.exp(-0.5 * p * p) / math.sqrt(2 * math.pi), 1.13, 0.8
    if act == "silu":
        g = torch.sigmoid(p)
        return p * g, g * (1 + p * (1 - g)), 1.1, 0.5
    return p, torch.ones_like(p), 1.0, 0.0


def slopes(t):
    return t.double() if t.dtype == torch.float32 else torch.where(t == -32768, math.nan, t.double() / 16384)


@pytest.mark.parametrize("case,dtype", ALL)
def test_forward(case, dtype):
    n, d_in, d_out, _, whole = case[:5]
    X, W, b, R, _ = layer(n, d_in, d_out, dtype, whole)
    p0, ab0 = X.double() @ W.double(), X.double().abs() @ W.double().abs()
    for i, act in enumerate(ACTS):
        bias, residual, slope_too, out_dtype = (b, None)[i == 1], (None, R)[i != 0], i != 1, (dtype, torch.float32)[i == 2]
        p, ab = (p0, ab0) if bias is None else (p0 + b.double(), ab0 + b.double().abs())
        dp = (d_in + 8) * S * ab
        a, slope, lip, curve = activation(p, act)
        near = 0.0 if act in ("none", "relu") else S * (1 + p.abs())
        z = a if residual is None else a + R.double()
        out = torch.full((n, d_out + 3), 7.0, device="cuda", dtype=out_dtype)
        kept = torch.full((n, d_out + 5), 7, device="cuda", dtype=B.slope_like(X).dtype) if slope_too else None
        B.ftc_linear(X, W, bias=bias, act=ACTS[act], residual=residual, out=out[:, :d_out], slope=kept[:, :d_out] if slope_too else None)
        check(f"Z {act}", out[:, :d_out], z, lip * dp + 16 * near + z.abs() * (4 * S + HALF_STEP[out_dtype]) + TINY[out_dtype])
        assert bool((out[:, d_out:] == 7).all())
        if slope_too:
            sure = p.abs() > dp if act == "relu" else torch.ones_like(p, dtype=torch.bool)
            off = (slopes(kept[:, :d_out]) - slope).abs()
            assert bool((off <= curve * dp + (2.0 ** -15 if dtype != torch.float32 else 0.0) + 32 * near)[sure].all()), act
            assert bool((kept[:, d_out:] == 7).all())
        if residual is not None and out_dtype == dtype:      # the same bits on top of the residual
            place = R.clone(memory_format=torch.preserve_format)
            B.ftc_linear(X, W, bias=bias, act=ACTS[act], residual=place, out=place)
            assert torch.equal(place, out[:, :d_out])


@pytest.mark.parametrize("case,dtype", ALL)
def test_backward(case, dtype):
    n, d_in, d_out, _, whole = case[:5]
    X, W, b, _, G = layer(n, d_in, d_out, dtype, whole)
    for act in ("none", "gelu"):
        slope = None
        if act != "none":
            slope = B.slope_like(G)
            B.ftc_linear(X, W, bias=b, act=ACTS[act], slope=slope)
        dt = torch.float32 if act == "none" else dtype
        dP = G.double() if slope is None else G.double() * slopes(slope)
        u, t = (0.0, 0.0) if slope is None else (HALF_STEP[dtype] + S, TINY[dtype])
        add = rows(n, d_in, dtype, 6, d_in + 1) if act == "none" else None
        out = torch.full((n, d_in + 5), 7.0, device="cuda", dtype=dt)
        dX, dW, db = B.ftc_linear_backward(X, W, G, slope=slope, dX=out[:, :d_in], dX_add=add, dw_dtype=dt)
        for name, got, x, y, k in (("dX", dX, dP, W.double().t(), d_out), ("dW", dW, X.double().t(), dP, n)):
            want, ab = x @ y, x.abs() @ y.abs()
            lost = (y.abs().sum(0)[None, :] if name == "dX" else x.abs().sum(1)[:, None]) * t
            if name == "dX" and add is not None:
                want, ab = want + add.double(), ab + add.double().abs()
            check(f"{name} {act}", got, want, ab * (u + (k + 8) * S) + lost + want.abs() * HALF_STEP[dt] + TINY[dt])
        want = dP.sum(0)
        check(f"db {act}", db, want, dP.abs().sum(0) * (n + 8) * S + want.abs() * HALF_STEP[dt] + TINY[dt])
        assert bool((out[:, d_in:] == 7).all())
        again = B.ftc_linear_backward(X, W, G, slope=slope, dX_add=add, dx_dtype=dt, dw_dtype=dt)
        assert all(torch.equal(x, y) for x, y in zip(again, (dX, dW, db)))
        if add is not None:
            keep = B.ftc_linear_backward(X, W, G, dX_add=add, want_dW=False, want_db=False)[0]
            place = add.clone(memory_format=torch.preserve_format)
            B.ftc_linear_backward(X, W, G, dX_add=place, dX=place, want_dW=False, want_db=False)
            assert torch.equal(place, keep)


@pytest.mark.parametrize("case", [c for c in CASES if c[3]], ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}")
def test_infinities_in_fp32(case):
    """Infinities and NaN in every block of a wave, in the last tile and in numbers that bf16 pieces do not hold: results as of a product in fp32."""
    n, d_in, d_out, _, whole = case[:5]
    X, W, _, _, G = layer(n, d_in, d_out, torch.float32, whole)
    X, W, G = X.clone(memory_format=torch.preserve_format), W.clone(), G.clone(memory_format=torch.preserve_format)
    big = torch.finfo(torch.float32).max
    for i, r in enumerate((0, 33, n // 2, n - 1)):
        X[min(r, n - 1), (7 * i + 3) % d_in] = (math.inf, -math.inf, math.nan, big)[i]
        G[min(r, n - 1), (5 * i + 1) % d_out] = (math.nan, big, math.inf, -math.inf)[i]
    W[d_in - 1, d_out - 1] = math.inf
    W[3 % d_in, 40 % d_out] = 0.0
    def products(x, y, k):
        """The product, and the sums of what its finite numbers add to it on either side of zero."""
        a, b = x.nan_to_num(0, 0, 0), y.nan_to_num(0, 0, 0)
        up = a.clamp(min=0) @ b.clamp(min=0) + a.clamp(max=0) @ b.clamp(max=0)
        return x @ y, up, up - a @ b, k
    dX, dW, _ = B.ftc_linear_backward(X, W, G, want_db=False)
    for name, got, (want, up, down, k) in (("Z", B.ftc_linear(X, W), products(X.double(), W.double(), d_in)),
                                           ("dX", dX, products(G.double(), W.double().t(), d_out)),
                                           ("dW", dW, products(X.double().t(), G.double(), n))):
        bound = (up + down) * (k + 8) * S
        # sums within a rounding of the largest number may fall to either side of it.  Where the terms of one sign add up to more than that, a sum
        # that is not comes out infinite if those come first; where those of both signs do (or an infinity and the others), infinite or NaN
        far = (up > big) | (down > big)
        open_ = (want.abs() - big).abs() <= bound + big * 2 * S
        open_ |= far & ~want.isnan() & ((want.abs() <= big) | ((up > big) & (down > big)) | ((want == math.inf) & (down > big)) | ((want == -math.inf) & (up > big)))
        assert open_.sum() <= 16
        want = torch.where(want.abs() > big, torch.copysign(torch.full_like(want, math.inf), want), want)
        want[open_] = 0.0
        check(name, got.masked_fill(open_, 0.0), want, bound)
