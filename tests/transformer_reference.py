"""The operators of a graph transformer from their formulas, in 64 bits (numpy, on the CPU), each with a bound on how far a
correct implementation may be off, element by element.

The bounds count roundings.  u is half a step of the type an output (or an operand of a second product) is rounded to; s is 2^-24,
half a step of fp32, in which sums of n terms are held: off by at most (n + 8) s times the sum of their absolute values.  fp16 has no
steps below 2^-24, so a rounding there is off by up to 2^-25 more."""
import math

import numpy as np
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
S = 2.0 ** -24


def f64(t):
    return t.detach().cpu().double().numpy()


def check(name, got, want, bound):
    """got (tensor) against want, within bound; NaN and infinities exactly."""
    got = f64(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN elsewhere"
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), f"{name}: infinities elsewhere"
    off = np.abs(got[fine] - want[fine])
    share = off / np.maximum(bound[fine], 1e-300)
    worst = float(share.max()) if share.size else 0.0
    print(f"{name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.3f} times the bound"


# ---- embedding ------------------------------------------------------------------------------------------------
def embedding(ids, E, scale, out_dtype):
    ids, E = ids.cpu().numpy(), f64(E)
    ok = (ids >= 0) & (ids < E.shape[0])
    out = np.zeros((len(ids), E.shape[1]))
    out[ok] = E[ids[ok]] * scale
    return out, np.abs(out) * (2 * S + HALF_STEP[out_dtype]) + TINY[out_dtype]


def embedding_backward(ids, g, vocab, scale, out_dtype):
    ids, g = ids.cpu().numpy(), f64(g)
    dE, ab, count = np.zeros((vocab, g.shape[1])), np.zeros((vocab, g.shape[1])), np.zeros((vocab, 1))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(dE, ids[ok], g[ok] * scale)
    np.add.at(ab, ids[ok], np.abs(g[ok] * scale))
    np.add.at(count, ids[ok], 1)
    return dE, ab * (count + 2) * S + np.abs(dE) * HALF_STEP[out_dtype] + TINY[out_dtype]


# ---- linear -------------------------------------------------------------------------------------------------------
_erf = np.vectorize(math.erf, otypes=[float])


def activation(p, act):
    """act(p), act'(p), and bounds of |act'| and |act''|; act: none, relu, gelu, silu."""
    if act == "relu":
        return np.maximum(p, 0), (p > 0).astype(float), 1.0, 0.0
    if act == "gelu":
        cdf = 0.5 * (1 + _erf(p / math.sqrt(2)))
        return p * cdf, cdf + p * np.exp(-0.5 * p * p) / math.sqrt(2 * math.pi), 1.13, 0.8
    if act == "silu":
        g = 1 / (1 + np.exp(-p))
        return p * g, g * (1 + p * (1 - g)), 1.1, 0.5
    return p, np.ones_like(p), 1.0, 0.0


def linear(X, W, bias, act, residual, out_dtype):
    """Z and its bound; act'(P), its bound, and how far P is off."""
    x, w = f64(X), f64(W)
    k = x.shape[1]
    p, ab = x @ w, np.abs(x) @ np.abs(w)
    if bias is not None:
        p, ab = p + f64(bias), ab + np.abs(f64(bias))
    dp = (k + 8) * S * ab
    a, slope, lip, curve = activation(p, act)
    # exp and erf of the device: a few steps of fp32, on values of size 1
    da = lip * dp + (0 if act in ("none", "relu") else 16 * S * (1 + np.abs(p)))
    z = a if residual is None else a + f64(residual)
    fixed = 2.0 ** -15 if X.dtype != torch.float32 else 0.0
    dslope = curve * dp + fixed + (0 if act in ("none", "relu") else 32 * S * (1 + np.abs(p)))
    return z, da + 4 * S * np.abs(z) + np.abs(z) * HALF_STEP[out_dtype] + TINY[out_dtype], slope, dslope, dp, p


def slope_values(t):
    """What a slope tensor stands for."""
    return f64(t) if t.dtype == torch.float32 else np.where(t.cpu().numpy() == -32768, np.nan, t.cpu().numpy() / 16384.0)


def linear_backward(X, W, dZ, slope, dx_dtype, dw_dtype):
    """[(dX, bound), (dW, bound), (db, bound)] for the slopes as they are."""
    x, w, g = f64(X), f64(W), f64(dZ)
    dp = g if slope is None else g * slope_values(slope)
    n, d_out = g.shape
    u = 0.0 if slope is None else HALF_STEP[X.dtype] + S  # dP for the products
    t = 0.0 if slope is None else TINY[X.dtype]
    res = []
    for a, b, k, dt in ((dp, w.T, d_out, dx_dtype), (x.T, dp, n, dw_dtype)):
        want, ab = a @ b, np.abs(a) @ np.abs(b)
        other = (np.abs(w.T).sum(0)[None, :] if a is dp else np.abs(x.T).sum(1)[:, None]) * t
        res.append((want, ab * (u + (k + 8) * S) + other + np.abs(want) * HALF_STEP[dt] + TINY[dt]))
    db = dp.sum(0)
    res.append((db, np.abs(dp).sum(0) * (n + 8) * S + np.abs(db) * HALF_STEP[dw_dtype] + TINY[dw_dtype]))
    return res


# ---- attention -----------------------------------------------------------------------------------------------------
def attention(Q, K, V, q_ptr, kv_ptr, heads, kv_heads, scale, mask=None, dOut=None, keep=None):
    """dict of (value, bound): out, lse and, with dOut, dQ, dK, dV.  Rows of no graph come as `keep` has them (NaN)."""
    dt = Q.dtype
    u, tiny = HALF_STEP[dt], TINY[dt]
    q, k, v = f64(Q), f64(K), f64(V)
    n_q, n_kv = q.shape[0], k.shape[0]
    D, group = q.shape[1] // heads, heads // kv_heads
    qp, kp = q_ptr.cpu().tolist(), kv_ptr.cpu().tolist()
    seen = np.ones(n_kv, bool) if mask is None else mask.cpu().numpy() != 0
    new = lambda n, c: (np.full((n, c), np.nan), np.zeros((n, c)))
    res = dict(out=new(n_q, heads * D), lse=new(n_q, heads))
    if dOut is not None:
        do = f64(dOut)
        res.update(dQ=new(n_q, heads * D), dK=new(n_kv, kv_heads * D), dV=new(n_kv, kv_heads * D))
    for g in range(len(qp) - 1):
        rows, keys = slice(qp[g], qp[g + 1]), np.arange(kp[g], kp[g + 1])
        for name in res:
            at = rows if name in ("out", "lse", "dQ") else slice(kp[g], kp[g + 1])
            res[name][0][at] = 0
        res["lse"][0][rows] = -np.inf
        keys = keys[seen[kp[g]:kp[g + 1]]]
        n, lq = len(keys), qp[g + 1] - qp[g]
        if n == 0 or lq == 0:
            continue
        for h in range(heads):
            hq, hk = slice(h * D, h * D + D), slice(h // group * D, h // group * D + D)
            a, b, c = q[rows, hq], k[keys, hk], v[keys, hk]
            s, sab = scale * a @ b.T, abs(scale) * np.abs(a) @ np.abs(b.T)
            ds_s = sab * (D + 8) * S                     # scores
            m = s.max(1, keepdims=True)
            e = np.exp(s - m)
            l = e.sum(1, keepdims=True)
            p, lse = e / l, (m + np.log(l))[:, 0]
            # relative error of a probability: its score's and the sum's, the exponent's in fp32, the sum's n roundings; lse once more
            ep = 2 * ds_s.max(1, keepdims=True) + (n + 16) * S + 8 * S * (np.abs(s).max(1, keepdims=True) + np.abs(lse)[:, None])
            out = p @ c
            dout = (p * (u + ep) + tiny) @ np.abs(c) + u * np.abs(out) + tiny + (n + 8) * S * (p @ np.abs(c))
            res["out"][0][rows, hq], res["out"][1][rows, hq] = out, dout
            res["lse"][0][rows, h], res["lse"][1][rows, h] = lse, (ep[:, 0] + 8 * S * (1 + np.abs(lse)))
            if dOut is None:
                continue
            w = do[rows, hq]
            dp, dpab = w @ c.T, np.abs(w) @ np.abs(c.T)
            delta = (p * dp).sum(1, keepdims=True)
            # delta from the rounded output, or from the probabilities
            ddelta = (np.abs(w) * dout).sum(1, keepdims=True) + (D + 8) * S * (np.abs(w) * (np.abs(out) + dout)).sum(1, keepdims=True) \
                + (p * (np.abs(dp) * (ep + (n + 8) * S) + dpab * (D + 8) * S)).sum(1, keepdims=True)
            ds = p * (dp - delta)
            dds = p * (np.abs(dp - delta) * ep + (dpab * (D + 8) * S + ddelta + 2 * S * (np.abs(dp) + np.abs(delta))) * (1 + ep)) + u * np.abs(ds)
            dds = dds * (1 + u) + tiny
            gq, gk, gv = scale * ds @ b, scale * ds.T @ a, p.T @ w
            sums = lambda x, y, terms: (terms + 8) * S * np.abs(x) @ np.abs(y)
            res["dQ"][0][rows, hq] = gq
            res["dQ"][1][rows, hq] = abs(scale) * (dds @ np.abs(b) + sums(ds, b, n)) + (u + 2 * S) * np.abs(gq) + tiny
            bk = abs(scale) * (dds.T @ np.abs(a) + sums(ds.T, a, lq * group))
            bv = (p * (u + ep) + tiny).T @ np.abs(w) + sums(p.T, w, lq * group)
            for name, val, bound in (("dK", gk, bk), ("dV", gv, bv)):
                res[name][0][keys, hk] += val
                res[name][1][keys, hk] += bound
    if dOut is not None:
        for name in ("dK", "dV"):
            val, bound = res[name]
            bound += (u + 2 * S) * np.abs(np.nan_to_num(val)) * (1 + u) + tiny
    return res
