"""The norms around a block, weights by group, and the norm over all gradients from their formulas, in 64 bits (numpy, on the CPU), each with a
bound on how far a correct implementation may be off, element by element: roundings are counted as in transformer_reference."""
import numpy as np
import torch

from transformer_reference import HALF_STEP, S, TINY, f64, linear, linear_backward

EPS = 1e-5


def _mean(x):
    return x.mean(1, keepdims=True)


def _normed(t, dt, kind, eps):
    """The normalised rows of t, which is off by up to dt: xh, how far that is off, the factor and its relative error, the mean and its error."""
    d = t.shape[1]
    mean, dm = np.zeros((t.shape[0], 1)), np.zeros((t.shape[0], 1))
    if kind == "layer":
        mean, dm = _mean(t), _mean(dt) + (d + 8) * S * _mean(np.abs(t))
    dev = t - mean
    ddev = dt + dm + S * np.abs(dev)
    v = _mean(dev ** 2)
    dv = _mean(2 * np.abs(dev) * ddev + ddev ** 2) + (d + 8) * S * v
    r = 1 / np.sqrt(v + eps)
    # a relative error q of v + eps is one of up to q / 2 / (1 - q) of its root, for q below 1
    q = np.minimum(dv / (v + eps), 0.9)
    er = q / 2 / (1 - q) + 4 * S
    xh = dev * r
    return xh, r * ddev * (1 + er) + np.abs(xh) * (er + 2 * S), r, er, mean, dm


def block(X, F, x_scale, post, post_w, post_b, gate, pre, pre_w, pre_b, dH=None, dU=None, dw_dtype=torch.float32, eps=EPS):
    """dict of (value, bound): H, U, stats and, with dH or dU, the gradients that there are."""
    dt, (n, d) = X.dtype, X.shape
    wide = lambda t: None if t is None else f64(t)
    x, f, g, pw, pb, w, b = (wide(t) for t in (X, F, gate, post_w, post_b, pre_w, pre_b))
    rounded = lambda v, e, t=dt: (v, e + (np.abs(v) + e) * HALF_STEP[t] + TINY[t])
    stats, dstats = np.zeros((n, 4)), np.zeros((n, 4))
    stats[:, 1] = stats[:, 3] = 1

    def affine(xh, dxh, weight, bias):
        p = xh * (1 if weight is None else weight) + (0 if bias is None else bias)
        return p, dxh * (1 if weight is None else np.abs(weight)) + 2 * S * (np.abs(xh * (1 if weight is None else weight)) + (0 if bias is None else np.abs(bias)))

    def keep(at, r, er, mean, dm):
        stats[:, at], stats[:, at + 1], dstats[:, at], dstats[:, at + 1] = mean[:, 0], r[:, 0], dm[:, 0], (r * er)[:, 0]
    if f is None:
        h, dh = x_scale * x, np.abs(x_scale * x) * S
    else:
        p, dp = f, np.zeros_like(f)
        if post != "none":
            fh, dfh, rf, erf_, *m = _normed(f, dp, post, eps)
            keep(0, rf, erf_, *m)
            p, dp = affine(fh, dfh, pw, pb)
        gp, dgp = (p, dp) if g is None else (g * p, np.abs(g) * dp + S * np.abs(g * p))
        h, dh = x_scale * x + gp, dgp + 2 * S * (np.abs(x_scale * x) + np.abs(gp))
    res = dict(H=rounded(h, dh))
    if pre != "none":
        hh, dhh, rh, erh, *m = _normed(h, dh, pre, eps)
        keep(2, rh, erh, *m)
        res["U"] = rounded(*affine(hh, dhh, w, b))
    res["stats"] = stats, dstats + 2 * S * np.abs(stats)
    if dH is None and dU is None:
        return res

    def back(gr, dgr, xh, dxh, r, er, weight, kind):
        """The gradient of a normed row, of its weight and of its bias."""
        sums = lambda v, dv: rounded(v.sum(0), dv.sum(0) + (n + 8) * S * np.abs(v).sum(0), dw_dtype)
        gw, dgw = (gr, dgr) if weight is None else (gr * weight, np.abs(weight) * dgr + S * np.abs(gr * weight))
        dot, ddot = gw * xh, np.abs(gw) * dxh + dgw * (np.abs(xh) + dxh)
        s1, ds1 = _mean(dot), _mean(ddot) + (d + 8) * S * _mean(np.abs(dot))
        s2, ds2 = np.zeros_like(s1), np.zeros_like(s1)
        if kind == "layer":
            s2, ds2 = _mean(gw), _mean(dgw) + (d + 8) * S * _mean(np.abs(gw))
        size = np.abs(gw) + np.abs(xh * s1) + np.abs(s2)
        off = dgw + dxh * np.abs(s1) + (np.abs(xh) + dxh) * ds1 + ds2 + 4 * S * size
        return (r * (gw - xh * s1 - s2), r * (1 + er) * off + r * size * (er + 2 * S)), \
            sums(gr * xh, np.abs(gr) * dxh + dgr * (np.abs(xh) + dxh)), sums(gr, dgr)
    dh_, ddh = (f64(dH) if dH is not None else np.zeros((n, d))), np.zeros((n, d))
    if dU is not None:
        (v, e), dw, db = back(f64(dU), np.zeros((n, d)), hh, dhh, rh, erh, w, pre)
        dh_, ddh = dh_ + v, e + 2 * S * (np.abs(dh_) + np.abs(v))
        if w is not None:
            res["dpre_w"] = dw
        if b is not None:
            res["dpre_b"] = db
    res["dX"] = rounded(x_scale * dh_, abs(x_scale) * ddh + S * np.abs(x_scale * dh_))
    if f is None:
        return res
    if g is not None:
        v, e = dh_ * p, ddh * (np.abs(p) + dp) + np.abs(dh_) * dp + S * np.abs(dh_ * p)
        res["dgate"] = rounded(v, e) if gate.dim() == 2 else rounded(v.sum(0), e.sum(0) + (n + 8) * S * np.abs(v).sum(0), dw_dtype)
        dh_, ddh = dh_ * g, np.abs(g) * ddh + S * np.abs(dh_ * g)
    if post != "none":
        (dh_, ddh), dw, db = back(dh_, ddh, fh, dfh, rf, erf_, pw, post)
        if pw is not None:
            res["dpost_w"] = dw
        if pb is not None:
            res["dpost_b"] = db
    res["dF"] = rounded(dh_, ddh)
    return res


# ---- dense layers by group: the dense layer's values and bounds for each group's rows, NaN where there is no group --------------------------------
def grouped(X, W, ptr, bias, act, residual, out_dtype):
    """(Z, bound), (slope, bound), where the slope is sure."""
    n, d_out = X.shape[0], W.shape[2]
    z, dz, s, ds, sure = (np.full((n, d_out), np.nan) if i in (0, 2) else np.zeros((n, d_out)) for i in range(5))
    for g, (a, b) in enumerate(zip(ptr, ptr[1:])):
        if b > a:
            at = slice(a, b)
            z[at], dz[at], s[at], ds[at], dp, p = linear(X[at], W[g], None if bias is None else bias[g], act, None if residual is None else residual[at], out_dtype)
            sure[at] = np.abs(p) > dp if act == "relu" else 1
    return (z, dz), (s, ds), sure > 0


def grouped_backward(X, W, ptr, dZ, slope, dx_dtype, dw_dtype):
    """[(dX, bound), (dW, bound), (db, bound)] for the slopes as they are."""
    (n, d_in), (groups, _, d_out) = X.shape, W.shape
    dX, dW, db = (np.full((n, d_in), np.nan), np.zeros((n, d_in))), (np.zeros(W.shape), np.zeros(W.shape)), (np.zeros((groups, d_out)), np.zeros((groups, d_out)))
    for g, (a, b) in enumerate(zip(ptr, ptr[1:])):
        if b > a:
            at = slice(a, b)
            for to, where, (value, bound) in zip((dX, dW, db), (at, g, g), linear_backward(X[at], W[g], dZ[at], None if slope is None else slope[at], dx_dtype, dw_dtype)):
                to[0][where], to[1][where] = value, bound
    return [dX, dW, db]
