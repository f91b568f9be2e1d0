"""Bounds of the norms around a block as the kernels add: a row in lanes of 8 or 16 numbers, these in a tree, and the mean in two steps (block_reference.py allows for one sum behind the
other over a whole row, and one step, which is no bound at all for a mean beside a small spread)."""
import numpy as np

import block_reference
from block_reference import _mean
from transformer_reference import S

# Roundings that a number of a row passes on its way into the row's sum: of 1 / d and of its product, 16 of a lane's own numbers, 6 in a wave, 16 waves of a workgroup.
SUM = 40
# Sums over rows: those of 120 rows here (`of_rows`), 8 for what a workgroup and the kernel behind it add on the way.  A lane has at most 120 rows of any test, so 16 lane groups, or as many
# parts of 64 threads each, are in it, too.
ROWS = 120


def normed(t, dt, kind, eps):
    """block_reference._normed, with the mean m' = m + mean(t - m), m off by SUM roundings of the numbers, m' by as many of the distances and by its own one."""
    ev_more, mean, dm = 0.0, np.zeros((t.shape[0], 1)), np.zeros((t.shape[0], 1))
    if kind == "layer":
        mean = _mean(t)
        first = SUM * S * _mean(np.abs(t) + dt)              # of m
        spread = _mean(np.abs(t - mean) + dt) + first
        step = (SUM + 2) * S * spread                        # of mean(t - m)
        dm = _mean(dt) + step + S * (np.abs(mean) + step)
        # the variance from distances to m: its square step is taken off, which is at most a 64th of all, or the squares are summed again around m'
        v = _mean((t - mean) ** 2)
        ev_more = 2 * np.minimum(first, np.sqrt(v / 63)) * step + step ** 2 + (step + S * np.abs(mean)) ** 2
    dev = t - mean
    v = _mean(dev ** 2)
    ev = _mean(2 * np.abs(dev) * dt + dt ** 2) + (SUM + 8) * S * v * 64 / 63 + ev_more + S * eps
    r = 1 / np.sqrt(v + eps)
    q = np.minimum(ev / (v + eps), 0.9)
    er = q / 2 / (1 - q) + 4 * S
    xh, ddev = dev * r, dt + dm + S * np.abs(dev)
    return xh, r * ddev * (1 + er) + np.abs(xh) * (er + 2 * S), r, er, mean, dm


def block(monkeypatch, X, F, x_scale, *args, **k):
    """block_reference.block with these bounds of a row's statistics.  h = 1 x is x itself."""
    alone = F is None and x_scale == 1
    monkeypatch.setattr(block_reference, "_normed", lambda t, dt, kind, eps: normed(t, 0 * dt if alone else dt, kind, eps))
    return block_reference.block(X, F, x_scale, *args, **k)


ROW_WISE = ("H", "U", "stats", "dX", "dF")


def of_rows(monkeypatch, s, dH, dU, **k):
    """The same for many rows: (value, bound) of each name, sums over the rows from those of ROWS rows each."""
    n = s["X"].shape[0]
    cut = lambda t, at: t[at] if t is not None and t.dim() == 2 else t
    s = {name: t if t is None else t.cpu() for name, t in s.items()}
    dH, dU = (t if t is None else t.cpu() for t in (dH, dU))
    parts = []
    for a in range(0, n, ROWS):
        at = slice(a, a + ROWS)
        parts.append(block(monkeypatch, **{name: cut(t, at) for name, t in s.items()}, dH=cut(dH, at), dU=cut(dU, at), **k))
    rows = lambda name: name in ROW_WISE or (name == "dgate" and s["gate"].dim() == 2)
    return {name: tuple((np.concatenate if rows(name) else np.add.reduce)([p[name][i] for p in parts]) for i in (0, 1)) for name in parts[0]}


def tight(name, value, bound, share=0.05):
    """That a result is held to something: almost all bounds are small beside the numbers' size."""
    size = np.sqrt(np.mean(value ** 2))
    assert np.quantile(bound, 0.99) < share * size, f"{name}: bounds of {np.quantile(bound, 0.99):.2g} for numbers of {size:.2g}"
