"""The oracle of the norms around a block: its gradients against differences of its values."""
import numpy as np
import pytest
import torch

import block_reference as R


@pytest.mark.parametrize("post,pre,gate", [("none", "rms", "none"), ("rms", "layer", "vector"), ("layer", "rms", "rows"), ("layer", "none", "vector")])
def test_gradients_along_a_direction(post, pre, gate):
    gen = torch.Generator().manual_seed(3)
    n, d = 5, 11
    new = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)
    norm = lambda kind, t: t if kind != "none" else None
    given = dict(X=new(n, d), F=new(n, d), post_w=norm(post, new(d)), post_b=norm(post, new(d)),
                 gate=dict(none=None, vector=new(d), rows=new(n, d))[gate], pre_w=norm(pre, new(d)), pre_b=norm(pre, new(d)))
    dH, dU = new(n, d), norm(pre, new(n, d))
    R.HALF_STEP[torch.float64], R.TINY[torch.float64] = 0.0, 0.0
    run = lambda at, **k: R.block(**at, x_scale=0.75, post=post, pre=pre, dw_dtype=torch.float64, **k)

    def loss(at):
        r = run(at)
        return (r["H"][0] * dH.numpy()).sum() + ((r["U"][0] * dU.numpy()).sum() if dU is not None else 0)
    grads = run(given, dH=dH, dU=dU)
    for name, t in given.items():
        if t is None:
            continue
        along, step = new(*t.shape), 1e-5
        moved = lambda s: loss({**given, name: t + s * along})
        want = (moved(step) - moved(-step)) / (2 * step)
        got = (grads["d" + name][0] * along.numpy()).sum()
        # third derivatives are below 1e3 here, roundings of a loss of 1e2 below 1e-13
        assert abs(got - want) < 1e-7 + 1e-7 * abs(want), (name, got, want)
