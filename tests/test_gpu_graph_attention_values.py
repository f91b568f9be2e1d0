"""Attention where numbers are unusual: rows without a key that hold NaN."""
import pytest
import torch

from test_gpu_graph_attention import DTYPES, Batch
from test_gpu_graph_attention_whole import Whole

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def spoil(t, n):
    """NaN and infinities in some of the first n rows, one kind a row."""
    for i, v in enumerate((NAN, INF, -INF)):
        t[i:n:5, i::7] = v


@pytest.mark.parametrize("kind", [Batch, Whole], ids=["odd", "whole"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [24, 64, 128])
@pytest.mark.parametrize("lens,qlens", [([50, 64, 3, 40], None), ([450, 64, 3, 700], None), ([2000, 70], [3, 1]), ([0, 90], [70, 2])],
                         ids=["one wave", "four waves", "parts", "no keys"])
def test_rows_without_a_key_are_zeros_whatever_they_hold(kind, dtype, D, lens, qlens):
    """A graph whose nodes are all masked, as those that fill a batch up: its queries and their gradients may be anything."""
    b = kind(lens, 2, 1, D, dtype, qlens=qlens, masked=0.3, seed=2)
    n = (qlens or lens)[0]
    b.mask[:lens[0]] = 0
    clean = b.run()
    spoil(b.Q, n), spoil(b.dO, n)
    got = b.run()
    for key in got:
        assert torch.equal(got[key], clean[key]), key
    assert bool((got["out"][:n] == 0).all()) and bool((got["lse"][:n] == -INF).all()) and bool((got["dQ"][:n] == 0).all())
    assert bool((got["dK"][:lens[0]] == 0).all()) and bool((got["dV"][:lens[0]] == 0).all())


@pytest.mark.parametrize("kind", [Batch, Whole], ids=["odd", "whole"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,qlens", [([150], None), ([700], None), ([3000], [4])], ids=["one wave", "four waves", "parts"])
def test_rows_that_hold_nan_and_see_a_key(kind, dtype, lens, qlens):
    """One key in the last tile is seen: rows of NaN give NaN, the others what they gave before."""
    b = kind(lens, 1, 1, 64, dtype, qlens=qlens, masked=0.3, seed=3)
    b.mask.fill_(0)
    b.mask[lens[0] - 1] = 1
    clean = b.run(False)
    b.Q[1, 5] = NAN
    got = b.run(False)
    keep = torch.arange(b.n_q, device="cuda") != 1
    assert torch.equal(got["out"][keep], clean["out"][keep]) and torch.equal(got["lse"][keep], clean["lse"][keep])
    assert bool(got["out"][1].isnan().all()) and bool(got["lse"][1].isnan().all())
