"""Attention where numbers are unusual: rows without a key that hold NaN, long rows whose maximum stays while others' rises, scales next to zero."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from test_gpu_graph_attention import DTYPES, Batch, offsets
from test_gpu_graph_attention_whole import Whole
from transformer_reference import attention

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


def test_long_rows_beside_rows_whose_maximum_rises():
    """Every 32nd query finds a larger score in every tile of keys; the largest of the others is that of the first key, 40 to 60, which has about half of
    their weight, and the other 8191 share the rest.  Weights that the first key has must not change with the tiles that follow: out in
    column 0 is p_0 - (1 - p_0).

    lse is a sum with roundings of half a step of 16 to 128 each (score 1.9e-6, in base two 2.6e-6, result 1.9e-6) and of the sum itself, 4096 additions
    in a lane, half a step of 0.5 to 1 each with random signs: 64 / sqrt(3) 2^-25, five times that 5.5e-6: 1.2e-5; out the same in p_0 (1 - p_0) twice, and
    8192 additions into a sum of up to 1: five times 90 / sqrt(3) 2^-25, 8e-6: 1.4e-5.  Both are given twice that."""
    n_q, n, D = 33_024, 8192, 16   # enough queries that the keys stay in one part
    gen = torch.Generator().manual_seed(5)
    Q, K, V = torch.zeros((n_q, D)), torch.zeros((n, D)), torch.randn((n, D), generator=gen)
    Q[:, 1] = 160 + 80 * torch.rand(n_q, generator=gen)
    Q[::32] = 0
    Q[::32, 0] = 200.0
    K[:, 0] = torch.arange(n) / n
    K[:, 1] = 1 - 36 / 200 * (1 + 0.2 * (torch.rand(n, generator=gen) - 0.5))
    K[0, 1] = 1
    V[:, 0], V[0, 0] = -1, 1
    out, lse = torch.empty((n_q, D), device="cuda"), torch.empty((n_q, 1), device="cuda")
    B.ftc_graph_attention(Q.cuda(), K.cuda(), V.cuda(), offsets([n_q]), offsets([n]), heads=1, scale=0.25, out=out, lse=lse)
    for some in (slice(0, 128), slice(16_384, 16_512), slice(n_q - 128, n_q)):
        s = Q[some].double() @ K.double().t() * 0.25
        want = torch.softmax(s, 1) @ V.double()
        off_lse = (lse[some, 0].cpu().double() - torch.logsumexp(s, 1)).abs().max().item()
        off = (out[some, 0].cpu().double() - want[:, 0]).abs().max().item()
        print(f"lse {off_lse:.2e}, out {off:.2e}", flush=True)
        assert off_lse <= 2.4e-5 and off <= 2.8e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-36, -1e-36])
def test_scales_next_to_zero(dtype, scale):
    """Products of 1e31 and more: a scale of zero leaves nothing of them, 1e-36 only 1e-4."""
    for kind, lens in ((Batch, [90, 5, 33]), (Whole, [90, 5, 33]), (Whole, [300, 170])):
        b = kind(lens, 4, 2, 32, dtype, masked=0.3, seed=13)
        b.Q.mul_(1e15), b.K.mul_(1e15)
        b.scale = scale
        got = b.run(False)
        at = 0
        for n in lens:
            seen = b.mask[at:at + n] != 0
            s = scale * b.Q[at:at + n, :32].double() @ b.K[at:at + n, :32][seen].double().t()
            want = torch.softmax(s, 1) @ b.V[at:at + n, :32][seen].double()
            u = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
            bound = (2 * u + 2 * (n + 60) * 2.0 ** -24) * b.V.double().abs().max()   # p and out are rounded, sums of n and of 32 products
            off = (got["out"][at:at + n, :32].double() - want).abs().max()
            assert off <= bound, (lens, float(off), float(bound))
            at += n


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [8, 20, 32])
@pytest.mark.parametrize("qlens,lens", [([400], [400]), ([6], [2000]), ([3, 1, 2], [700, 900, 40])], ids=["whole", "parts", "parts of some"])
def test_gradients_where_values_have_a_mean(dtype, D, qlens, lens):
    """V around ten: <dO, out> of a rounded out is off by ten times the half steps of what ds is made of.  With D up to 32 dQ and dK are as far off as
    results that are only rounded, or a few times that: 2.5 in the 2-norm (the roundings of dQ itself, of two operands of ds and of lse are 1.5)."""
    for heads, kv_heads in ((1, 1), (2, 1)):
        b = Whole(lens, heads, kv_heads, D, dtype, qlens=qlens, seed=7) if D % 8 == 0 else Batch(lens, heads, kv_heads, D, dtype, qlens=qlens, seed=7)
        b.V.add_(10)
        got, want = b.run(), attention(*b.args(), heads, kv_heads, b.scale, None, b.dO)
        for key in ("dQ", "dK"):
            exact = torch.from_numpy(want[key][0])
            rounded = (exact.to(dtype).double() - exact).norm()
            off = (got[key].cpu().double() - exact).norm()
            print(f"{dtype} D={D} {qlens} {key}: {off / rounded:.2f}", flush=True)
            assert off <= 2.5 * rounded, key
