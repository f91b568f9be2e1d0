"""Attention inside the graphs of a packed batch where rows and heads are whole 16-byte pieces, as models lay them out: the kernels that load
straight to LDS, with one and four waves a workgroup, the other side whole and in parts, and every padded width.  Formulas and bounds as in
test_gpu_graph_attention.py, whose batches have odd rows."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from test_gpu_graph_attention import DTYPES, Batch, offsets

pytestmark = pytest.mark.gpu


class Whole(Batch):
    """Q, K, V column ranges of one matrix, or of two; a gap of 16 bytes behind the rows of every second batch."""

    def __init__(self, lens, heads, kv_heads, D, dtype, qlens=None, masked=0.0, seed=0, before=0, behind=0, spread=1.0):
        gen = torch.Generator().manual_seed(seed)
        gap = 16 // torch.empty(0, dtype=dtype).element_size() if seed % 2 else 0
        new = lambda n, c: torch.randn((n, c + gap), generator=gen).mul_(spread).to(dtype).cuda()[:, :c]
        self.heads, self.kv_heads, self.D = heads, kv_heads, D
        n_kv = before + sum(lens) + behind
        self.kv_ptr = offsets(lens, before)
        hd, kd = heads * D, kv_heads * D
        if qlens is None:
            self.q_ptr, n_q = self.kv_ptr, n_kv
            qkv = new(n_kv, hd + 2 * kd)
            self.Q, self.K, self.V = qkv[:, :hd], qkv[:, hd:hd + kd], qkv[:, hd + kd:]
        else:
            self.q_ptr, n_q = offsets(qlens, before), before + sum(qlens) + behind
            kv = new(n_kv, 2 * kd)
            self.Q, self.K, self.V = new(n_q, hd), kv[:, :kd], kv[:, kd:]
        self.dO = new(n_q, hd)
        self.n_q, self.n_kv, self.scale = n_q, n_kv, D ** -0.5
        self.mask = (torch.rand(n_kv, generator=gen) >= masked).to(torch.uint8).cuda() if masked else None
        for t in (self.Q, self.K, self.V, self.dO):
            e = t.element_size()
            assert t.data_ptr() % 16 == 0 and t.stride(0) * e % 16 == 0 and D * e % 16 == 0


def waves(rows, other, graphs, D):
    """Waves of a workgroup, as the launches choose them."""
    most = (160 if D <= 64 else 64) * graphs
    return 1 if rows <= 64 * graphs or (rows <= most and other <= most) else 4


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [8, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_one_wave(dtype, D, masked):
    """Graphs of a few tiles: ends inside a tile, of one row, of none."""
    for lens in ([1], [32, 64, 33], [5, 0, 64, 1, 31, 65, 40, 63]):
        assert waves(sum(lens), sum(lens), len(lens), D) == 1
        Whole(lens, 2, 2, D, dtype, masked=masked, seed=D + len(lens)).check(f"{dtype} D={D} {lens} masked {masked}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [8, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_four_waves(dtype, D, masked):
    """Graphs of several workgroups; whole tiles, ends inside one, waves without rows; few of them, so that the other side is in parts."""
    for lens in ([128, 256, 300], [513, 1, 170, 0, 700], [2051]):
        assert waves(sum(lens), sum(lens), len(lens), D) == 4 or D == 128
        Whole(lens, 2, 2, D, dtype, masked=masked, seed=D + len(lens)).check(f"{dtype} D={D} {lens} masked {masked}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (6, 2), (12, 4)])
@pytest.mark.parametrize("D", [8, 64, 96, 128])
def test_shared_heads(dtype, heads, kv_heads, D):
    """Several query heads to a K/V head, their rows in the same tiles."""
    for lens in ([23, 0, 40, 31], [330, 1, 200]):
        Whole(lens, heads, kv_heads, D, dtype, masked=0.2, seed=heads + len(lens)).check(f"{dtype} D={D} {heads} over {kv_heads} {lens}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [16, 64, 128])
@pytest.mark.parametrize("qlens,lens", [([1], [1]), ([1, 1, 1], [2000, 1, 900]), ([3, 0, 1, 2], [700, 50, 0, 64]), ([1000], [5]), ([2000, 3], [40, 0]),
                                        ([1] * 40, [60, 3] * 20), ([600, 20], [20, 600])], ids=lambda v: f"{len(v)}x{max(v)}")
def test_queries_of_their_own(dtype, D, qlens, lens):
    for heads, kv_heads in ((2, 2), (4, 1)):
        Whole(lens, heads, kv_heads, D, dtype, qlens=qlens, masked=0.1, seed=len(qlens) + heads).check(f"{dtype} D={D} {qlens[:4]} over {lens[:4]}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_workgroups(dtype):
    """Enough of them that the other side is not in parts, with four waves each."""
    Whole([300, 170, 250, 1, 0, 199] * 10, 8, 4, 32, dtype, masked=0.1, seed=5).check(f"{dtype} 60 graphs")
    Whole([300, 170, 250, 1, 0, 199] * 5, 8, 8, 128, dtype, seed=6).check(f"{dtype} 30 graphs of wide heads")


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_no_graph_stay(dtype):
    for qlens in (None, [2, 1, 0]):
        for lens in ([40, 0, 70], [400, 0, 270]):
            Whole(lens, 2, 1, 32, dtype, qlens=qlens, before=3, behind=9, seed=1).check(f"{dtype} rows outside")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [24, 64, 72, 128])
@pytest.mark.parametrize("lens", [[50, 64, 3, 40], [450, 64, 3, 700]], ids=["one wave", "four waves"])
def test_masks_and_what_they_hide(dtype, D, lens):
    """Hidden rows may hold anything, and so may the shared memory of a workgroup before: a batch of NaN runs ahead of every call."""
    b = Whole(lens, 2, 1, D, dtype, masked=0.5, seed=2)
    b.mask[:lens[0]] = 0
    hidden = b.mask == 0
    dirt = Whole(lens, 2, 1, 128, dtype, seed=3)
    dirt.Q.fill_(float("nan")), dirt.K.fill_(float("nan")), dirt.V.fill_(float("nan"))
    dirt.run()
    got = b.check(f"{dtype} D={D} masks")
    for t, bad in ((b.K, float("nan")), (b.V, float("inf"))):
        t[hidden] = torch.where(torch.arange(t.shape[1], device="cuda") % 3 == 0, bad, -1e4).to(dtype)
    dirt.run()
    again = b.run()
    for key in got:
        assert torch.equal(got[key], again[key]), key
    assert bool((got["out"][:lens[0]] == 0).all()) and bool((got["dQ"][:lens[0]] == 0).all())
    assert bool((got["dK"][hidden] == 0).all()) and bool((got["dV"][hidden] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_results_do_not_depend_on_the_layout(dtype):
    """Whole pieces and odd rows of the same numbers give the same bits."""
    for lens, D in (([40, 23, 64], 40), ([300, 513, 1], 40), ([300, 513, 1], 128)):
        b = Whole(lens, 4, 2, D, dtype, masked=0.2, seed=4)
        got = b.run()
        odd = lambda t: torch.cat([t, t[:, :1]], 1)[:, :t.shape[1]]
        b.Q, b.K, b.V, b.dO = odd(b.Q), odd(b.K), odd(b.V), odd(b.dO)
        assert b.Q.stride(0) % 2 == 1
        again = b.run()
        for key in got:
            assert torch.equal(got[key], again[key]), key


def largest_difference(run, inputs, grads, h):
    """For every input its directional difference along its gradient, which has the length of the gradient, and that length."""
    res = []
    for t, g in zip(inputs, grads):
        d = g.double() / g.double().norm()
        keep = t.clone()
        t.copy_((keep.double() + h * d).float())
        up, step = run(), t.double()
        t.copy_((keep.double() - h * d).float())
        step = (step - t.double())
        down = run()
        t.copy_(keep)
        res.append(((up - down).item(), (step * g.double()).sum().item()))
    return res


def test_gradient_along_itself():
    """Central differences of <out, dO> in fp32 along the gradient, where they are as large as they can be: 2 h |gradient|, 0.8 to 0.95 with h = 2^-5
    here.  The third-order term is below 3e-6 (in 64 bits).  out has 49 x 48 results of size up to 1, off by some (49 + 24) 2^-24 = 4e-6 with
    signs of their own, times |dO| of size 1: 48 4e-6 = 2e-4 in the sum; 4e-3 is twenty times that and half a percent of the difference."""
    for kind in (Batch, Whole):
        b = kind([40, 9], 2, 1, 24, torch.float32, masked=0.2, seed=6)
        got = b.run()
        f = lambda: (B.ftc_graph_attention(*b.args(), **b.kw()).double() * b.dO.double()).sum()
        for name, (diff, want) in zip(("dQ", "dK", "dV"), largest_difference(f, (b.Q, b.K, b.V), [got[k] for k in ("dQ", "dK", "dV")], 2.0 ** -5)):
            print(name, diff, want, flush=True)
            assert want > 20 * 4e-3, name          # a missing gradient, or one of the other sign, is far outside
            assert abs(diff - want) <= 4e-3, name
