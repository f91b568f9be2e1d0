"""The dense layer with weights for every group of rows, and its gradients, against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from block_reference import grouped, grouped_backward
from paper_2412_12218_amd import binding as B
from transformer_reference import check, slope_values

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = dict(none=B.FTC_ACT_NONE, relu=B.FTC_ACT_RELU, gelu=B.FTC_ACT_GELU, silu=B.FTC_ACT_SILU)


def matrix(n, d, dtype, seed, ld=None, shift=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    ld = ld or d
    whole = (torch.randn(n * ld + shift, generator=gen) * scale).to(dtype).cuda()
    return whole[shift:].view(n, ld)[:, :d]


def offsets(ptr):
    return torch.tensor(ptr, dtype=torch.int32, device="cuda")


def layer(n, groups, d_in, d_out, dtype, seed=0, bias=True, residual=True, ldx=None, shift=0):
    W = matrix(groups * d_in, d_out, dtype, seed + 1, scale=d_in ** -0.5).view(groups, d_in, d_out)
    return matrix(n, d_in, dtype, seed, ldx, shift), W, matrix(groups, d_out, dtype, seed + 2) if bias else None, \
        matrix(n, d_out, dtype, seed + 3, d_out + 1) if residual else None


# offsets (the last one's row is the number of rows unless rows follow it), widths
SHAPES = [([0, 1], 1, 1, 1), ([0, 0, 1, 1], 1, 40, 30), ([0, 3, 3, 8, 8, 20], 20, 33, 65), ([2, 5, 70, 70, 135], 140, 64, 64), ([0, 64, 128, 192], 192, 72, 136),
          ([0, 63, 128, 193, 193, 321], 321, 100, 129), ([5, 5, 5], 9, 16, 24), ([0, 130, 131, 600], 600, 256, 264), ([0] * 40 + [7] * 60 + [9] * 30, 9, 24, 40),
          ([0, 2, 4, 5], 6, 2000, 70), ([0, 1, 2, 3, 40], 40, 1030, 7), ([3, 1500, 1600], 1605, 16, 9), ([0, 2500, 2500, 3000], 3000, 40, 32)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ptr,n,d_in,d_out", SHAPES, ids=lambda x: str(x)[:20])
def test_forward_and_slope(dtype, ptr, n, d_in, d_out):
    groups = len(ptr) - 1
    rows = np.zeros(n, bool)
    rows[ptr[0]:ptr[-1]] = True
    for i, act in enumerate(ACTS):
        X, W, b, R = layer(n, groups, d_in, d_out, dtype, seed=i, bias=i % 2 == 0, residual=i >= 2, ldx=d_in + 3 * (i % 2), shift=i % 3)
        for out_dtype in {dtype, torch.float32}:
            slope = torch.full((n, d_out + 2), 7, device="cuda", dtype=B.slope_like(X).dtype)
            out = torch.full((n, d_out + 3), 7.0, device="cuda", dtype=out_dtype)
            B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=ACTS[act], residual=R, out=out[:, :d_out], slope=slope[:, :d_out])
            (z, dz), (s, ds), sure = grouped(X, W, ptr, b, act, R, out_dtype)
            check(f"Z {dtype} {ptr[:8]} {d_in} {d_out} {act} -> {out_dtype}", out[:, :d_out][torch.from_numpy(rows).cuda()], z[rows], dz[rows])
            got = slope_values(slope[:, :d_out])
            assert np.all(np.abs(got - s)[sure] <= ds[sure])
            for t in (out, slope):
                assert bool((t[:, d_out:] == 7).all()) and bool((t[torch.from_numpy(~rows).cuda()] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ptr,n,d_in,d_out", SHAPES, ids=lambda x: str(x)[:20])
def test_backward(dtype, ptr, n, d_in, d_out):
    groups, rows = len(ptr) - 1, slice(ptr[0], ptr[-1])
    for act in ("none", "gelu"):
        X, W, b, _ = layer(n, groups, d_in, d_out, dtype, seed=7, residual=False, ldx=d_in + 1)
        dZ = matrix(n, d_out, dtype, 99, d_out + 3, 1)
        slope = None
        if act != "none":
            slope = B.slope_like(dZ).zero_()
            B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=ACTS[act], slope=slope)
        for wide in (False, True):
            dt = torch.float32 if wide else dtype
            dX = torch.full((n, d_in + 5), 7.0, device="cuda", dtype=dt)
            gx, dW, db = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dX=dX[:, :d_in], dw_dtype=dt)
            want = grouped_backward(X, W, ptr, dZ, slope, dt, dt)
            name = f"{dtype} {ptr[:8]} {d_in} {d_out} {act} -> {dt}"
            check(f"dX {name}", gx[rows], want[0][0][rows], want[0][1][rows])
            check(f"dW {name}", dW, *want[1])
            check(f"db {name}", db, *want[2])
            assert bool((dX[:, d_in:] == 7).all()) and bool((dX[:ptr[0]] == 7).all()) and bool((dX[ptr[-1]:] == 7).all())
            again = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dx_dtype=dt, dw_dtype=dt)
            assert torch.equal(again[0][rows], gx[rows]) and torch.equal(again[1], dW) and torch.equal(again[2], db)


# sizes at which a program asks for tiles of 128 and 256 and for parts, on the whole-piece kernels
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,d_in,d_out", [([3000, 0, 517, 1, 2600], 256, 384), ([40, 5000, 129], 1024, 512), ([300] * 20, 128, 264), ([2, 0, 1, 3], 4096, 512),
                                             ([9000], 64, 64), ([1, 2, 0, 1] * 16, 512, 1032)], ids=str)
def test_larger(dtype, lens, d_in, d_out):
    ptr = np.cumsum([0] + lens).tolist()
    n = ptr[-1]
    X, W, b, R = layer(n, len(lens), d_in, d_out, dtype)
    slope = B.slope_like(R[:, :d_out].contiguous())
    out = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_SILU, residual=R, slope=slope)
    (z, dz), _, _ = grouped(X, W, ptr, b, "silu", R, dtype)
    check(f"Z {dtype} {lens[:6]} {d_in} {d_out}", out, z, dz)
    dZ = matrix(n, d_out, dtype, 5)
    add = matrix(n, d_in, dtype, 6)
    want = grouped_backward(X, W, ptr, dZ, slope, dtype, dtype)
    dX, dW, db = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dw_dtype=dtype)
    for name, got, (value, bound) in zip(("dX", "dW", "db"), (dX, dW, db), want):
        check(f"{name} {dtype} {lens[:6]} {d_in} {d_out}", got, value, bound)
    wide = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dX_add=add, dx_dtype=torch.float32, want_dW=False, want_db=False)[0]
    narrow = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dX_add=add, dX=add.clone(), want_dW=False, want_db=False)[0]
    inplace = add.clone()
    B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, dX_add=inplace, dX=inplace, want_dW=False, want_db=False)
    assert torch.equal(inplace, narrow) and torch.equal(narrow, wide.to(dtype))


@pytest.mark.parametrize("groups", [63, 64, 65, 200, 512, 513, 3000])
def test_many_groups(groups):
    """Of no row, of one, and of several tiles, in front of which and behind which there are rows of no group."""
    lens = [(0, 1, 3, 0, 130)[(i * i + i // 7) % 5] if i % 50 else 300 for i in range(groups)]
    lens = [x if sum(lens) < 40_000 else min(x, 9) for x in lens]
    ptr = (np.cumsum([0] + lens) + 3).tolist()
    n, rows = ptr[-1] + 5, slice(3, ptr[-1])
    for dtype, d_in, d_out in ((torch.float16, 16, 24), (torch.float32, 9, 8)):
        X, W, b, _ = layer(n, groups, d_in, d_out, dtype, residual=False)
        slope = B.slope_like(X.new_empty((n, d_out))).zero_()
        out = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_SILU, slope=slope)
        (z, dz), _, _ = grouped(X, W, ptr, b, "silu", None, dtype)
        check(f"Z {groups} {dtype}", out[rows], z[rows], dz[rows])
        dZ = matrix(n, d_out, dtype, 5)
        dX, dW, db = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope)
        want = grouped_backward(X, W, ptr, dZ, slope, dtype, torch.float32)
        check(f"dX {groups} {dtype}", dX[rows], want[0][0][rows], want[0][1][rows])
        check(f"dW {groups} {dtype}", dW, *want[1])
        check(f"db {groups} {dtype}", db, *want[2])


def test_one_group_is_the_dense_layer():
    """The same sums, perhaps in other parts: each is within the bound of the formula, so they are within twice that of each other."""
    for dtype in DTYPES:
        X, W, b, R = layer(700, 1, 136, 200, dtype)
        want = B.ftc_linear(X, W[0], bias=b[0].contiguous(), act=B.FTC_ACT_GELU, residual=R)
        got = B.ftc_grouped_linear(X, W, offsets([0, 700]), bias=b, act=B.FTC_ACT_GELU, residual=R)
        (_, dz), _, _ = grouped(X, W, [0, 700], b, "gelu", R, dtype)
        check(f"{dtype}", got, want.double().cpu().numpy(), 2 * dz)


def test_parts_of_the_gradient():
    ptr = offsets([0, 30, 30, 70])
    X, W, b, _ = layer(70, 3, 40, 50, torch.float16, residual=False)
    slope = torch.empty((70, 50), dtype=torch.int16, device="cuda")
    B.ftc_grouped_linear(X, W, ptr, bias=b, act=B.FTC_ACT_SILU, slope=slope)
    dZ = matrix(70, 50, torch.float16, 5)
    dX, dW, db = B.ftc_grouped_linear_backward(X, W, ptr, dZ, slope=slope)
    only = lambda **k: B.ftc_grouped_linear_backward(X, W, ptr, dZ, slope=slope, **{**dict(want_dX=False, want_dW=False, want_db=False), **k})
    assert torch.equal(only(want_dX=True)[0], dX) and torch.equal(only(want_dW=True)[1], dW) and torch.equal(only(want_db=True)[2], db)
    assert only() == (None, None, None)


def test_no_rows_and_no_groups():
    W = matrix(3 * 8, 16, torch.bfloat16, 1).view(3, 8, 16)
    X = torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")
    ptr = offsets([0, 0, 0, 0])
    assert B.ftc_grouped_linear(X, W, ptr).shape == (0, 16)
    dX, dW, db = B.ftc_grouped_linear_backward(X, W, ptr, torch.empty((0, 16), dtype=torch.bfloat16, device="cuda"))
    assert bool((dW == 0).all()) and bool((db == 0).all()) and dW.shape == (3, 8, 16)
    X = matrix(5, 8, torch.bfloat16, 2)
    out = torch.full((5, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    B.ftc_grouped_linear(X, W[:0], offsets([0]), out=out)
    B.ftc_grouped_linear(X, W, offsets([5, 5, 5, 5]), out=out)
    assert bool((out == 7).all())
    # rows, none of them in a group: no gradient arrives at the weights
    _, dW, db = B.ftc_grouped_linear_backward(X, W, offsets([2, 2, 2, 2]), matrix(5, 16, torch.bfloat16, 3))
    assert bool((dW == 0).all()) and bool((db == 0).all())


def test_offsets_outside_the_rows():
    """Taken as the nearest end."""
    X, W, b, _ = layer(100, 3, 24, 40, torch.float16, residual=False)
    want = B.ftc_grouped_linear(X, W, offsets([0, 30, 100, 100]), bias=b)
    got = B.ftc_grouped_linear(X, W, offsets([-5, 30, 300, 1000]), bias=b)
    assert torch.equal(got, want)
    dZ = matrix(100, 40, torch.float16, 4)
    want = B.ftc_grouped_linear_backward(X, W, offsets([0, 30, 100, 100]), dZ)
    got = B.ftc_grouped_linear_backward(X, W, offsets([-5, 30, 300, 1000]), dZ)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_unusual_numbers_stay_in_their_group():
    """NaN and infinities of one group's rows and weights reach no other group, nor do those in the rows of no group."""
    ptr = [2, 40, 77, 100]
    for dtype in DTYPES:
        for d_in, d_out in ((64, 72), (50, 33)):
            X, W, b, _ = layer(103, 3, d_in, d_out, dtype, residual=False)
            dZ = matrix(103, d_out, dtype, 4)
            want = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b), *B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ)
            for t in (X, dZ):
                t[:2], t[100:] = float("nan"), float("inf")
                t[50, 3] = float("nan")
            W[1, 5, 7] = float("inf")
            got = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b), *B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ)
            for part in (slice(2, 40), slice(77, 100)):
                assert torch.equal(got[0][part], want[0][part]) and torch.equal(got[1][part], want[1][part])
            assert torch.equal(got[2][[0, 2]], want[2][[0, 2]]) and torch.equal(got[3][[0, 2]], want[3][[0, 2]])
            assert bool(got[0][50].isnan().all()) and bool(got[3][1, 3].isnan())


def test_captured_and_on_another_stream():
    lens = [500, 0, 90, 1200]
    ptr = np.cumsum([0] + lens).tolist()
    n, d_in, d_out, dtype = ptr[-1], 128, 192, torch.bfloat16
    X, W, b, _ = layer(n, 4, d_in, d_out, dtype, residual=False)
    dZ, at = matrix(n, d_out, dtype, 4), offsets(ptr)
    out, slope = torch.empty((n, d_out), dtype=dtype, device="cuda"), torch.empty((n, d_out), dtype=torch.int16, device="cuda")
    dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty_like(b)
    ws = B._workspace(max(B.lib().ftc_grouped_linear_workspace_bytes(n, 4, d_in, d_out), B.lib().ftc_grouped_linear_backward_workspace_bytes(n, 4, d_in, d_out)), "cuda")

    def step():
        B.ftc_grouped_linear(X, W, at, bias=b, act=B.FTC_ACT_GELU, out=out, slope=slope, ws=ws)
        B.ftc_grouped_linear_backward(X, W, at, dZ, slope=slope, dX=dX, dW=dW, db=db, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    first = [t.clone() for t in (out, dX, dW, db)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        for t in (out, slope, dX, dW, db, ws):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (out, dX, dW, db))), turn
    # other groups of the same rows through the same graph: the offsets are read when it runs
    other = np.cumsum([0, 1, 1000, 700, 89]).tolist()
    at.copy_(offsets(other))
    graph.replay()
    want = B.ftc_grouped_linear(X, W, offsets(other), bias=b, act=B.FTC_ACT_GELU, slope=B.slope_like(out))
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens", [[2600, 0, 1100, 700, 1], [8000, 3], [300] * 16], ids=str)
def test_last_turn_in_parts(dtype, lens):
    """More tiles of 256 than compute units, the last ones in parts of the contraction; in both directions, with bias, activation, residual and slopes."""
    d_in, d_out = 4096, 4104   # 340, 561 and 544 tiles of Z
    ptr = np.cumsum([0] + lens).tolist()
    n = ptr[-1]
    X, W, b, R = layer(n, len(lens), d_in, d_out, dtype)
    slope = B.slope_like(R[:, :d_out].contiguous())
    out = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_SILU, residual=R, slope=slope)
    dZ = matrix(n, d_out, dtype, 5)
    dX = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, slope=slope, want_dW=False, want_db=False)[0]
    again = B.ftc_grouped_linear(X, W, offsets(ptr), bias=b, act=B.FTC_ACT_SILU, residual=R)
    assert torch.equal(out, again)
    rows = torch.cat([torch.arange(max(0, p - 5), min(n, p + 5)) for p in ptr] + [torch.arange(n - 40, n), torch.arange(0, n, 97)]).unique()
    for g, (a, e) in enumerate(zip(ptr, ptr[1:])):
        at = rows[(rows >= a) & (rows < e)].cuda()
        if len(at):
            (z, dz), (s, ds), _ = grouped(X[at], W[g:g + 1], [0, len(at)], b[g:g + 1], "silu", R[at], dtype)
            check(f"Z {g}", out[at], z, dz)
            assert np.all(np.abs(slope_values(slope[at]) - s) <= ds)
            want, bound = grouped_backward(X[at], W[g:g + 1], [0, len(at)], dZ[at], slope[at], dtype, dtype)[0]
            check(f"dX {g}", dX[at], want, bound)


def test_weights_beyond_32_bits():
    """More than 2^32 bytes of weights, the last group's behind all of them."""
    groups, d_in, d_out = 600, 2048, 2048
    W = torch.zeros((groups, d_in, d_out), dtype=torch.float16, device="cuda")
    W[-1] = matrix(d_in, d_out, torch.float16, 1, scale=d_in ** -0.5)
    X, dZ = matrix(70, d_in, torch.float16, 2), matrix(70, d_out, torch.float16, 3)
    for first in (0, 64):   # rows in front of it: of the group before
        ptr = [0] * (groups - 1) + [first, 70]
        out = B.ftc_grouped_linear(X, W, offsets(ptr))
        at = slice(first, 70)
        (z, dz), _, _ = grouped(X[at], W[-1:], [0, 70 - first], None, "none", None, torch.float16)
        check("Z", out[at], z, dz)
        assert bool((out[:first] == 0).all())
        dX, dW, db = B.ftc_grouped_linear_backward(X, W, offsets(ptr), dZ, dw_dtype=torch.float16)
        want = grouped_backward(X[at], W[-1:], [0, 70 - first], dZ[at], None, torch.float16, torch.float16)
        check("dX", dX[at], *want[0])
        check("dW", dW[-1:], *want[1])
        check("db", db[-1:], *want[2])
        assert bool((dW[:groups - 2] == 0).all()) and bool((db[:groups - 2] == 0).all())


def test_two_streams_at_once():
    lens = [900, 0, 77, 2000, 3]
    ptr = np.cumsum([0] + lens).tolist()
    X, W, b, _ = layer(ptr[-1], 5, 256, 320, torch.bfloat16, residual=False)
    dZ, at = matrix(ptr[-1], 320, torch.bfloat16, 4), offsets(ptr)

    def step():
        slope = B.slope_like(dZ)
        return [B.ftc_grouped_linear(X, W, at, bias=b, act=B.FTC_ACT_GELU, slope=slope), *B.ftc_grouped_linear_backward(X, W, at, dZ, slope=slope)]
    want = step()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for turn in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i] = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
