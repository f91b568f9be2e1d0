"""The norm over all gradients and their clipping against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2412_12218_amd import binding as B
from transformer_reference import HALF_STEP, S, TINY, check, f64

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def numbers(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def norm_of(grads, scale=1.0):
    """In 64 bits, where a sum of squares of n numbers is off by at most n 2^-53 of itself: below a step of fp32 for all that is here."""
    return abs(scale) * math.sqrt(sum(float((f64(g) ** 2).sum()) for g in grads))


def check_norm(got, want):
    check("norm", got, np.array([want]), np.array([want * (HALF_STEP[F32] + 2.0 ** -30) + TINY[F32]]))


def check_clipped(got, grads, scale, max_norm):
    norm = norm_of(grads, scale)
    factor = scale * min(1.0, max_norm / norm) if norm else scale
    for i, (o, g) in enumerate(zip(got, grads)):
        # the factor in 64 bits, the product rounded to fp32 and from there to the type
        want = f64(g) * factor
        check(f"{i}", o, want, np.abs(want) * (S * (g.dtype != F32) + HALF_STEP[g.dtype] + 2.0 ** -30) * (1 + 2.0 ** -8) + TINY[g.dtype] + TINY[F32])


SHAPES = [[(1,)], [(7,), (0,), (3, 5), (1, 1)], [(100, 33), (8,), (2, 3, 40)], [(8192,), (8193,), (8191,)], [(5,)] * 200, [(300, 1000), (3, 700, 90), (1000,)] * 5, [(2_000_003,), (9,)]]


@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)} {s[0]}")
def test_norm_and_clipping(shapes):
    for dtypes in ([F32], [F16], [BF16], [F16, F32, BF16]):
        grads = [numbers(s, dtypes[i % len(dtypes)], i, 1 + i % 3) for i, s in enumerate(shapes)]
        kept = [g.clone() for g in grads]
        for scale in (1.0, -0.125):
            norm = norm_of(grads, scale)
            check_norm(B.ftc_grad_norm(grads, scale=scale), norm)
            for limit in (0.4 * norm, 2 * norm, math.inf):
                out = [torch.empty_like(g) for g in grads]
                got = B.ftc_clip_grad_norm(B.GradList(grads, out=out), limit, scale=scale)
                check_norm(got, norm)
                check_clipped(out, grads, scale, limit)
                again = [g.clone() for g in grads]  # in place, and the same
                assert torch.equal(B.ftc_clip_grad_norm(again, limit, scale=scale), got)
                assert all(torch.equal(a, b) for a, b in zip(again, out))
        assert all(torch.equal(a, b) for a, b in zip(grads, kept))


# on both sides of the number of tensors, and of numbers, from which on a program asks for other chunks, and of those
@pytest.mark.parametrize("shapes", [[(2048,), (2047,), (2049,), (4096,)], [(40, 77)] * 32, [(40, 77)] * 33, [(2 ** 20 - 9,), (9,)], [(2 ** 20 - 9,), (10,)],
                                    [(7,)] * 139 + [(2 ** 20 - 7 * 139,)], [(7,)] * 140 + [(2 ** 20,)], [(1, 3000)] * 300], ids=lambda s: f"{len(s)} {s[0]} {s[-1]}")
def test_chunks(shapes):
    for dtype in (F32, BF16):
        grads = [numbers(s, dtype, i) for i, s in enumerate(shapes)]
        norm = norm_of(grads)
        out = [torch.full_like(g, 7) for g in grads]
        got = B.ftc_clip_grad_norm(B.GradList(grads, out=out), 0.3 * norm)
        check_norm(got, norm)
        check_clipped(out, grads, 1.0, 0.3 * norm)
        assert torch.equal(B.ftc_grad_norm(grads), got)
        B.ftc_clip_grad_norm(grads, 0.3 * norm)
        assert all(torch.equal(a, b) for a, b in zip(grads, out))


def test_below_the_limit_everything_stays():
    grads = [numbers((50, 30), t, i) for i, t in enumerate((F32, F16, BF16))]
    kept = [g.clone() for g in grads]
    B.ftc_clip_grad_norm(grads, 1e4)
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    # at the limit itself, too
    t = torch.tensor([3.0, 4.0], device="cuda")
    assert B.ftc_clip_grad_norm([t], 5.0).item() == 5.0 and t.tolist() == [3.0, 4.0]
    B.ftc_clip_grad_norm([t], 0.0)
    assert t.tolist() == [0.0, 0.0]
    B.ftc_clip_grad_norm([t], 0.0)   # of nothing: nothing
    assert t.tolist() == [0.0, 0.0]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_column_ranges_of_a_matrix(dtype):
    for rows, width, cut, shift in ((70, 40, 16, 0), (333, 101, 33, 3), (5, 9000, 8191, 1), (4000, 3, 1, 0)):
        base = numbers((rows * width + shift,), dtype, rows)[shift:].view(rows, width)
        kept = base.clone()
        parts = [base[:, :cut], base[:, cut:]]
        want = norm_of(parts)
        check_norm(B.ftc_grad_norm(parts), want)
        wide = torch.full((rows, width + 5), 7.0, dtype=dtype, device="cuda")
        out = [wide[:, :cut], torch.empty((rows, width - cut), dtype=dtype, device="cuda")]
        B.ftc_clip_grad_norm(B.GradList(parts, out=out), 0.3 * want)
        check_clipped(out, parts, 1.0, 0.3 * want)
        assert bool((wide[:, cut:] == 7).all()) and torch.equal(base, kept)
        B.ftc_clip_grad_norm([parts[1]], 0.3 * norm_of(parts[1:]))   # in place: the other columns stay
        assert torch.equal(base[:, :cut], kept[:, :cut])
        check_clipped([base[:, cut:]], [kept[:, cut:]], 1.0, 0.3 * norm_of([kept[:, cut:]]))


def test_large_and_small_numbers():
    """Squares that fp32 does not hold, and norms next to its ends."""
    for value in (1e30, 1e-30, 3e38, 1e-42):
        t = torch.full((1000,), value, device="cuda")
        want = norm_of([t])
        if want < 3.4e38:
            check_norm(B.ftc_grad_norm([t]), want)
        else:
            assert B.ftc_grad_norm([t]).item() == math.inf    # the number is not one of fp32; clipping has it in 64 bits
        out = torch.empty_like(t)
        B.ftc_clip_grad_norm(B.GradList([t], out=[out]), 1e-3 * value)
        clipped = f64(t) * (1e-3 * value / want)
        check("clipped", out, clipped, np.abs(clipped) * 2.0 ** -23 + 2 * TINY[F32])
    mixed = [torch.full((3,), 1e25, device="cuda"), torch.full((10**6,), 1.0, device="cuda")]
    check_norm(B.ftc_grad_norm(mixed), norm_of(mixed))


def test_infinities_and_nan():
    for bad, others in ((math.inf, 0.0), (math.nan, math.nan)):
        t, u = torch.ones(20, device="cuda"), torch.ones(5000, device="cuda").half()
        t[3] = bad
        norm = B.ftc_clip_grad_norm([t, u], 1.0).item()
        assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
        assert math.isnan(t[3].item())
        assert bool(u.isnan().all()) if math.isnan(others) else bool((u == 0).all())


def test_nothing():
    assert B.ftc_grad_norm([]).item() == 0 and B.ftc_clip_grad_norm([], 1.0).item() == 0
    empty = [torch.empty((0, 5), device="cuda"), torch.empty(0, device="cuda").half()]
    assert B.ftc_grad_norm(empty).item() == 0 and B.ftc_clip_grad_norm(empty, 1.0).item() == 0


def test_the_same_every_time():
    grads = [numbers((1001, 999), F32, 1), numbers((77_777,), BF16, 2)]
    first = B.ftc_grad_norm(grads)
    assert all(torch.equal(B.ftc_grad_norm(grads), first) for _ in range(5))


def test_captured_and_on_another_stream():
    grads = [numbers((300, 200), F32, 1), numbers((9000,), F16, 2)] + [numbers((40,), BF16, i) for i in range(70)]
    kept = [g.clone() for g in grads]
    norm, listed = torch.empty(1, device="cuda"), B.GradList(grads)
    ws = B._workspace(listed.workspace_bytes(), "cuda")
    limit = 0.5 * norm_of(grads)
    want = [g.clone() for g in grads]
    want_norm = B.ftc_clip_grad_norm(want, limit)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.ftc_clip_grad_norm(listed, limit, norm=norm, ws=ws)
    side.synchronize()
    assert torch.equal(norm, want_norm) and all(torch.equal(a, b) for a, b in zip(grads, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ftc_clip_grad_norm(listed, limit, norm=norm, ws=ws)
    for turn in range(3):
        for g, k in zip(grads, kept):
            g.copy_(k)
        norm.zero_()
        ws.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want_norm) and all(torch.equal(a, b) for a, b in zip(grads, want)), turn


def test_gradients_beyond_32_bits():
    """A tensor of more than 2^31 numbers and 2^32 bytes; equal numbers, so the sums are known."""
    n = 2 ** 31 + 12_345
    t = torch.full((n,), 0.5, dtype=F16, device="cuda")
    t[-1] = 2.0
    want = math.sqrt((n - 1) * 0.25 + 4.0)
    check_norm(B.ftc_grad_norm([t]), want)
    B.ftc_clip_grad_norm([t], want / 2)      # halves
    assert bool((t[:-1] == 0.25).all()) and t[-1].item() == 1.0
    wide = torch.zeros((70_000, 33_000), dtype=F16, device="cuda")[:, :3]   # rows 66 kB apart, the last beyond 2^32 bytes
    wide.fill_(0.5)
    check_norm(B.ftc_grad_norm([wide]), math.sqrt(210_000 * 0.25))
    B.ftc_clip_grad_norm([wide], math.sqrt(210_000 * 0.25) / 2)
    assert bool((wide == 0.25).all())
