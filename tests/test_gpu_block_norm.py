"""The norms before and after a block with its gate and residual connection, and their gradients, against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from block_reference import block
from paper_2412_12218_amd import binding as B
from transformer_reference import check

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
KINDS = dict(none=B.FTC_NORM_NONE, rms=B.FTC_NORM_RMS, layer=B.FTC_NORM_LAYER)


def matrix(n, d, dtype, seed, ld=None, shift=0, scale=1.0, mean=0.0):
    gen = torch.Generator().manual_seed(seed)
    ld = ld or d
    whole = (torch.randn(n * ld + shift, generator=gen) * scale + mean).to(dtype).cuda()
    return whole[shift:].view(n, ld)[:, :d]


def vector(d, dtype, seed, mean):
    return matrix(1, d, dtype, seed, scale=0.3, mean=mean)[0].contiguous()


# (F, post, gate, pre), weights of the norms, biases
FORMS = [(0, "none", "none", "rms", 1, 0), (0, "none", "none", "layer", 1, 1), (1, "none", "none", "rms", 1, 0), (1, "rms", "vector", "rms", 1, 0),
         (1, "layer", "vector", "layer", 1, 1), (1, "none", "rows", "layer", 0, 0), (1, "layer", "rows", "rms", 1, 1), (1, "rms", "none", "none", 0, 1),
         (1, "none", "vector", "none", 0, 0)]


def given(n, d, dtype, form, seed=0, ld=0, shift=0, mean=0.3):
    has, post, gate, pre, weights, biases = form
    w = lambda kind, on, s, m: vector(d, dtype, seed + s, m) if kind != "none" and on else None
    return dict(X=matrix(n, d, dtype, seed, d + ld, shift, 2.0, mean), F=matrix(n, d, dtype, seed + 1, d + 2 * ld, shift, 1.0, mean) if has else None,
                post_w=w(post, weights, 2, 1.0), post_b=w(post, biases, 3, 0.0), pre_w=w(pre, weights, 4, 1.0), pre_b=w(pre, biases, 5, 0.0),
                gate=dict(none=None, vector=vector(d, dtype, seed + 6, 0.5), rows=matrix(n, d, dtype, seed + 7, d + ld, 0, 0.5))[gate])


def run(s, form, x_scale=0.875, **k):
    args = {k: v for k, v in s.items() if k != "X"}
    return B.ftc_block_norm(s["X"], x_scale=x_scale, post=KINDS[form[1]], pre=KINDS[form[3]], **args, **k)


def run_back(s, form, stats, x_scale=0.875, **k):
    args = {k: v for k, v in s.items() if k != "X"}
    return B.ftc_block_norm_backward(s["X"], stats, x_scale=x_scale, post=KINDS[form[1]], pre=KINDS[form[3]], **args, **k)


def padded(n, d, dtype, pad):
    whole = torch.full((n, d + pad), 7.0, device="cuda", dtype=dtype)
    return whole, whole[:, :d]


SIZES = [(1, 1), (3, 1), (2, 2), (5, 7), (37, 8), (300, 20), (65, 32), (1, 33), (129, 64), (20, 100), (70, 128), (33, 200), (9, 257), (6, 512), (5, 777), (4, 1024), (3, 1433),
         (2, 2048), (3, 2056), (2, 4096), (1, 4100), (2, 8192), (1, 8199), (2, 10000), (1, 16384), (2000, 40), (3000, 96)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", SIZES)
def test_values_and_gradients(dtype, n, d):
    for i, form in enumerate(FORMS):
        has, post, gate, pre, weights, biases = form
        ld, shift = (0, 0) if i % 3 == 0 else (8, 8) if i % 3 == 1 else (3, 1)
        s = given(n, d, dtype, form, seed=i, ld=ld, shift=shift)
        dH = None if i % 4 == 3 and pre != "none" else matrix(n, d, dtype, 50 + i, d + ld)
        dU = None if pre == "none" else matrix(n, d, dtype, 60 + i, d + ld, shift)
        wide = i % 2 == 0
        wdt = torch.float32 if wide else dtype
        want = block(**s, x_scale=0.875, post=post, pre=pre, dH=dH, dU=dU, dw_dtype=wdt)
        H_all, H = padded(n, d, dtype, ld)
        U_all, U = padded(n, d, dtype, ld)
        stats = torch.full((n, 4), 7.0, device="cuda")
        name = f"{dtype} {n} x {d} {form}"
        run(s, form, H=H, U=U if pre != "none" else None, stats=stats)
        check(f"H {name}", H, *want["H"])
        if pre != "none":
            check(f"U {name}", U, *want["U"])
        check(f"stats {name}", stats, *want["stats"])
        assert bool((H_all[:, d:] == 7).all()) and bool((U_all[:, d:] == 7).all())
        dX_all, dX = padded(n, d, dtype, ld)
        grads = run_back(s, form, stats, dH=dH, dU=dU, dX=dX, dw_dtype=wdt)
        assert bool((dX_all[:, d:] == 7).all())
        for key, got in grads._asdict().items():
            if dU is None and key in ("dpre_w", "dpre_b"):  # nothing arrives there
                assert got is None or bool((got == 0).all())
                continue
            assert (got is not None) == (key in want), (key, name)
            if got is not None:
                assert got.dtype == (dtype if key in ("dX", "dF") or got.dim() == 2 else wdt)
                check(f"{key} {name}", got, *want[key])
        again = run_back(s, form, stats, dH=dH, dU=dU, dw_dtype=wdt)
        assert all(a is b or torch.equal(a, b) for a, b in zip(grads, again))


def test_only_what_is_wanted():
    form = FORMS[4]
    s = given(50, 72, torch.float16, form)
    stats = torch.empty((50, 4), device="cuda")
    H, U = run(s, form, stats=stats)
    dH, dU = matrix(50, 72, torch.float16, 9), matrix(50, 72, torch.float16, 10)
    full = run_back(s, form, stats, dH=dH, dU=dU)
    for name in full._fields:
        one = run_back(s, form, stats, dH=dH, dU=dU, want=(name,))
        for key, got in one._asdict().items():
            assert (got is None) == (key != name)
        assert torch.equal(getattr(one, name), getattr(full, name))
    # values without statistics, and without the one or the other output
    stream = torch.cuda.current_stream().cuda_stream
    only = torch.empty_like(U)
    b = B._block(s["X"], s["F"], 0.875, B.FTC_NORM_LAYER, s["post_w"], s["post_b"], s["gate"], B.FTC_NORM_LAYER, s["pre_w"], s["pre_b"], 1e-5)
    B._check(B.lib().ftc_block_norm(b, None, 0, only.data_ptr(), 72, None, stream))
    assert torch.equal(only, U)


def test_in_place():
    form = FORMS[3]
    for dtype in DTYPES:
        for d in (40, 520, 3000):
            s = given(70, d, dtype, form)
            stats = torch.empty((70, 4), device="cuda")
            H, U = run(s, form, stats=stats)
            dH, dU = matrix(70, d, dtype, 9), matrix(70, d, dtype, 10)
            want = run_back(s, form, stats, dH=dH, dU=dU)
            got = run_back(s, form, stats, dH=dH, dU=dU, dX=dH)
            assert all(a is b or torch.equal(a, b) for a, b in zip(got, want))
            X = s["X"].clone()
            h, u = run({**s, "X": X}, form, H=X)
            assert torch.equal(X, H) and torch.equal(u, U)


def test_no_rows_and_no_gradients():
    form = FORMS[4]
    s = given(0, 24, torch.bfloat16, form)
    H, U = run(s, form)
    assert H.shape == (0, 24) and U.shape == (0, 24)
    g = run_back(s, form, torch.empty((0, 4), device="cuda"), dU=s["X"])
    for v in (g.dgate, g.dpost_w, g.dpost_b, g.dpre_w, g.dpre_b):
        assert v.shape == (24,) and bool((v == 0).all())
    # no gradient arrives: zeros
    s = given(6, 24, torch.bfloat16, form)
    stats = torch.empty((6, 4), device="cuda")
    run(s, form, stats=stats)
    assert all(bool((v == 0).all()) for v in run_back(s, form, stats))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [20, 300, 1500, 9000])
def test_rows_of_unusual_numbers(dtype, d):
    """Zeros, equal numbers, a large mean, numbers whose squares fp32 does not hold; infinities and NaN stay in their row."""
    big = 1e30 if dtype != torch.float16 else 6e4
    for kind in ("rms", "layer"):
        X = matrix(9, d, torch.float32, 3)
        X[0] = 0
        X[1] = 3.5
        X[2] = X[2] * 0.25 + 1000
        X[3] = X[3] * big if dtype != torch.float16 else X[3].clamp(-1, 1) * big
        X[4] = X[4] * 1e-4
        X = X.to(dtype)
        w, b = vector(d, dtype, 1, 1.0), vector(d, dtype, 2, 0.0)
        want = block(X, None, 1.0, "none", None, None, None, kind, w, b)
        stats = torch.empty((9, 4), device="cuda")
        _, U = B.ftc_block_norm(X, pre=KINDS[kind], pre_w=w, pre_b=b, stats=stats)
        check(f"U {dtype} {d} {kind}", U, *want["U"])
        bad = X.clone()
        bad[5, d // 2], bad[6, 0], bad[7, d - 1] = float("nan"), float("inf"), -float("inf")
        _, V = B.ftc_block_norm(bad, pre=KINDS[kind], pre_w=w, pre_b=b, stats=stats)
        rest = [0, 1, 2, 3, 4, 8]
        assert torch.equal(V[rest], U[rest])
        assert bool(V[5].isnan().all()) and bool(V[6, 0].isnan()) and bool(V[7, d - 1].isnan())
        if kind == "rms":  # what lies beside an infinite number is nothing
            assert torch.equal(V[6, 1:], b[1:]) and torch.equal(V[7, :-1], b[:-1])
        else:
            assert bool(V[6:8].isnan().all())


def test_gradient_of_large_numbers():
    """Rows beyond 1e19: the factor is small, the gradients of a row are, too, and those of the weights are as ever."""
    d = 96
    X = matrix(4, d, torch.float32, 1) * 1e25
    w = vector(d, torch.float32, 2, 1.0)
    dU = matrix(4, d, torch.float32, 3)
    for kind in ("rms", "layer"):
        want = block(X, None, 1.0, "none", None, None, None, kind, w, None, dU=dU)
        stats = torch.empty((4, 4), device="cuda")
        B.ftc_block_norm(X, pre=KINDS[kind], pre_w=w, stats=stats)
        g = B.ftc_block_norm_backward(X, stats, dU=dU, pre=KINDS[kind], pre_w=w)
        check(f"dX {kind}", g.dX, *want["dX"])
        check(f"dw {kind}", g.dpre_w, *want["dpre_w"])


def test_many_rows():
    """More rows than a launch has row groups, and sums over all of them."""
    for n, d, dtype in ((70_001, 16, torch.bfloat16), (9000, 264, torch.float16), (5000, 1032, torch.float32)):
        form = FORMS[6]
        s = given(n, d, dtype, form, seed=11)
        stats = torch.empty((n, 4), device="cuda")
        dH, dU = matrix(n, d, dtype, 9), matrix(n, d, dtype, 10)
        want = block(**s, x_scale=0.875, post="layer", pre="rms", dH=dH, dU=dU)
        H, U = run(s, form, stats=stats)
        check("H", H, *want["H"])
        check("U", U, *want["U"])
        for key, got in run_back(s, form, stats, dH=dH, dU=dU)._asdict().items():
            if got is not None:
                check(key, got, *want[key])


def test_captured_and_on_another_stream():
    form = FORMS[4]
    s = given(300, 136, torch.float16, form)
    n, d, dtype = 300, 136, torch.float16
    stats = torch.empty((n, 4), device="cuda")
    dH, dU = matrix(n, d, dtype, 9), matrix(n, d, dtype, 10)
    H, U = torch.empty((n, d), dtype=dtype, device="cuda"), torch.empty((n, d), dtype=dtype, device="cuda")
    ws = B._workspace(B.lib().ftc_block_norm_backward_workspace_bytes(n, d), "cuda")
    grads = [t for t in run_back(s, form, torch.ones_like(stats), dH=dH, dU=dU)]
    names = B.BlockGrads._fields

    def step():
        run(s, form, H=H, U=U, stats=stats)
        run_back(s, form, stats, dH=dH, dU=dU, ws=ws, **dict(zip(names, grads)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    first = [t.clone() for t in [H, U, *grads]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        for t in (H, U, stats, ws, *grads):
            t.zero_()
        s["X"].mul_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, [H, U, *grads])), turn


@pytest.mark.parametrize("d", [20, 64, 250])
def test_rows_far_apart(d):
    """Rows of a workgroup beyond 2^31 bytes of each other, and a matrix beyond 2^32."""
    ld = 9_000_000
    whole = torch.zeros(130 * ld, dtype=torch.float16, device="cuda")
    X = whole.view(130, ld)[:, 5:5 + d]
    X.copy_(matrix(130, d, torch.float16, 1))
    near = X.contiguous()
    w, dU = vector(d, torch.float16, 2, 1.0), matrix(130, d, torch.float16, 3)
    stats, far_stats = torch.empty((130, 4), device="cuda"), torch.empty((130, 4), device="cuda")
    _, want = B.ftc_block_norm(near, pre=B.FTC_NORM_LAYER, pre_w=w, stats=stats)
    _, got = B.ftc_block_norm(X, pre=B.FTC_NORM_LAYER, pre_w=w, stats=far_stats)
    # other lanes have a row: sums of d numbers in another order
    ref = block(near, None, 1.0, "none", None, None, None, "layer", w, None, dU=dU)
    check("U", got, *ref["U"])
    check("U of near rows", want, *ref["U"])
    g = B.ftc_block_norm_backward(X, far_stats, dU=dU, pre=B.FTC_NORM_LAYER, pre_w=w)
    check("dX", g.dX, *ref["dX"])
    check("dpre_w", g.dpre_w, *ref["dpre_w"])


def test_two_streams_at_once():
    form = FORMS[4]
    n, d, dtype = 3000, 264, torch.bfloat16
    s = given(n, d, dtype, form)
    dH, dU = matrix(n, d, dtype, 9), matrix(n, d, dtype, 10)
    stats = torch.empty((n, 4), device="cuda")
    H, U = run(s, form, stats=stats)
    want = [H, U, *run_back(s, form, stats, dH=dH, dU=dU)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for turn in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                own = torch.empty((n, 4), device="cuda")
                h, u = run(s, form, stats=own)
                got[i] = [h, u, *run_back(s, form, own, dH=dH, dU=dU)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
