"""Block norms of many rows: the kernels that large passes take (non-temporal accesses from 85 MB on), in all types and at rows of whole 16 bytes and others, and wide rows of which a
workgroup has more than one; values of every row and sums over all of them."""
import pytest
import torch

from block_rows import of_rows, tight
from paper_2412_12218_amd import binding as B
from test_gpu_block_norm import FORMS, given, matrix, run, run_back
from transformer_reference import check

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
PASS = 85 << 20     # bytes of the matrices of a pass from which on its accesses have the hint


def step(monkeypatch, n, d, dtype, form, ld=0, shift=0):
    """A training step against its formulas; the bytes of the matrices of its two passes."""
    has, post, gate, pre, _, _ = form
    s = given(n, d, dtype, form, seed=3, ld=ld, shift=shift)
    dH, dU = matrix(n, d, dtype, 9, d + ld, shift), matrix(n, d, dtype, 10)
    want = of_rows(monkeypatch, s, dH, dU, x_scale=0.875, post=post, pre=pre)
    stats = torch.full((n, 4), 7.0, device="cuda")
    H = torch.empty((n, d), dtype=dtype, device="cuda") if has else None
    H, U = run(s, form, H=H, stats=stats)
    grads = run_back(s, form, stats, dH=dH, dU=dU)
    got = dict(U=U, stats=stats, **{k: g for k, g in grads._asdict().items() if g is not None}, **(dict(H=H) if has else {}))
    assert set(got) - {"stats"} == set(want) - {"stats"} - (set() if has else {"H"})
    for name, t in got.items():
        check(f"{name} {dtype} {n} x {d} {form}", t, *want[name])
        if name != "stats":
            tight(name, *want[name])
    again = run_back(s, form, stats, dH=dH, dU=dU)
    assert all(a is b or torch.equal(a, b) for a, b in zip(grads, again))
    each = n * d * dtype.itemsize
    return each * (2 + 2 * has + (gate == "rows")), each * (4 + 2 * has + 2 * (gate == "rows"))


ALONE, GATE, BOTH, ROWS = FORMS[1], FORMS[3], FORMS[4], FORMS[5]


@pytest.mark.parametrize("n,d,dtype,form,ld,shift", [
    (75_001, 128, BF16, ROWS, 0, 0), (75_001, 128, F16, ROWS, 0, 0),           # narrow rows, several a wave
    (15_001, 768, F16, BOTH, 0, 0), (15_001, 768, BF16, BOTH, 8, 8),           # two waves a row
    (12_001, 1024, BF16, GATE, 0, 0), (11_601, 1032, F16, GATE, 0, 0),         # 128 and 192 lanes, all of them, or not
    (47_003, 250, BF16, BOTH, 0, 0), (5801, 2049, F16, BOTH, 3, 1), (59_001, 100, F32, FORMS[8], 3, 1), (24_001, 250, F32, GATE, 0, 0),   # rows that are not whole 16 bytes
    (115_001, 100, F32, ALONE, 0, 0), (230_001, 100, BF16, ALONE, 0, 0), (230_001, 100, F16, FORMS[0], 0, 0), (12_001, 999, F32, ALONE, 0, 0)],   # without a block
    ids=str)
def test_large_passes(monkeypatch, n, d, dtype, form, ld, shift):
    if form[3] == "none":
        s = given(n, d, dtype, form, seed=3, ld=ld, shift=shift)
        dH = matrix(n, d, dtype, 9)
        want = of_rows(monkeypatch, s, dH, None, x_scale=0.875, post=form[1], pre="none")
        H, _ = run(s, form)
        check("H", H, *want["H"])
        for name, got in run_back(s, form, None, dH=dH)._asdict().items():
            if got is not None:
                check(name, got, *want[name])
                tight(name, *want[name])
        assert 3 * n * d * dtype.itemsize <= PASS < 5 * n * d * dtype.itemsize     # the gradients' pass
        return
    forward, backward = step(monkeypatch, n, d, dtype, form, ld, shift)
    assert PASS < forward < backward


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,form", [(1100, 3080, BOTH), (1100, 4096, BOTH), (1101, 4095, ROWS), (700, 4100, BOTH), (699, 6001, GATE), (520, 8192, ROWS), (600, 8199, BOTH), (600, 8200, ROWS),
                                      (521, 10_000, ALONE), (400, 16_384, BOTH), (300, 16_383, GATE)], ids=str)
def test_wide_rows_in_turn(monkeypatch, dtype, n, d, form):
    """More rows than a launch has workgroups: of up to 512 lanes 512 forward and 256 backward, of 1024 lanes 256 of each."""
    step(monkeypatch, n, d, dtype, form)
    assert n > (512 if d <= 4096 else 256)


def test_large_pass_in_place():
    """h on top of x and dX on top of dH, in a pass with the hint."""
    for n, d, dtype in ((15_001, 768, BF16), (47_003, 250, F16)):
        s = given(n, d, dtype, BOTH)
        stats = torch.empty((n, 4), device="cuda")
        H, U = run(s, BOTH, stats=stats)
        dH, dU = matrix(n, d, dtype, 9), matrix(n, d, dtype, 10)
        want = run_back(s, BOTH, stats, dH=dH, dU=dU)
        got = run_back(s, BOTH, stats, dH=dH, dU=dU, dX=dH)
        assert all(a is b or torch.equal(a, b) for a, b in zip(got, want))
        X = s["X"].clone()
        h, u = run({**s, "X": X}, BOTH, H=X)
        assert torch.equal(X, H) and torch.equal(u, U)
