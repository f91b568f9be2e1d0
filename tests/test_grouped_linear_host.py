"""What the grouped dense layer refuses, on the host, before anything is launched (the pointers are never followed); and the numbers by which its kernels find
their groups, for groups of all kinds.  CPU only."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

from paper_2412_12218_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = lambda i: 0x10000 * i
INVALID, UNSUPPORTED, ALIGN, WORKSPACE = B.FTC_EINVAL, B.FTC_EUNSUPPORTED, B.FTC_EALIGN, B.FTC_EWORKSPACE


def forward(**k):
    a = dict(n=4, ptr=P(20), groups=3, X=P(1), ldx=8, dtype=1, d_in=8, W=P(2), d_out=16, bias=P(3), act=2, R=P(4), ldr=16, slope=P(5), lds=16, Z=P(6), ldz=16, zdt=1,
             ws=P(7), bytes=1 << 40) | k
    return B.lib().ftc_grouped_linear(*a.values(), None)


def backward(**k):
    a = dict(n=4, ptr=P(20), groups=3, X=P(1), ldx=8, dtype=1, d_in=8, W=P(2), d_out=16, slope=P(3), lds=16, dZ=P(4), ldz=16, add=None, lda=0, dX=P(5), lddx=8, dxt=1,
             dW=P(6), db=P(7), dwt=0, ws=P(8), bytes=1 << 40) | k
    return B.lib().ftc_grouped_linear_backward(*a.values(), None)


BOTH = [(dict(n=-1), INVALID), (dict(groups=-1), INVALID), (dict(ptr=None), INVALID), (dict(ptr=P(20) + 2), ALIGN), (dict(d_in=0), INVALID), (dict(d_out=0), INVALID),
        (dict(n=(1 << 30) + 1), UNSUPPORTED), (dict(groups=(1 << 20) + 1), UNSUPPORTED), (dict(d_in=(1 << 20) + 1), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED),
        (dict(ldx=7), INVALID), (dict(X=None), INVALID), (dict(W=None), INVALID), (dict(lds=15), INVALID), (dict(X=P(1) + 1), ALIGN),
        (dict(n=1 << 30, groups=1 << 20, d_in=1 << 20, d_out=1 << 20, ldx=1 << 20, ldr=1 << 20, lds=1 << 20, ldz=1 << 20, lddx=1 << 20), UNSUPPORTED)]
CASES = [(f, {x: v for x, v in k.items() if not (f is forward and x == "lddx") and not (f is backward and x == "ldr")}, code) for f in (forward, backward) for k, code in BOTH] + [
    (forward, dict(act=4), INVALID), (forward, dict(Z=None), INVALID), (forward, dict(ldz=15), INVALID), (forward, dict(ldr=15), INVALID), (forward, dict(zdt=2), UNSUPPORTED),
    (forward, dict(Z=P(1)), INVALID), (forward, dict(Z=P(2)), INVALID), (forward, dict(Z=P(3)), INVALID), (forward, dict(Z=P(5)), INVALID), (forward, dict(slope=P(2)), INVALID),
    (forward, dict(Z=P(4), ldz=17), INVALID), (forward, dict(slope=P(5) + 1), ALIGN),
    (backward, dict(dZ=None), INVALID), (backward, dict(ldz=15), INVALID), (backward, dict(lddx=7), INVALID), (backward, dict(dxt=2), UNSUPPORTED),
    (backward, dict(dwt=2), UNSUPPORTED), (backward, dict(dX=P(1)), INVALID), (backward, dict(dW=P(2)), INVALID), (backward, dict(db=P(6)), INVALID),
    (backward, dict(add=P(6), lda=8), INVALID), (backward, dict(add=P(9), lda=7), INVALID), (backward, dict(add=P(5), lda=9), INVALID),
    (backward, dict(ws=None), WORKSPACE), (backward, dict(bytes=64), WORKSPACE), (backward, dict(ws=P(8) + 16), ALIGN)]


@pytest.mark.parametrize("call,args,code", CASES, ids=lambda x: getattr(x, "__name__", str(x)))
def test_refused(call, args, code):
    assert call(**args) == code, B.lib().ftc_last_error()


def test_nothing_to_do():
    assert forward(n=0, X=None, Z=None) == B.FTC_OK and forward(groups=0, ptr=None) == B.FTC_OK and backward(groups=0, ptr=None) == B.FTC_OK
    assert B.lib().ftc_grouped_linear_workspace_bytes(-1, 1, 8, 8) == 0 and B.lib().ftc_grouped_linear_backward_workspace_bytes(8, 1, 0, 8) == 0


def test_binding_refuses(monkeypatch):
    monkeypatch.setattr(B, "_here", lambda *t: 0)
    X, W, ptr = torch.zeros(4, 8), torch.zeros(3, 8, 16), torch.zeros(4, dtype=torch.int32)
    for k in (dict(W=torch.zeros(3, 7, 16)), dict(W=W.half()), dict(W=torch.zeros(3, 16, 8).transpose(1, 2)), dict(group_ptr=ptr[:3]), dict(group_ptr=ptr.long()),
              dict(bias=torch.zeros(16)), dict(bias=torch.zeros(3, 16).half()), dict(residual=torch.zeros(4, 15)), dict(out=torch.zeros(4, 15)),
              dict(slope=torch.zeros(4, 16, dtype=torch.int16))):
        with pytest.raises(ValueError):
            B.ftc_grouped_linear(**(dict(X=X, W=W, group_ptr=ptr) | k))
    for k in (dict(dW=torch.zeros(3, 8, 15)), dict(db=torch.zeros(16)), dict(dZ=torch.zeros(4, 15)), dict(dX=torch.zeros(4, 9))):
        with pytest.raises(ValueError):
            B.ftc_grouped_linear_backward(**(dict(X=X, W=W, group_ptr=ptr, dZ=torch.zeros(4, 16)) | k))


def test_numbers_of_groups():
    """Tiles: those of a group from s // side + g on are as many as it needs before the next group's, and all of them are below n // side + groups, which is also what all
    groups need together.  Parts of a weight gradient: from 2 (s // side) on for groups of more than `side` rows, below 2 (n // side); and each such group has one first
    multiple of side behind its start."""
    rng = random.Random(5)
    for _ in range(3000):
        side, groups = rng.choice([1, 4, 32, 64, 100]), rng.randrange(1, 30)
        ptr = sorted(rng.randrange(0, rng.choice([3, 50, 1000])) for _ in range(groups + 1))
        n = ptr[-1] + rng.choice([0, 0, 1, 77])
        numbers, parts, joined = [], [], []
        for g, (s, e) in enumerate(zip(ptr, ptr[1:])):
            need = -(-(e - s) // side)
            numbers += range(s // side + g, s // side + g + max(need, 1))
            if e - s > side:
                parts += range(2 * (s // side), 2 * (s // side) + need)
            joined += [g for j in range(n // side) for row in [(j + 1) * side] if row < n and s <= row < e and e - s > side and s != row and row - s <= side]
        assert numbers == sorted(set(numbers)) and numbers[-1] < n // side + groups and len(numbers) <= n // side + groups
        assert parts == sorted(set(parts)) and (not parts or parts[-1] < 2 * (n // side))
        assert joined == [g for g, (s, e) in enumerate(zip(ptr, ptr[1:])) if e - s > side]


PLAN = """#include "grouped_plan.hpp"
#include <stdio.h>
int main(void) { int n, g, N, K, f32, fast; while (scanf("%d %d %d %d %d %d", &n, &g, &N, &K, &f32, &fast) == 6) {
  ftc::DensePlan p = ftc::grouped_plan(n, g, N, K, f32, fast), w = ftc::grouped_dw_plan(n, g, K, N, f32, fast);
  printf("%d %d %d %d %d %d %lld\\n", p.tile, p.splits, p.k_each, w.tile, w.splits, w.k_each, (long long)ftc::grouped_dw_parts(n, w)); } }"""


def test_plan(tmp_path):
    """Every tile and parts of the contraction are taken somewhere, and parts cover the contraction."""
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PLAN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2412_12218_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    rng = random.Random(3)
    asked = [(rng.choice([1, 7, 24, 300, 5000, 60000]), rng.choice([1, 3, 20, 200]), rng.choice([1, 64, 500, 4096]), rng.choice([1, 64, 100, 777, 4096]), rng.randrange(2),
              rng.randrange(2)) for _ in range(400)]
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, a)) for a in asked), text=True, capture_output=True, check=True).stdout
    plans = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert len(plans) == len(asked)
    for (n, g, N, K, f32, fast), (tile, splits, each, w_tile, w_splits, w_each, parts) in zip(asked, plans):
        assert 0 <= tile <= 3 and splits >= 1 and each % 64 == 0 and (splits - 1) * each < K <= splits * each
        assert 0 <= w_tile <= 2 and w_each % 64 == 0 and (w_splits - 1) * w_each < n <= w_splits * w_each
        assert all(t != 2 or (fast and not f32) for t in (tile, w_tile))
        assert parts == (2 * (n // w_each) if w_each < n else 0) and parts * N * K * 4 <= 2.1e9   # a plan of one part has none
    assert {p[0] for p in plans} == {0, 1, 2, 3} and any(p[1] > 1 for p in plans)
    # layers whose last tiles come in parts (test_gpu_grouped_linear.py): tiles of 256, between one and 128 more of them than a multiple of 256
    for n, g, N, K, tiles in ((4401, 5, 4104, 4096, 340), (4401, 5, 4096, 4104, 320), (8003, 2, 4104, 4096, 561), (4800, 16, 4096, 4104, 512)):
        out = subprocess.run([str(exe)], input=f"{n} {g} {N} {K} 0 1", text=True, capture_output=True, check=True).stdout
        assert out.split()[:2] == ["2", "1"] and tiles >= 256
    assert {p[3] for p in plans} == {0, 1, 2} and any(p[4] > 1 for p in plans) and any(p[4] == 1 for p in plans)
