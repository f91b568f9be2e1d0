"""Which layers take the tiles behind the last full turn of the compute units in parts, and which weight gradients are joined from parts: that the layers of
test_gpu_grouped_tail.py do, in all ways there are.  CPU only."""
import os
import subprocess

import pytest

from grouped_tail_layers import JOINED, MANY, TAILS, many_lengths

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ASK = """#include "grouped_plan.hpp"
#include <stdio.h>
int main(void) { int n, g, N, K, f32, fast; long long tiles; while (scanf("%d %d %d %d %d %d %lld", &n, &g, &N, &K, &f32, &fast, &tiles) == 7) {
  ftc::DensePlan p = ftc::grouped_plan(n, g, N, K, f32, fast), w = ftc::grouped_dw_plan(n, g, K, N, f32, fast);
  ftc::GroupedTail t = ftc::grouped_tail(tiles, K);
  printf("%d %d %d %d %d %d %d %d %lld\\n", p.tile, p.splits, (int)ftc::grouped_tail_on(n, g, N, K), t.full, t.rest, t.parts, ftc::tail_each(K, t.parts), w.k_each,
         (long long)ftc::grouped_dw_parts(n, w)); } }"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    src, exe = at / "tail.cpp", at / "tail"
    src.write_text(ASK)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2412_12218_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def call(*numbers):
        out = subprocess.run([str(exe)], input=" ".join(map(str, numbers)), text=True, capture_output=True, check=True).stdout
        return dict(zip(("tile", "splits", "on", "full", "rest", "parts", "each", "dw_rows", "dw_parts"), map(int, out.split())))
    return call


def tiles_of(lens, N):
    return sum(-(-x // 256) for x in lens) * -(-N // 256)


def test_layers_with_a_tail(ask):
    """Tiles of 256, some of which, up to 128, are behind a multiple of 256 and come in parts; Z of a layer or its dX, or both."""
    empty, parts = 0, set()
    for lens, d_in, d_out in TAILS:
        took = 0
        for N, K in ((d_out, d_in), (d_in, d_out)):
            p = ask(sum(lens), len(lens), N, K, 0, 1, tiles_of(lens, N))
            if p["tile"] != 2 or not p["on"] or not p["rest"]:
                continue
            took += 1
            assert p["splits"] == 1 and 0 < p["rest"] <= 128 and p["parts"] >= 2 and p["rest"] * p["parts"] <= 256 and p["full"] % 256 == 0 < p["full"]
            assert p["each"] % 64 == 0 and p["each"] * p["parts"] >= K
            empty += (p["parts"] - 1) * p["each"] >= K
            parts.add(p["parts"])
        assert took, (lens, d_in, d_out)
    assert empty == 2 and {3, 4, 5, 8} <= parts


def test_many_groups_with_a_tail(ask):
    """Beyond 512 groups tiles are numbered without being counted: the numbers n / 256 + groups, some of which stand for nothing."""
    for (n, groups, d_in, d_out) in MANY:
        lens = many_lengths(n, groups)
        assert len(lens) == groups > 512 and sum(lens) == n
        p = ask(n, groups, d_out, d_in, 0, 1, (n // 256 + groups) * -(-d_out // 256))
        assert (p["tile"], p["splits"], p["on"]) == (2, 1, 1) and 0 < p["rest"] <= 128 and p["parts"] >= 2
        assert sum(-(-x // 256) for x in lens) < n // 256 + groups


def test_joined_weight_gradients(ask):
    """Groups of several chunks of rows, so that parts are joined, for matrices of numbers that are no multiple of the four a thread has."""
    left = set()
    for lens, d_in, d_out in JOINED:
        for f32 in (0, 1):
            p = ask(sum(lens), len(lens), d_out, d_in, f32, 0, 1)
            assert p["dw_parts"] > 0 and sum(x > p["dw_rows"] for x in lens) >= 2
        left.add(d_in * d_out % 4)
    assert left >= {1, 2, 3}
