"""Which tile a product of the dense layer takes, asked on the host (csrc/dense_plan.hpp, the header the launches include): the layers
of dense_tiles.CASES reach the tiles that they are there for."""
import os
import shutil
import subprocess

import pytest

from dense_tiles import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVER = r"""
#include <cstdio>
#include "dense_plan.hpp"
int main()  // M, N, K, fp32, whole pieces -> side of the tile, parts of the contraction, indices of a part
{
    int m, n, k, f32, whole;
    while (std::scanf("%d %d %d %d %d", &m, &n, &k, &f32, &whole) == 5) {
        const ftc::DensePlan p = ftc::dense_plan(m, n, k, f32, whole);
        std::printf("%d %d %d\n", ftc::dense_side(p.tile), p.splits, p.k_each);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    folder = tmp_path_factory.mktemp("plan")
    (folder / "plan.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "paper_2412_12218_amd", "csrc"), "-o",
                    str(folder / "plan"), str(folder / "plan.cpp")], check=True)

    def ask(products):
        out = subprocess.run([str(folder / "plan")], input="\n".join("%d %d %d %d %d" % p for p in products), capture_output=True, text=True,
                             check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_layers_of_the_larger_tiles(plans):
    seen = set()
    for n, d_in, d_out, f32, whole, *want in CASES:
        products = [(n, d_out, d_in, f32, whole), (n, d_in, d_out, f32, whole), (d_in, d_out, n, f32, whole)]
        got = [p[:2] for p in plans(products)]
        assert got == want, (n, d_in, d_out, f32, whole, got)
        for which, (m, c, k, _, _), (tile, parts) in zip(("Z", "dX", "dW"), products, got):
            if tile > 64:
                seen.add((which, f32, whole, tile))
                # a remainder in each side, and inside the step of 128 bytes
                assert m % tile and c % tile and k % (32 if f32 else 64), (which, m, c, k, tile)
    # 256: 16 bits in whole pieces only
    assert seen == {(w, f, p, t) for w in ("Z", "dX", "dW") for f in (False, True) for p in (False, True) for t in (128, 256) if t == 128 or (p and not f)}


def test_parts_cover_the_contraction(plans):
    """Every index is in one part, none of the parts is empty, and a part begins at a multiple of a step."""
    products = [(m, n, k, f32, whole) for m in (1, 64, 513, 20000) for n in (1, 70, 4096) for k in (1, 63, 64, 65, 1000, 20001, 1 << 20)
                for f32 in (0, 1) for whole in (0, 1)]
    for (_, _, k, _, _), (_, parts, each) in zip(products, plans(products)):
        assert each % 64 == 0 and (parts - 1) * each < k <= parts * each
