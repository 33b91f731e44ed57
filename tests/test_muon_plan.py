"""Host check of the plan of the Newton-Schulz products: the library's own plan,
through a small program linked with it (no kernel is launched)."""
import os
import subprocess
import tempfile

import pytest

from paper_1808_04728_amd import binding as B
from paper_1808_04728_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")

# reads "rows cols dtype momentum" lines, writes the plan of each matrix
SRC = r"""
#include "cf_kernels.h"
#include <cstdio>
int main() {
  int r, c, dt, mom;
  while (scanf("%d %d %d %d", &r, &c, &dt, &mom) == 4) {
    const long long off = 0;
    cf::NsTable T{};
    cf::ns_plan(1, &off, &r, &c, dt, mom != 0, &T);
    const cf::NsMat &M = T.mat[0];
    if (M.mt) printf("0 0 0 0 0 0 0\n");
    else printf("%d %d %d %d %d %d %d\n", 1, M.mp, M.np, M.tile_sq, M.tile_long, M.tile_gram, M.slices);
  }
}
"""


@pytest.fixture(scope="module")
def plan():
    """plan([(rows, cols), ...]) -> [(mp, np, tile_sq, tile_long, tile_gram, slices)], None
    for a matrix of the skinny kernels."""
    with tempfile.TemporaryDirectory() as td:
        src, exe = os.path.join(td, "t.cpp"), os.path.join(td, "t")
        with open(src, "w") as f:
            f.write(SRC)
        at, lib = os.path.split(B.LIB_PATH)
        subprocess.run([build.HIPCC, "-std=c++17", "--offload-host-only", "-I", build.CSRC, src, "-L" + at, "-l:" + lib,
                        "-Wl,-rpath," + at, "-o", exe], check=True, capture_output=True)

        def call(shapes, dt=0, momentum=False):
            text = "".join(f"{r} {c} {dt} {int(momentum)}\n" for r, c in shapes)
            out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
            rows = [tuple(map(int, line.split())) for line in out.splitlines()]
            assert len(rows) == len(shapes)
            return [r[1:] if r[0] else None for r in rows]

        yield call


def test_offsets_in_a_tile_fit_32_bits(plan):
    """The kernels keep a row's byte offset from its tile's first row in 32 bits: 4 bytes a
    column of the padded array, 112 bytes more in a row's piece."""
    ms = [129, 160, 192, 193, 224, 256, 257, 384, 512, 513, 640, 700, 768, 1024, 1025, 1536, 2048, 4096, 16384]
    ns = [16384, 1 << 20, 4210000, 4210784, 4300000, 5592405, 8388608, 8454688, 8500000, 8600000, 12000000, (1 << 24) - 1, 1 << 24]
    shapes = [(m, n) for m in ms for n in ns] + [(n, m) for m in ms for n in ns]
    for (r, c), (mp, np_, sq, lng, gram, slices) in zip(shapes, plan(shapes)):
        assert (min(gram, mp) - 1) * 4 * np_ + 112 < 1 << 32, (r, c, gram)
        assert (max(sq, lng) - 1) * 4 * mp + 112 < 1 << 32


def test_every_tile_is_run(plan):
    """The sizes of test_gpu_muon_tiles.py take each tile in each product, the Gram product's
    whole and in slices, the long side's for tall and for wide matrices."""
    import test_gpu_muon_tiles as tiles

    shapes = tiles.SHAPES
    plans = plan(shapes)
    assert plans == plan(shapes, dt=1) == plan(shapes, momentum=True)
    sides = {32, 64, 128, 192, 256}
    assert {p[2] for p in plans} == sides
    assert {p[3] for (r, c), p in zip(shapes, plans) if r < c} == sides
    assert {p[3] for (r, c), p in zip(shapes, plans) if r > c} == sides
    assert {p[4] for p in plans if p[5] == 1} == sides
    assert {p[4] for p in plans if p[5] > 1} == sides
