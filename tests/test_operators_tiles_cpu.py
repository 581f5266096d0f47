"""Which tile each size of the operators' matrix products takes, so that the sizes the GPU
tests run still reach every tile there is."""

import os
import shutil
import subprocess

import pytest

from .operator_sizes import LINEAR, MUON, ORTH, UNITS

OPS = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1902_06714_amd", "csrc_ops")
TILES = ["32 by 4", "64 by 2", "64", "128", "192", "256", "128 x 192"]       # as MmShape has them

PROGRAM = r"""
#include <cstdio>
#include "mm_shape.h"
using namespace nf;
static_assert(MM_32_GROUPS == 0 && MM_64_GROUPS == 1 && MM_64 == 2 && MM_128 == 3 && MM_192 == 4 && MM_256 == 5 &&
              MM_128_192 == 6, "the names' order");
int main() {
  long long kind, a, b, c, units;
  while (std::scanf("%lld %lld %lld %lld %lld", &kind, &a, &b, &c, &units) == 5) {
    if (kind == 2) {
      std::printf("%d\n", (int)linear_shape(a, c, (b + 15) / 16 * 16, units));
    } else {
      const long long m = b < c ? b : c, n = b < c ? c : b;
      for (int p = PROD_GRAM; p <= PROD_LAST; ++p) std::printf("%d ", (int)orth_shape((OrthProduct)p, kind == 1, a, m, n, units));
      std::printf("\n");
    }
  }
}
"""


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs a host C++ compiler")
    d = tmp_path_factory.mktemp("tiles")
    (d / "tiles.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", OPS, str(d / "tiles.cpp"), "-o", str(d / "tiles")], check=True)

    def ask(kind, sizes):
        text = "\n".join(" ".join(map(str, (kind, *s, UNITS))) for s in sizes)
        out = subprocess.run([str(d / "tiles")], input=text, capture_output=True, text=True, check=True).stdout
        return [[TILES[int(v)] for v in line.split()] for line in out.splitlines()]
    return ask


@pytest.mark.parametrize("parts", [0, 1])
def test_orthogonalisation(tiles, parts):
    for turned in (False, True):
        sizes = [(c, n, m) if turned else (c, m, n) for c, m, n in ORTH]
        for size, want, got in zip(sizes, ORTH.values(), tiles(parts, sizes)):
            assert tuple(got) == (*want, want[2]), (size, got)
    for k in range(3):
        assert {w[k] for w in ORTH.values()} == set(TILES[:6])
    assert {ORTH[s][2] for s in MUON} == set(TILES[:6])


def test_linear_layers(tiles):
    for size, want, got in zip(LINEAR, LINEAR.values(), tiles(2, LINEAR)):
        assert got == [want], (size, got)
    assert set(LINEAR.values()) == set(TILES)


def test_the_widest_workloads_tiles(tiles):
    """4096 x 4096 steps and layers take tiles that the sizes above have."""
    assert tiles(1, [(1, 4096, 4096)]) == [["192", "192", "256", "256"]]
    assert tiles(2, [(8192, 4096, 4096), (10000, 784, 1024)]) == [["256"], ["128 x 192"]]
