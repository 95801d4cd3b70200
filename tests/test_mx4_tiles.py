"""Which kernels and tiles the product of 4-bit codes takes for given sizes: the
rules themselves, compiled for the host, at the sizes of the GPU tests that mean to
reach each of them."""
import os
import shutil
import subprocess

import pytest

from tests import test_gpu_mx4_tiles as sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2107_02103_amd", "csrc", "dpc_mx4_tiles.h")
PROGRAM = r"""
#include <cstdio>
#include "%s"
int main() {
  int m, n, k, e;
  while (std::scanf("%%d %%d %%d %%d", &m, &n, &k, &e) == 4) {
    const Mx4Tile t = kMx4Tiles[mx4_tile(m, n, (k + 255) / 256, e, e > 1)];
    std::printf("%%d %%d %%d %%lld %%lld\n", t.bm, t.bn, (int)mx4_few_rows(m, n, e, e > 1),
                (long long)mx4_most_tiles(m, e, e > 1, t.bm), (long long)mx4_likely_tiles(m, e, e > 1, t.bm));
  }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs a host compiler")
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(PROGRAM % HEADER)
    subprocess.check_call(["g++", "-std=c++17", str(d / "rules.cpp"), "-o", str(d / "rules")])

    def ask(*questions):
        text = "".join(" ".join(map(str, q)) + "\n" for q in questions)
        out = subprocess.run([str(d / "rules")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return ask


def test_the_tests_reach_their_tiles(rules):
    for tile, (m, n, k) in sizes.DENSE.items():
        assert rules((m, n, k, 1))[0][:3] == tile + (0,), (tile, m)
    for tile, (m, n, k) in sizes.ROUTED.items():
        assert rules((m, n, k, sizes.EXPERTS))[0][:3] == tile + (0,), (tile, m)


def test_the_tests_stand_around_few_rows(rules):
    for few, tiled in sizes.FEW:
        assert rules(few, tiled)[0][2] == 1 and rules(few, tiled)[1][2] == 0, (few, tiled)


def test_tiles_never_fall_short(rules):
    """Whatever the rows of each group, the launch has as many tiles as there are."""
    for m, groups, size in ((1, 1, 64), (100, 3, 64), (1000, 64, 128), (63, 7, 64), (5000, 2, 256)):
        r = rules((m, 4096, 4096, groups))[0]
        worst = sum(-(-c // r[0]) for c in [1] * min(groups, m - 1) + [m - min(groups, m - 1)])
        assert r[3] >= worst or r[3] == m
    assert rules((2 ** 27, 2 ** 24, 256, 1))[0][:2] == (256, 256)
