"""Which kernels and tiles the 8-bit layers take for given sizes: the rules
themselves, compiled for the host, at the sizes of the GPU tests that mean to
reach each of them."""
import os
import shutil
import subprocess

import pytest

from tests import test_gpu_i8_rules, test_gpu_i8_tiles

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2107_02103_amd", "csrc", "dpc_i8_tiles.h")
PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "%s"
int main() {
  char what[16];
  int a, b, c, d, e;
  while (std::scanf("%%15s %%d %%d %%d %%d %%d", what, &a, &b, &c, &d, &e) == 6) {
    if (!std::strcmp(what, "tile")) {
      const I8Tile t = kI8Tiles[i8_tile(a, b, c, d, e != 0)];
      std::printf("%%d %%d\n", t.bm, t.bn);
    } else if (!std::strcmp(what, "few")) {
      std::printf("%%d 0\n", (int)i8_few_rows(a, b, d, e != 0));
    } else if (!std::strcmp(what, "one")) {
      std::printf("%%d 0\n", (int)i8_one_kernel(a, b, c, d));
    } else {
      std::printf("%%d 0\n", (int)i8_most_tiles(a, b, e != 0, c));
    }
  }
}
"""


def _ld(k):
    return (k + 127) // 128 * 128


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


def test_the_routed_tests_reach_their_tiles(rules):
    E = test_gpu_i8_tiles.EXPERTS
    for tile, (ntok, n, k) in test_gpu_i8_tiles.SIZES.items():
        got, few = rules(("tile", 2 * ntok, n, _ld(k), E, 1), ("few", 2 * ntok, n, 0, E, 1))
        assert got == tile and few[0] == 0
    assert len(test_gpu_i8_tiles.SIZES) == 4


def test_the_tests_of_kernels_that_change_stand_on_both_sides(rules):
    for t, k, few, many in test_gpu_i8_rules.ONE_KERNEL:
        chunk = {"f64": 2, "f32": 4, "f16": 8, "bf16": 8}[t]
        a, b = rules(("one", few, k, _ld(k), chunk, 0), ("one", many, k, _ld(k), chunk, 0))
        assert a != b, (t, k)
    for E, n, k, (few, more) in test_gpu_i8_rules.FEW_ROWS:
        assert rules(("few", few, n, 0, E, 1), ("few", more, n, 0, E, 1)) == [(1, 0), (0, 0)], (E, n)


def test_tiles_of_groups_are_enough(rules):
    # rows dealt to the groups in the worst way: as many groups as there are rows end inside a tile
    asked, want = [], []
    for size in (16, 32, 64, 128, 256):
        for m in (1, 5, size, size + 1, 3 * size - 1, 1000, 1 << 27):
            for G in (1, 2, 7, 1024):
                ends = min(G, m - 1)                # groups with one row each, the rest in the empty rows
                asked.append(("most", m, G, size, 0, 1))
                want.append(ends + -(-(m - ends) // size))
    for q, (got, _), w in zip(asked, rules(*asked), want):
        assert w <= got <= q[1], q
    assert rules(("most", 257, 1, 256, 0, 0), ("most", 256, 1, 256, 0, 0)) == [(2, 0), (1, 0)]


def test_launches_stay_below_2_to_the_32_threads(rules):
    # the largest products that 288 GB hold, in 16 bits: tiles of 256 x 256 if no other fits a launch
    for m, n in ((1 << 27, 1000), (1 << 20, 1 << 17), (1 << 17, 1 << 20), (1 << 13, 1 << 24)):
        (bm, bn), = rules(("tile", m, n, 128, 1, 0))
        threads = {(256, 256): 512}.get((bm, bn), 256)
        assert ((m + bm - 1) // bm * ((n + bn - 1) // bn) + 7) // 8 * 8 * threads < 1 << 32
