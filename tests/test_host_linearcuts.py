"""The sizes that the GPU tests give the tile kernels take every way a product is
cut: each tile, whole and with k split, for every operation and type.  Compiles
the host rule by itself (no GPU), so a change of its model that leaves a way
without a test fails here."""
import os
import shutil
import subprocess

import pytest

from linear_cuts import CUTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILES = ["256x256", "128x128", "64x128", "32x128"]
MAIN = r"""
#include <cstdio>
#include "linear_shape.h"
int main() {
  long op, elt, rows, i, o;
  while (scanf("%ld %ld %ld %ld %ld", &op, &elt, &rows, &i, &o) == 5) {
    const dattri::GemmShape g = dattri::gemm_shape(op == 2 ? o : rows, op == 0 ? o : i, op == 0 ? i : op == 1 ? o : rows,
                                                   (int)elt, op != 2, op == 0);
    printf("%d %d %d %d\n", (int)g.v, g.splits, g.sps, g.kw);
  }
}
"""


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("cuts")
    src = d / "main.cpp"
    src.write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2609_38767_amd", "csrc"), str(src), "-o",
                    str(d / "cut")], check=True)
    text = "".join(f"{op} {4 if t == 'f32' else 2} {n} {i} {o}\n" for op, t, n, i, o, _, _ in CUTS)
    out = subprocess.run([str(d / "cut")], input=text, capture_output=True, text=True, check=True).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_sizes_take_the_cut_they_stand_for(cuts):
    assert len(cuts) == len(CUTS)
    for (op, t, n, i, o, tile, split), (v, splits, sps, kw) in zip(CUTS, cuts):
        assert (TILES[v], splits > 1) == (tile, split), (op, t, n, i, o, TILES[v], splits)
        assert not (op == 0 and n <= 4 and o >= 2048)  # the few-row form's


def test_every_cut_has_a_size():
    ways = {(op, t, tile, split) for op in range(3) for t in ("f32", "bf16") for tile in TILES for split in (False, True)
            if not (op == 2 and tile in ("64x128", "32x128"))}
    assert {c[:2] + c[5:] for c in CUTS} == ways


def test_last_splits_are_short(cuts):
    """Of every way with splits one size at least whose last split has fewer stages than the others."""
    short, split = set(), set()
    for (op, t, n, i, o, tile, _), (_, splits, sps, kw) in zip(CUTS, cuts):
        if splits > 1:
            k = i if op == 0 else o if op == 1 else n
            stages = -(-k * (4 if t == "f32" else 2) // kw)
            split.add((op, t, tile))
            if stages < splits * sps:
                short.add((op, t, tile))
    assert short == split, split - short
