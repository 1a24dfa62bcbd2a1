"""The sizes that the GPU tests give the 8-bit products and the experts' products
take every way they are cut.  Compiles the host rules by themselves (no GPU), so
a change of their models that leaves a way without a test fails here."""
import os
import shutil
import subprocess

import pytest

from block_cuts import CUTS8, CUTSX

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r"""
#include <cstdio>
#include "expert_shape.h"
#include "linear8_shape.h"
int main() {
  char kind;
  long a[6];
  while (scanf(" %c", &kind) == 1) {
    for (int i = 0; i < (kind == 'p' ? 4 : 6); ++i)
      if (scanf("%ld", a + i) != 1) return 1;
    if (kind == 'p') {  // elt, rows, d_in, d_out
      const dattri::Shape8 g = dattri::shape8(a[1], a[3], a[2], (int)a[0]);
      printf("%d %d %d\n", (int)g.v, g.splits, g.sps);
    } else {  // op, elt, rows, experts, d_in, d_out
      const long op = a[0], m = op == 2 ? a[5] : a[2], n = op == 0 ? a[5] : a[4], k = op == 0 ? a[4] : op == 1 ? a[5] : a[2];
      const dattri::ExpertShape g = dattri::expert_shape(op == 2, a[2], a[3], m, n, k, (int)a[1], op == 0);
      printf("%d %d %d\n", (int)g.v, g.splits, g.kw);
    }
  }
}
"""
TILES = ["256x256", "128x128", "64x128", "32x128"]


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("cuts")
    src = d / "main.cpp"
    src.write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2609_38767_amd", "csrc"), str(src), "-o",
                    str(d / "cut")], check=True)

    def run(lines):
        out = subprocess.run([str(d / "cut")], input="\n".join(lines), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def elt(t):
    return 4 if t == "f32" else 2


def test_8bit_sizes_take_the_cut_they_stand_for(ask):
    got = ask([f"p {elt(t)} {n} {i} {o}" for t, n, i, o, _, _ in CUTS8])
    assert len(got) == len(CUTS8)
    for (t, n, i, o, tile, split), (v, splits, sps) in zip(CUTS8, got):
        assert ((TILES[:3] + ["few"])[v], splits > 1) == (tile, split), (t, n, i, o, v, splits)
        if split:
            assert -(-i // 128) < splits * sps  # the last split is short
    ways = {(t, tile, split) for t in ("f32", "bf16") for tile in ("256x256", "128x128", "64x128") for split in (False, True)
            if not (t == "f32" and tile == "256x256")} | {("f32", "few", False), ("bf16", "few", False)}
    assert {(c[0], c[4], c[5]) for c in CUTS8} == ways
    assert {(c[0], c[4], c[5], c[2] % 16 == 0) for c in CUTS8} == {w + (a,) for w in ways for a in (False, True)}


def test_no_other_cut_is_reached(ask):
    """float32 results never take 256 x 256 and the form without tiles never splits, whatever the size."""
    sizes = [(n, i, o) for n in (1, 16, 17, 64, 65, 300, 5000, 100000) for i in (1, 129, 5000, 65536) for o in (1, 300, 20000)]
    for n, i, o in sizes:
        (v4, s4, _), (v2, s2, _) = ask([f"p {e} {n} {i} {o}" for e in (4, 2)])
        few = n < 8 or (n <= 16 and i * o < 40000000)
        assert v4 != 0 and (v4 == 3) == (v2 == 3) == few and (not few or s4 == s2 == 1)


def test_expert_sizes_take_the_cut_they_stand_for(ask):
    got = ask([f"e {op} {elt(t)} {n} {e} {i} {o}" for op, t, n, e, i, o, _, _ in CUTSX])
    assert [(TILES[v], splits > 1) for v, splits, _ in got] == [c[6:] for c in CUTSX]
    ways = {(op, t, tile, s) for op in (0, 1) for t in ("f32", "bf16") for tile in TILES for s in (False, True)
            if not (s and (tile == "256x256" or (tile == "64x128" and t == "f32")))}
    ways |= {(2, t, "128x128", s) for t in ("f32", "bf16") for s in (False, True)} | {(2, "bf16", "256x256", False), (2, "f32", "64x128", False)}
    assert {(c[0], c[1], c[6], c[7]) for c in CUTSX} == ways


def test_no_other_expert_cut_is_reached(ask):
    """256 x 256 is never split, nor float32 in 64 x 128; weight gradients take their own, whatever the size."""
    sizes = [(n, e, i, o) for n in (1, 50, 3000, 100000) for e in (1, 9, 300) for i in (8, 700, 16384) for o in (40, 5000)]
    for op in range(3):
        for b in (2, 4):
            for (n, e, i, o), (v, splits, _) in zip(sizes, ask([f"e {op} {b} {n} {e} {i} {o}" for n, e, i, o in sizes])):
                assert 1 <= splits <= 32 and (splits == 1 or v == 1 or v == 3 or (v == 2 and b == 2))
                assert op < 2 or v == 1 or v == (0 if b == 2 else 2)
