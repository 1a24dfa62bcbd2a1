"""The cuts of the experts' products at the ends of what the entry points take.
Compiles the host rules by themselves (no GPU)."""
import os
import shutil
import subprocess

import pytest

from expert_cuts import BIG, FEW, PADDED

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r"""
#include <cstdio>
#include "expert_shape.h"
int main() {
  char kind;
  long a[6];
  while (scanf(" %c", &kind) == 1) {
    for (int i = 0; i < (kind == 't' ? 3 : 6); ++i)
      if (scanf("%ld", a + i) != 1) return 1;
    if (kind == 't') {  // which, rows, rows of a tile
      printf("%d\n", dattri::tile_rows((dattri::Rows)a[0], (int)a[1], (int)a[2]));
    } else {  // op, elt, rows, experts, d_in, d_out
      const long op = a[0], m = op == 2 ? a[5] : a[2], n = op == 0 ? a[5] : a[4], k = op == 0 ? a[4] : op == 1 ? a[5] : a[2];
      const dattri::ExpertShape g = dattri::expert_shape(op == 2, a[2], a[3], m, n, k, (int)a[1], op == 0);
      printf("%d %d %d\n", (int)g.v, g.splits, g.kw);
    }
  }
}
"""


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


def test_tile_rows_of_any_segment(ask):
    """All tile rows, those filled to more than half, the one filled to half at most: up to the most rows that a call takes."""
    sizes = [n + k for n in (0, 32, 64, 128, 256, 1000, 1 << 20, (1 << 31) - 256, (1 << 31) - 128, (1 << 31) - 32)
             for k in range(-129, 258) if 0 <= n + k < 1 << 31]
    for tm in (32, 64, 128, 256):
        got = ask([f"t {which} {n} {tm}" for n in sizes for which in range(3)])
        for n, (full, rest) in zip(sizes, (divmod(n, tm) for n in sizes)):
            k = 3 * sizes.index(n)
            more = rest > tm // 2
            assert [v for v, in got[k:k + 3]] == [full + (rest > 0), full + more, int(rest > 0 and not more)], (n, tm)


def cut(ask, cases):
    return ask([f"e {op} {4 if t == 'f32' else 2} {n} {e} {i} {o}" for op, t, n, e, i, o, *_ in cases])


def test_few_rows_split_in_two(ask):
    assert [(v, splits) for v, splits, _ in cut(ask, FEW)] == [(3, c[6]) for c in FEW]
    assert {(c[0], c[1], c[6]) for c in FEW} == {(op, t, s) for op in (0, 1) for t in ("f32", "bf16") for s in (1, 2)}


def test_largest_tiles_of_many_experts(ask):
    assert [v for v, _, _ in cut(ask, BIG)] == [0] * len(BIG)
    assert all(c[3] + 2 > 64 for c in BIG)  # segments: more than a wave has lanes


def test_padded_weight_gradients(ask):
    got = ask([f"e 2 {4 if t == 'f32' else 2} {n} {e} {i} {o}" for t, n, e, i, o, _, _ in PADDED])
    assert [(["256x256", "128x128", "64x128"][v], splits > 1) for v, splits, _ in got] == [c[5:] for c in PADDED]
