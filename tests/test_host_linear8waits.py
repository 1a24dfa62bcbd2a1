"""The 8-bit tile kernels' hand-written waits hold in the code the compiler
emits (host-only: reads the gfx950 assembly of this build).

A stage of the ring has landed once no more than the loads of the stages behind
it are outstanding, which is right only while every vector-memory operation of
the loop is one of the ring's loads and each stage issues the same number."""
import re

import pytest

from test_host_linearwaits import _loop
from test_host_waitcounts import _asm

# bytes per result, WM, WN, BM, BN, buffers; direct loads per wave and stage: the rows' and one of scales
SHAPES = {(2, 2, 4, 4, 2, 2): 9, (2, 2, 4, 2, 1, 4): 5, (2, 2, 2, 1, 2, 4): 7, (4, 2, 2, 2, 2, 2): 9,
          (4, 2, 2, 1, 2, 4): 7}


@pytest.fixture(scope="module")
def asm():
    return _asm("linear8.hip")


@pytest.mark.parametrize("op", [0, 3])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "".join(map(str, s)))
def test_ring_waits(asm, op, shape):
    name = f"_ZN6dattri14linear8_kernelILi{op}E" + "".join(f"Li{v}E" for v in shape)
    start = next(i for i, l in enumerate(asm) if l.startswith(name) and ":" in l)
    end = next(i for i in range(start, len(asm)) if asm[i].startswith(".Lfunc_end"))
    body = [t for t in (l.split(";")[0].strip() for l in asm[start:end]) if t]
    assert not any(t.startswith("scratch_") for t in body)
    loop, loads, buffers = _loop(body), SHAPES[shape], shape[-1]
    memory = [t for t in loop if t.startswith(("buffer_", "global_", "flat_"))]
    assert len(memory) == buffers * loads and all(t.startswith("buffer_load_dword") and t.endswith(" lds") for t in memory)
    assert sum(t.startswith("buffer_load_dword ") for t in memory) == buffers  # the scales
    at = [i for i, t in enumerate(loop) if re.match(r"s_waitcnt vmcnt", t)]
    waits = [int(re.match(r"s_waitcnt vmcnt\((\d+)\)", loop[i])[1]) for i in at]
    assert waits == [(buffers - 2) * loads] * buffers
    for i, j in zip(at, at[1:]):
        assert sum(t.endswith(" lds") for t in loop[i:j]) == loads
        # the barrier stands between the wait and the loads into the buffer that it frees
        after = [t for t in loop[i:j] if t == "s_barrier" or t.endswith(" lds")]
        assert after[0] == "s_barrier" and after.count("s_barrier") == 1
    assert loop.count("s_barrier") == buffers
