"""The linear tile kernels' hand-written waits hold in the code the compiler
emits (host-only: reads the gfx950 assembly of this build).

The ring of stage buffers is waited for by counting (all but the loads of two
stages), which is right only while no other vector-memory operation stands in
the loop and nothing drains the ring; the transposing LDS reads are inline
assembly, whose results may not be touched before the wait that follows them;
and accumulators and fragments have to stay in registers."""
import re

import pytest

from test_host_waitcounts import _asm

# (op, A contiguous, B contiguous, bytes per element, bytes of k per stage, WM, WN, BM, BN); loads per wave
# and 64 bytes of k by the last four
SHAPES = {(2, 2, 4, 4): 8, (2, 2, 2, 2): 4, (2, 2, 1, 2): 3, (1, 4, 1, 1): 3}
OPS = {0: (1, 1), 1: (1, 0), 2: (0, 0)}
KERNELS = [(op, a, b, e, 128 if a and b and e == 2 and shape[2] == 4 else 64) + shape
           for real, (a, b) in OPS.items() for op in (real, 3) for e in (2, 4)
           for shape in SHAPES if not (real == 2 and shape[2] == 1)]


@pytest.fixture(scope="module")
def asm():
    return _asm("linear.hip")


def _kernel(lines, key):
    op, a, b, e, kw, *shape = key
    name = f"_ZN6dattri11gemm_kernelILi{op}ELb{a}ELb{b}ELi{e}ELi{kw}E" + "".join(f"Li{v}E" for v in shape)
    start = next(i for i, l in enumerate(lines) if l.startswith(name) and ":" in l)
    end = next(i for i in range(start, len(lines)) if lines[i].startswith(".Lfunc_end"))
    body = [l.split(";")[0].strip() for l in lines[start:end]]
    return [l for l in body if l]


def _loop(body):
    """The main loop: from the label its last branch goes back to, where MFMA and barriers are."""
    labels = {l[:-1]: i for i, l in enumerate(body) if l.endswith(":")}
    for i, l in enumerate(body):
        m = re.match(r"s_cbranch_\w+ (\.LBB\w+)", l)
        if m and labels.get(m.group(1), i) < i:
            text = body[labels[m.group(1)]:i]
            if any(t.startswith("v_mfma") for t in text) and "s_barrier" in text:
                return text
    raise AssertionError("no main loop")


def _registers(text):
    out = set()
    for m in re.finditer(r"\bv(?:\[(\d+):(\d+)\]|(\d+))", text):
        out |= set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}
    return out


@pytest.mark.parametrize("key", KERNELS, ids=lambda k: "".join(map(str, k)))
def test_ring_waits(asm, key):
    body = _kernel(asm, key)
    assert not any(t.startswith("scratch_") for t in body)
    buffers = 256 // key[4]
    loop, loads = _loop(body), SHAPES[key[5:]] * key[4] // 64
    memory = [t for t in loop if t.startswith(("buffer_", "global_", "flat_"))]
    assert len(memory) == buffers * loads and all(t.startswith("buffer_load_dwordx4") and t.endswith(" lds") for t in memory)
    waits = [int(m[1]) for t in loop for m in [re.match(r"s_waitcnt vmcnt\((\d+)\)", t)] if m]
    left = (buffers - 2) * loads  # that may be under way at a barrier
    assert waits == [left] * buffers, waits
    # between two waits one stage's loads, so exactly the awaited stage's are the older ones
    at = [i for i, t in enumerate(loop) if re.match(r"s_waitcnt vmcnt", t)]
    for i, j in zip(at, at[1:]):
        assert sum(t.endswith(" lds") for t in loop[i:j]) == loads
    assert loop.count("s_barrier") == buffers


@pytest.mark.parametrize("key", [k for k in KERNELS if k[3] == 2 and not k[2]], ids=lambda k: "".join(map(str, k)))
def test_transposed_reads_are_waited_for(asm, key):
    body = _kernel(asm, key)
    pending, seen = set(), 0
    for t in body:
        if t.startswith("ds_read_b64_tr_b16"):
            dst, rest = t.split(",", 1)
            assert not _registers(rest) & pending, t
            assert not _registers(dst) & pending, t
            pending |= _registers(dst)
            seen += 1
        elif re.match(r"s_waitcnt .*lgkmcnt\(0\)", t):
            pending.clear()
        elif re.match(r"s_c?branch|s_endpgm", t):
            assert not pending, t  # nothing under way where the text's order ends
        else:
            assert not _registers(t) & pending, t
    assert seen
