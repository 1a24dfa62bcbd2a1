"""Edges of the model-side entry points that show without a GPU.  Calls that get
as far as a launch run in a child process that sees no device: there they end
in E_HIP, and a crash of the host code ends the child alone."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def child(code):
    """Status name that the call in `code` ends with ("OK" if none), in a process without a device."""
    text = ("import paper_2609_38767_amd as dt\nP = 1 << 20\ntry:\n" +
            "".join(f"    {line}\n" for line in code.splitlines()) +
            "    print('OK')\nexcept dt.DattriError as e:\n    print(e.status_name)\n")
    r = subprocess.run([sys.executable, "-c", text], cwd=ROOT, capture_output=True, text=True,
                       env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])
    return r.stdout.split()[-1]


@pytest.mark.parametrize("vocab", [1, 262143, 262144, (1 << 31) - 1])
def test_embedding_grad_without_tokens(vocab):
    """No tokens and a table of any size: on to the launch that zeroes the table, through no division by zero work."""
    ws = "dt.dattri_embedding_grad_workspace_bytes(0, %d, 4)" % vocab
    call = "dt.dattri_embedding_grad(None, 0, 1, None, 8, 0, 1.0, %d, 4, P, 0, %d, 1 << 44, %s, 0)"
    assert child(call % (vocab, 0, ws)) == "E_HIP"
    assert child(call % (vocab, 1, ws)) == "OK"  # nothing is added: no launch


OVERLAPS = '''
import ctypes, random
import paper_2609_38767_amd as dt

def status(fn, *args):
    try:
        fn(*args)
    except dt.DattriError as e:
        return e.status_name
    return "OK"

def bytes_of(at, rows, width, stride):
    return {at + i * stride + b for i in range(rows) for b in range(width)}

rng = random.Random(5)
seen = {True: 0, False: 0}
for trial in range(4000):  # a table and an output of 2-byte elements anywhere around each other
    d = rng.choice([1, 2, 3, 7])
    same = rng.random() < 0.4
    lt = d + rng.randrange(0, 9)
    lo = lt if same else d + rng.randrange(0, 9)
    vocab, n = rng.randrange(1, 7), rng.randrange(1, 7)
    table = 4096
    out = table + 2 * rng.randrange(-n * lo - 2, vocab * lt + 3)
    tokens = 1 << 20
    want = bool(bytes_of(table, vocab, 2 * d, 2 * lt) & bytes_of(out, n, 2 * d, 2 * lo))
    got = status(dt.dattri_embedding, table, lt, vocab, d, 1, tokens, 4, n, 1.0, out, lo, 0)
    assert got == ("E_INVALID_ARG" if want else "E_HIP"), (trial, d, lt, lo, vocab, n, out - table, want, got)
    seen[want] += 1
assert min(seen.values()) > 500, seen

# the clipping list: sources and outputs of 4-byte elements in any order
seen = {True: 0, False: 0}
for trial in range(4000):
    k = rng.randrange(1, 5)
    sizes = [rng.randrange(0, 4) for _ in range(k)]
    src = [4096 + 4 * rng.randrange(0, 24) for _ in range(k)]
    dst = [s if rng.random() < 0.5 else 4096 + 4 * rng.randrange(0, 40) for s in src]
    read = [bytes_of(p, 1, 4 * n, 1) for p, n in zip(src, sizes)]
    written = [bytes_of(p, 1, 4 * n, 1) for p, n in zip(dst, sizes)]
    want = any(written[i] & written[j] for i in range(k) for j in range(i)) or \\
        any(written[i] & read[j] for i in range(k) for j in range(k) if i != j or src[i] != dst[i])
    arr = lambda t, v: (t * k)(*v)
    types = arr(ctypes.c_int32, [0] * k)
    args = [arr(ctypes.c_void_p, src), arr(ctypes.c_int64, sizes), types]
    tail = [k, 1.0, 1 << 20, 1 << 21, 1 << 16, 0]
    got = status(dt.dattri_clip_gradients, *args, arr(ctypes.c_void_p, dst), types, *tail)
    assert got == ("E_INVALID_ARG" if want else "E_HIP"), (trial, sizes, src, dst, want, got)
    assert status(dt.dattri_clip_gradients, *args, None, None, *tail) == "E_HIP"  # norm alone: sources may overlap
    seen[want] += 1
assert min(seen.values()) > 500, seen
'''


def test_overlap_by_every_byte():
    """What shares a byte is refused and what lies between another buffer's rows is not, by enumeration."""
    child(OVERLAPS)


LINEAR = """n, i, o = 4, 24, 24
A = dict(X=P, W=2 * P, b=3 * P, R=4 * P, Y=5 * P, Z=6 * P, G=7 * P, D=8 * P, Pp=9 * P, dW=10 * P, db=11 * P, w=12 * P)
def call(op, **kw):
    a = dict(A, **kw)
    ws = dt.dattri_linear_workspace_bytes(op, n, i, o, 1, True)
    try:
        if op == 0:
            dt.dattri_linear(a['X'], 0, a['W'], 0, a['b'], 4, a['R'], 0, a['Y'], 0, a['Z'], 0, n, i, o, 1, a['w'], ws, 0)
        elif op == 1:
            dt.dattri_linear_input_grad(a['G'], 0, a['W'], 0, a['R'], 0, 4, a['Z'], 0, a['D'], 0, a['Pp'],
                                        0, n, i, o, 1, a['w'], ws, 0)
        else:
            dt.dattri_linear_weight_grad(a['G'], 0, a['X'], 0, a['dW'], 0, a['db'], 0, n, i, o, 1, a['w'], ws, 0)
    except dt.DattriError as e:
        return e.status_name
for op, free, bad in (
        (0, [{}, dict(Y='R'), dict(R='X'), dict(b=None, Y='b'), dict(Z=None, R='Y'), dict(Y=5 * P + 2, R=4 * P)],
         ['YX', 'YW', 'Yb', 'YZ', 'ZX', 'ZW', 'Zb', 'ZR', ('Y', 'R', 16), ('R', 'Y', 64), ('Y', 'X', 190)]),
        (1, [{}, dict(D='R'), dict(Pp='R'), dict(Pp='Z'), dict(R='Z'), dict(R='Z', Pp='Z')],
         ['DG', 'DW', ('D', 'R', 16), ('D', 'Z', 16), ('Pp', 'G', 0), ('Pp', 'W', 2), ('Pp', 'D', 10), ('Pp', 'Z', 48),
          ('Pp', 'R', 48)]),
        (2, [{}, dict(dW=None, X='db'), dict(G='X')], [('dW', 'G', 4), ('dW', 'X', 0), ('db', 'dW', 8), ('db', 'G', 0),
                                                       ('db', 'X', 64)])):
    for kw in free:
        kw = {k: A[v] if isinstance(v, str) else v for k, v in kw.items()}
        assert call(op, **kw) == 'E_HIP', (op, kw, call(op, **kw))
    for b in bad:
        out, other, off = b if isinstance(b, tuple) else (b[0], b[1], 0)
        assert call(op, **{out: A[other] + off}) == 'E_INVALID_ARG', (op, b)
need = dt.dattri_linear_workspace_bytes(0, 16, 4096, 128, 1, True)
assert need > 0
def ws(at):
    try:
        dt.dattri_linear(P, 0, 2 * P, 0, None, 0, None, 0, 4 * P, 0, None, 0, 16, 4096, 128, 1, at, need, 0)
    except dt.DattriError as e:
        return e.status_name
assert [ws(a) for a in (P, 2 * P, 4 * P, 4 * P - 256, 8 * P)] == ['E_INVALID_ARG'] * 4 + ['E_HIP']
g = dt.dattri_embedding_grad_workspace_bytes(64, 50, 8)
def grad(go=P, tokens=2 * P, out=3 * P, w=4 * P):
    try:
        dt.dattri_embedding_grad(go, 0, 1, tokens, 4, 64, 1.0, 50, 8, out, 0, 0, w, g, 0)
    except dt.DattriError as e:
        return e.status_name
assert grad() == 'E_HIP'
for kw in (dict(out=P + 1020), dict(out=2 * P), dict(w=P), dict(w=3 * P), dict(tokens=4 * P)):
    assert grad(**kw) == 'E_INVALID_ARG', kw
"""


def test_outputs_apart_from_everything_else():
    """Every output of the linear layers against every other buffer; the aliases that the header allows go on."""
    child("\n".join(LINEAR.splitlines()))


def test_stream_of_another_gpu_is_refused():
    """A call runs on the stream it was given or raises: it does not fall back to the current one."""
    from types import SimpleNamespace

    import torch

    from paper_2609_38767_amd import layers
    at = [SimpleNamespace(device=torch.device("cuda", k)) for k in range(2)]
    with pytest.raises(ValueError, match="stream is on cuda:1, the tensors on cuda:0"):
        layers._elsewhere(at[0], at[1])
