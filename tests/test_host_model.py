"""Refusals and sizes of the model-side entry points (no GPU): every bad call
returns the documented status before any GPU work."""
import ctypes

import pytest

import paper_2609_38767_amd as dt

P = 1 << 20  # an aligned address that no call here reaches


def status(fn, *args):
    with pytest.raises(dt.DattriError) as e:
        fn(*args)
    return e.value.status_name


def test_embedding_errors():
    def call(table=P, ld=0, vocab=10, d=8, dtype=0, tokens=P, tb=8, n=4, out=P, ldo=0):
        return status(dt.dattri_embedding, table, ld, vocab, d, dtype, tokens, tb, n, 1.0, out, ldo, 0)
    for kw in (dict(table=None), dict(out=None), dict(tokens=None), dict(tb=2), dict(n=-1), dict(vocab=-1), dict(d=0),
               dict(ld=7), dict(ldo=-1), dict(table=P + 2), dict(tokens=P + 4)):
        assert call(**kw) == "E_INVALID_ARG", kw
    assert call(dtype=5) == "E_DTYPE"
    for kw in (dict(n=1 << 31), dict(vocab=1 << 31), dict(d=(1 << 24) + 1), dict(ld=1 << 23), dict(ld=1 << 62)):
        assert call(**kw) == "E_UNSUPPORTED", kw
    dt.dattri_embedding(None, 0, 0, 8, 0, None, 8, 0, 1.0, None, 0, 0)  # no tokens: nothing to do


def test_embedding_grad_errors():
    ws = dt.dattri_embedding_grad_workspace_bytes(100, 50, 8)

    def call(g=P, ld=0, dtype=1, tokens=P, tb=4, n=100, vocab=50, d=8, out=P, ldo=0, w=P, wb=ws):
        return status(dt.dattri_embedding_grad, g, ld, dtype, tokens, tb, n, 1.0, vocab, d, out, ldo, 0, w, wb, 0)
    for kw in (dict(g=None), dict(out=None), dict(tokens=None), dict(tb=0), dict(n=-1), dict(d=0), dict(ld=3),
               dict(out=P + 2), dict(ldo=-4)):
        assert call(**kw) == "E_INVALID_ARG", kw
    assert call(dtype=-1) == "E_DTYPE"
    for kw in (dict(w=None), dict(wb=ws - 1), dict(w=P + 16)):
        assert call(**kw) == "E_WORKSPACE", kw
    assert status(dt.dattri_embedding_grad_workspace_bytes, -1, 5, 8) == "E_INVALID_ARG"
    assert dt.load().dattri_embedding_grad_workspace_bytes(1, 1, 1, None) == -1


def test_embedding_grad_workspace_covers_its_parts():
    for n in (0, 1, 31, 32, 4096, 4097, 1 << 20, (1 << 31) - 1):
        for d in (1, 769, 4096):
            need = dt.dattri_embedding_grad_workspace_bytes(n, 128000, d)
            # two (key, position) buffers and a float32 row for every 32 positions
            assert need >= 16 * n + n // 32 * d * 4


def linear_ws(op, n, i, o, dtype, aligned):
    return dt.dattri_linear_workspace_bytes(op, n, i, o, dtype, aligned)


def test_linear_errors():
    n, i, o = 4, 24, 40
    ws = max(linear_ws(op, n, i, o, 0, False) for op in range(3)) + 256

    def fwd(X=P, lx=0, W=P, lw=0, b=None, act=0, R=None, lr=0, Y=P, ly=0, Z=None, lz=0, n=n, i=i, o=o, dtype=0, w=P,
            wb=ws):
        return status(dt.dattri_linear, X, lx, W, lw, b, act, R, lr, Y, ly, Z, lz, n, i, o, dtype, w, wb, 0)
    for kw in (dict(X=None), dict(W=None), dict(Y=None), dict(lx=23), dict(lw=1), dict(ly=39), dict(lr=-1), dict(lz=2),
               dict(n=-1), dict(i=0), dict(o=0), dict(act=5), dict(act=-1), dict(X=P + 2), dict(b=P + 1),
               dict(R=P, lr=48, ly=56)):
        assert fwd(**kw) == "E_INVALID_ARG", kw
    assert fwd(dtype=2) == "E_DTYPE"
    for kw in (dict(n=1 << 31), dict(i=1 << 25), dict(o=1 << 25), dict(lx=1 << 22)):
        assert fwd(**kw) == "E_UNSUPPORTED", kw

    def inp(G=P, lg=0, W=P, R=None, lr=0, act=0, Z=None, lz=0, D=None, ld=0, Pp=P, lp=0, dtype=1, w=P, wb=ws):
        return status(dt.dattri_linear_input_grad, G, lg, W, 0, R, lr, act, Z, lz, D, ld, Pp, lp, n, i, o, dtype, w,
                      wb, 0)
    for kw in (dict(G=None), dict(W=None), dict(Pp=None), dict(act=1), dict(act=9, Z=P), dict(lg=39), dict(lp=3),
               dict(D=P), dict(R=P, lr=40, lp=48), dict(Z=P, lz=40, lp=48, act=1), dict(D=2 * P, Z=2 * P, act=1)):
        assert inp(**kw) == "E_INVALID_ARG", kw

    def wgt(G=P, X=P, dW=P, ldw=0, db=None, n=n, dtype=0, w=P, wb=ws):
        return status(dt.dattri_linear_weight_grad, G, 0, X, 0, dW, ldw, db, 0, n, i, o, dtype, w, wb, 0)
    for kw in (dict(G=None), dict(X=None), dict(dW=None), dict(ldw=23), dict(db=P + 2), dict(n=-2)):
        assert wgt(**kw) == "E_INVALID_ARG", kw
    lib = dt.load()
    assert lib.dattri_linear_workspace_bytes(0, 1, 1, 1, 0, 0, None) == -1
    assert status(linear_ws, 3, 1, 1, 1, 0, 0) == "E_INVALID_ARG"
    assert status(linear_ws, 0, 1, 1, 1, 4, 0) == "E_DTYPE"


@pytest.mark.parametrize("op", range(3))
@pytest.mark.parametrize("dtype", [0, 1])
def test_linear_workspace_is_checked(op, dtype):
    """Wherever a call needs workspace, less of it, none and a misaligned one are refused."""
    for n, i, o in ((1, 4096, 64), (3, 33, 65), (64, 8192, 64), (129, 4096, 72), (1030, 200, 264)):
        for off in (0, 4):  # aligned operands and misaligned ones
            need = linear_ws(op, n, i, o, dtype, off == 0)
            assert need <= linear_ws(op, n, i, o, dtype, False)
            a = P + off

            def call(w, wb):
                if op == 0:
                    dt.dattri_linear(a, 0, a, 0, None, 0, None, 0, P, 0, None, 0, n, i, o, dtype, w, wb, 0)
                elif op == 1:
                    dt.dattri_linear_input_grad(a, 0, a, 0, None, 0, 0, None, 0, None, 0, P, 0, n, i, o, dtype, w, wb, 0)
                else:
                    dt.dattri_linear_weight_grad(a, 0, a, 0, P, 0, P, 0, n, i, o, dtype, w, wb, 0)
            if need:
                for w, wb in ((None, need), (P, need - 1), (P + 128, need)):
                    assert status(call, w, wb) == "E_WORKSPACE"


def arrays(ptrs, sizes, types):
    n = len(ptrs)
    return (ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*sizes), (ctypes.c_int32 * n)(*types)


def test_clip_errors():
    def call(ptrs=(P, P), sizes=(5, 0), types=(0, 1), outs=(P, P), otypes=(0, 1), bound=1.0, nc=P, w=P, wb=1 << 20):
        g, s, t = arrays(ptrs, sizes, types)
        o = (ctypes.c_void_p * len(outs))(*outs) if outs is not None else None
        ot = (ctypes.c_int32 * len(otypes))(*otypes) if otypes is not None else None
        return status(dt.dattri_clip_gradients, g, s, t, o, ot, len(sizes), bound, nc, w, wb, 0)
    for kw in (dict(ptrs=(None, P)), dict(sizes=(-1, 2)), dict(outs=(None, P)), dict(outs=None), dict(otypes=None),
               dict(bound=-1.0), dict(bound=float("nan")), dict(nc=None), dict(nc=P + 2), dict(ptrs=(P + 2, P)),
               dict(otypes=(1, 1))):
        assert call(**kw) == "E_INVALID_ARG", kw
    for kw in (dict(types=(3, 0)), dict(otypes=(0, 2))):
        assert call(**kw) == "E_DTYPE", kw
    for kw in (dict(w=None), dict(wb=8), dict(w=P + 8)):
        assert call(**kw) == "E_WORKSPACE", kw
    assert dt.load().dattri_clip_gradients(None, None, None, None, None, 1, 1.0, P, P, 1024, None) == -1
    assert dt.load().dattri_clip_workspace_bytes(None, 1, ctypes.byref(ctypes.c_size_t())) == -1
    assert dt.load().dattri_clip_workspace_bytes(None, 0, None) == -1
    one = (ctypes.c_int64 * 1)(1 << 50)
    assert status(dt.dattri_clip_workspace_bytes, one, 1) == "E_UNSUPPORTED"


def test_clip_workspace_grows_with_the_list():
    sizes = (ctypes.c_int64 * 1000)(*([1 << 20] * 1000))
    assert dt.dattri_clip_workspace_bytes(sizes, 0) > 0
    assert dt.dattri_clip_workspace_bytes(sizes, 1000) >= dt.dattri_clip_workspace_bytes(sizes, 1)
