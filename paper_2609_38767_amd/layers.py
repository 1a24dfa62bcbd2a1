"""The model-side operators over the C ABI, with torch owning the device buffers.

``embedding`` / ``embedding_grad``, ``linear`` / ``linear_input_grad`` /
``linear_weight_grad`` and ``gradient_norm`` / ``clip_gradients`` make up the
step of an attributed model: the inputs given to ``linear`` are the blocks A and
the rows that ``linear_input_grad`` returns are the blocks B that a
``ProjectionSession`` captures.  All computation happens in libdattri's HIP
kernels.

Nothing here is differentiated by autograd: results do not require grad whatever
the inputs do, and the backward products are calls of their own.  Writing into a
tensor counts as a change of it, so that autograd refuses to use what it has
saved of it.

Rows are the last axis: ``x [..., d]`` with unit stride along d and one stride
between rows (a contiguous tensor, or a view of padded rows).  An output may not
share memory with what else the call reads or writes, except where a function
says that it may be one of its inputs.  ``stream`` is a
torch stream or a raw handle of the tensors' GPU, or None (its current one);
outputs and workspaces are allocated on the stream that the call runs on.  As
with torch's own streams it has to wait for what made the inputs, and they have
to live until it has read them.
"""
from array import array
from operator import attrgetter

import torch

from . import (DATTRI_BF16, DATTRI_F32, DATTRI_ACT_GELU, DATTRI_ACT_GELU_TANH, DATTRI_ACT_NONE, DATTRI_ACT_RELU,
               DATTRI_ACT_SILU, DATTRI_LINEAR_FORWARD, DATTRI_LINEAR_INPUT_GRAD, DATTRI_LINEAR_WEIGHT_GRAD,
               dattri_clip_gradients, dattri_clip_workspace_bytes, dattri_embedding, dattri_embedding_grad,
               dattri_embedding_grad_workspace_bytes, dattri_linear, dattri_linear_input_grad, dattri_linear_weight_grad,
               dattri_linear_workspace_bytes)

ACTS = {"none": DATTRI_ACT_NONE, "relu": DATTRI_ACT_RELU, "gelu": DATTRI_ACT_GELU,
        "gelu_tanh": DATTRI_ACT_GELU_TANH, "silu": DATTRI_ACT_SILU}
_CODES = {torch.float32: DATTRI_F32, torch.bfloat16: DATTRI_BF16}
_dtype = attrgetter("dtype")


def _elsewhere(t, stream):
    """None if the call runs where it is, else the context to run it in: the
    tensors' device, the stream that was asked for."""
    if stream is None and t.device.index == torch.cuda.current_device():
        return None
    dev = torch.cuda.device(t.device)
    if stream is None:
        return dev
    if isinstance(stream, int):
        with dev:  # handle 0 is the default stream, which has an object of its own
            stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    elif stream.device != t.device:
        raise ValueError(f"stream is on {stream.device}, the tensors on {t.device}")
    return torch.cuda.stream(stream)


def _on_gpu(*tensors):
    dev = None
    for t in tensors:
        if t is not None:
            if not t.is_cuda:
                raise ValueError("tensors must be on the GPU")
            if dev is not None and t.device != dev:
                raise ValueError("tensors must be on one GPU")
            dev = t.device


def _code(t, what):
    code = _CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32 or bfloat16, not {t.dtype}")
    return code


def _rows(t, what, dtype=None, shape=None, width=None):
    """(rows, width, stride between rows) of t [..., width]."""
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} is {t.dtype}, expected {dtype}")
    if t.dim() == 0:
        raise ValueError(f"{what} needs at least one axis")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} is {tuple(t.shape)}, expected {tuple(shape)}")
    w = t.shape[-1]
    if width is not None and w != width:
        raise ValueError(f"{what} has rows of {w}, expected {width}")
    n = t.numel() // w if w else 0
    if t.is_contiguous():
        return n, w, w
    if w > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what} must have unit stride along its last axis")
    ld, span = None, 1  # the stride of the innermost axis with several rows; every other one continues it
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = stride
        elif stride != ld * span:
            raise ValueError(f"{what} must have one stride between its rows")
        span *= size
    if ld is not None and ld < w:
        raise ValueError(f"the rows of {what} overlap")
    return n, w, ld if ld is not None else w


def _matrix(t, what, dtype, width=None, shape=None):
    if t.dim() != 2:
        raise ValueError(f"{what} must have two axes")
    return _rows(t, what, dtype, shape, width)


def _vector(t, what, n, dtype):
    if t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} vector of {n}")


def _tokens(tokens):
    if tokens.dtype not in (torch.int32, torch.int64):
        raise ValueError("tokens must be int32 or int64")
    return tokens if tokens.is_contiguous() else tokens.contiguous()


def _act(act):
    if act not in ACTS:
        raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTS)}")
    return ACTS[act]


def _on_16(t, ld):
    e = t.element_size()
    return t.data_ptr() % 16 == 0 and ld * e % 16 == 0


def _changed(out):
    """The kernels write behind torch's back: tells autograd that what the
    caller handed in (a tensor, a list of them or None) has changed."""
    if out is not None:
        torch.autograd.graph.increment_version(out)


def _workspace(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def embedding(table, tokens, scale=1.0, out=None, stream=None):
    """scale * table[tokens]: [*tokens.shape, d] of the table's type.  Tokens
    outside the table (padding) give zeros."""
    _on_gpu(table, tokens, out)
    ctx = _elsewhere(table, stream)
    if ctx is not None:
        with ctx:
            return embedding(table, tokens, scale, out)
    code = _code(table, "table")
    tokens = _tokens(tokens)
    vocab, d, ld = _matrix(table, "table", table.dtype)
    given = out
    if out is None:
        out = torch.empty((*tokens.shape, d), dtype=table.dtype, device=table.device)
    n, _, ld_out = _rows(out, "out", table.dtype, (*tokens.shape, d))
    dattri_embedding(table, ld, vocab, d, code, tokens, tokens.element_size(), tokens.numel(), scale, out, ld_out)
    _changed(given)
    return out


def embedding_grad(grad_out, tokens, vocab, scale=1.0, out=None, accumulate=False, stream=None):
    """Gradient [vocab, d] (float32) of an embedding table from the gradient
    [*tokens.shape, d] of the looked-up rows.  accumulate=True adds to `out`."""
    _on_gpu(grad_out, tokens, out)
    ctx = _elsewhere(grad_out, stream)
    if ctx is not None:
        with ctx:
            return embedding_grad(grad_out, tokens, vocab, scale, out, accumulate)
    code = _code(grad_out, "grad_out")
    tokens = _tokens(tokens)
    if grad_out.shape[:-1] != tokens.shape:
        raise ValueError(f"grad_out is {tuple(grad_out.shape)} for tokens of {tuple(tokens.shape)}")
    _, d, ld = _rows(grad_out, "grad_out")
    given = out
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((vocab, d), dtype=torch.float32, device=grad_out.device)
    _, _, ld_out = _matrix(out, "out", torch.float32, shape=(vocab, d))
    n = tokens.numel()
    ws_bytes = dattri_embedding_grad_workspace_bytes(n, vocab, d)
    dattri_embedding_grad(grad_out, ld, code, tokens, tokens.element_size(), n, scale, vocab, d, out, ld_out,
                          accumulate, _workspace(ws_bytes, out.device), ws_bytes)
    _changed(given)
    return out


def linear(x, weight, bias=None, act="none", residual=None, keep_preact=False, out=None, stream=None):
    """y = act(x weight^T + bias) + residual, weight [d_out, d_in]; with
    keep_preact (y, z), z = x weight^T + bias.  `out` may be the residual."""
    _on_gpu(x, weight, bias, residual, out)
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return linear(x, weight, bias, act, residual, keep_preact, out)
    code, dt = _code(x, "x"), x.dtype
    d_out, d_in, ld_w = _matrix(weight, "weight", dt)
    n, _, ld_x = _rows(x, "x", width=d_in)
    shape = x.shape[:-1] + (d_out,)
    if bias is not None:
        _vector(bias, "bias", d_out, dt)
    ld_r = _rows(residual, "residual", dt, shape)[2] if residual is not None else 0
    given = out
    if out is None:
        out = torch.empty(shape, dtype=dt, device=x.device)
    ld_y = _rows(out, "out", dt, shape)[2]
    z = torch.empty(shape, dtype=dt, device=x.device) if keep_preact else None
    ws_bytes = dattri_linear_workspace_bytes(DATTRI_LINEAR_FORWARD, n, d_in, d_out, code,
                                             _on_16(x, ld_x) and _on_16(weight, ld_w))
    dattri_linear(x, ld_x, weight, ld_w, bias, _act(act), residual, ld_r, out, ld_y, z, 0, n, d_in, d_out, code,
                  _workspace(ws_bytes, x.device), ws_bytes)
    _changed(given)
    return (out, z) if keep_preact else out


def linear_input_grad(g, weight, residual=None, act="none", preact=None, both=False, out=None, stream=None):
    """(g weight + residual) * act'(preact): the gradient of a layer's input
    carried through the activation below.  g [..., d_out] is the gradient of the
    layer's pre-activation, residual the gradient that reaches its input by
    other ways, preact the pre-activation below.  With act="none" the gradient
    of the input itself.  both=True returns (input gradient, that times the
    slope), where the layer below adds its residual after its activation.
    `out` receives the (last) result and may be the residual or preact."""
    _on_gpu(g, weight, residual, preact, out)
    ctx = _elsewhere(g, stream)
    if ctx is not None:
        with ctx:
            return linear_input_grad(g, weight, residual, act, preact, both, out)
    code, dt = _code(g, "g"), g.dtype
    d_out, d_in, ld_w = _matrix(weight, "weight", dt)
    n, _, ld_g = _rows(g, "g", width=d_out)
    shape = g.shape[:-1] + (d_in,)
    a = _act(act)
    if a != DATTRI_ACT_NONE and preact is None:
        raise ValueError(f"act={act!r} needs preact")
    ld_r = _rows(residual, "residual", dt, shape)[2] if residual is not None else 0
    ld_z = _rows(preact, "preact", dt, shape)[2] if preact is not None else 0
    given = out
    if out is None:
        out = torch.empty(shape, dtype=dt, device=g.device)
    ld_p = _rows(out, "out", dt, shape)[2]
    d = torch.empty(shape, dtype=dt, device=g.device) if both else None
    ws_bytes = dattri_linear_workspace_bytes(DATTRI_LINEAR_INPUT_GRAD, n, d_in, d_out, code,
                                             _on_16(g, ld_g) and _on_16(weight, ld_w))
    dattri_linear_input_grad(g, ld_g, weight, ld_w, residual, ld_r, a, preact, ld_z, d, 0, out, ld_p, n, d_in, d_out,
                             code, _workspace(ws_bytes, g.device), ws_bytes)
    _changed(given)
    return (d, out) if both else out


def linear_weight_grad(g, x, bias=False, out=None, out_bias=None, accumulate=False, stream=None):
    """g^T x, the float32 gradient [d_out, d_in] of a layer's weight from the
    gradient of its pre-activation and its input; with bias=True (that, the
    float32 column sums of g).  accumulate=True adds to out (and out_bias)."""
    _on_gpu(g, x, out, out_bias)
    ctx = _elsewhere(g, stream)
    if ctx is not None:
        with ctx:
            return linear_weight_grad(g, x, bias, out, out_bias, accumulate)
    code = _code(g, "g")
    n, d_out, ld_g = _rows(g, "g")
    if x.shape[:-1] != g.shape[:-1]:
        raise ValueError(f"x is {tuple(x.shape)} for g of {tuple(g.shape)}")
    _, d_in, ld_x = _rows(x, "x", g.dtype)
    if accumulate and (out is None or (bias and out_bias is None)):
        raise ValueError("accumulate needs out (and out_bias)")
    given = [t for t in (out, out_bias if bias else None) if t is not None]
    if out is None:
        out = torch.empty((d_out, d_in), dtype=torch.float32, device=g.device)
    ld_dw = _matrix(out, "out", torch.float32, shape=(d_out, d_in))[2]
    if bias and out_bias is None:
        out_bias = torch.empty(d_out, dtype=torch.float32, device=g.device)
    if bias:
        _vector(out_bias, "out_bias", d_out, torch.float32)
    ws_bytes = dattri_linear_workspace_bytes(DATTRI_LINEAR_WEIGHT_GRAD, n, d_in, d_out, code,
                                             _on_16(g, ld_g) and _on_16(x, ld_x))
    dattri_linear_weight_grad(g, ld_g, x, ld_x, out, ld_dw, out_bias if bias else None, accumulate, n, d_in, d_out,
                              code, _workspace(ws_bytes, g.device), ws_bytes)
    _changed(given)
    return (out, out_bias) if bias else out


def _host_list(tensors, what, device):
    """Host arrays of the tensors' addresses, element counts and types.  Whole
    lists at a time: a training step hands over hundreds of small tensors."""
    T, n = torch.Tensor, len(tensors)
    if set(map(T.get_device, tensors)) != {device}:
        raise ValueError(f"{what} must be on one GPU")
    if not all(map(T.is_contiguous, tensors)):
        raise ValueError(f"{what} must be contiguous")
    try:
        types = array("i", map(_CODES.__getitem__, map(_dtype, tensors)))
    except KeyError:
        raise ValueError(f"{what} must be float32 or bfloat16") from None
    return array("Q", map(T.data_ptr, tensors)), array("q", map(T.numel, tensors)), types


def _clip(grads, max_norm, out, stream):
    grads = grads if isinstance(grads, list) else list(grads)
    if not grads:
        raise ValueError("no gradients")
    _on_gpu(grads[0])
    ctx = _elsewhere(grads[0], stream)
    if ctx is not None:
        with ctx:
            return _clip(grads, max_norm, out, None)
    device = grads[0].get_device()
    src, sizes, types = _host_list(grads, "gradients", device)
    dst = otypes = None
    if out is grads:
        dst, otypes = src, types
    elif out is not None:
        out = list(out)
        dst, osizes, otypes = _host_list(out, "out", device)
        if osizes != sizes:
            raise ValueError("out must have the gradients' sizes")
    norm_coef = torch.empty(2, dtype=torch.float32, device=grads[0].device)
    n = len(grads)
    ws_bytes = dattri_clip_workspace_bytes(sizes, n)
    dattri_clip_gradients(src, sizes, types, dst, otypes, n, max_norm, norm_coef,
                          _workspace(ws_bytes, norm_coef.device), ws_bytes)
    _changed(out)
    return norm_coef[0], norm_coef[1]


def gradient_norm(grads, stream=None):
    """The 2-norm (a float32 scalar on the GPU) of all gradients together."""
    return _clip(grads, float("inf"), None, stream)[0]


def clip_gradients(grads, max_norm, out=None, stream=None):
    """Scales the gradients so that their 2-norm together is at most max_norm,
    in place or into `out` (tensors of the same sizes, float32 or bfloat16).
    No gradient may come twice (shared weights: once), nor overlap another.
    Returns (norm before, coefficient), float32 scalars on the GPU."""
    grads = list(grads)
    return _clip(grads, max_norm, grads if out is None else out, stream)
