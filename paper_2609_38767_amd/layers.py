"""The model-side operators over the C ABI, with torch owning the device buffers.

``embedding`` / ``embedding_grad``, ``rms_norm`` / ``rms_norm_grad``, ``linear`` /
``linear_input_grad`` / ``linear_weight_grad`` and ``gradient_norm`` /
``clip_gradients`` make up the step of an attributed model: the inputs given to
``linear`` are the blocks A and the rows that ``linear_input_grad`` returns are
the blocks B that a ``ProjectionSession`` captures.  ``expert_linear`` and its
backward products are the linear layers of a model of experts; ``linear_8bit``
is the linear layer of a model whose weights are held in 8 bits, with
``rms_norm_8bit`` or ``quantize_rows`` for its rows and ``quantize_weight`` and
``transpose_8bit`` for its weights.  All computation happens in libdattri's HIP
kernels (``transpose_8bit`` only moves values).

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
               dattri_embedding_grad_workspace_bytes, dattri_expert_linear, dattri_expert_linear_input_grad,
               dattri_expert_linear_weight_grad, dattri_expert_linear_workspace_bytes, dattri_linear, dattri_linear_scaled,
               dattri_linear_scaled_workspace_bytes, dattri_linear_input_grad, dattri_linear_weight_grad,
               dattri_linear_workspace_bytes, dattri_quantize_rows, dattri_quantize_weight, dattri_rms_norm,
               dattri_rms_norm_grad, dattri_rms_norm_grad_workspace_bytes)

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


def _like(t):
    """An empty tensor of t's shape and type, dense (0.6 us less than torch.empty takes for it)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


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


def rms_norm(x, weight, residual=None, eps=1e-6, out=None, out_sum=None, stream=None):
    """y = h / sqrt(mean(h^2) + eps) * weight over the last axis, h = x +
    residual; with a residual (y, h).  `out` and `out_sum` receive them and may
    each be x or the residual (not both the same)."""
    return _norm(x, weight, residual, eps, out, out_sum, True, False, stream)


def rms_norm_8bit(x, weight, residual=None, eps=1e-6, keep=False, out=None, out_sum=None, stream=None):
    """rms_norm with its result in 8 bits: (values [..., d] float8_e4m3fn, scales
    [..., ceil(d / 128)] float32), what ``linear_8bit`` takes for its rows.
    Returns that pair; with keep=True (or `out`) or a residual a tuple of it, y
    and h as far as they are there."""
    return _norm(x, weight, residual, eps, out, out_sum, keep or out is not None, True, stream)


def _norm(x, weight, residual, eps, out, out_sum, keep, eight, stream):
    _on_gpu(x, weight, residual, out, out_sum)
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return _norm(x, weight, residual, eps, out, out_sum, keep, eight, None)
    code, dt = _code(x, "x"), x.dtype
    n, d, ld_x = _rows(x, "x")
    _vector(weight, "weight", d, dt)
    ld_r = _rows(residual, "residual", dt, x.shape)[2] if residual is not None else 0
    if out_sum is not None and residual is None:
        raise ValueError("out_sum needs a residual")
    given = [t for t in (out, out_sum) if t is not None]
    ld_y = ld_h = 0  # dense, as what is made here is
    if out is not None:
        ld_y = _rows(out, "out", dt, x.shape)[2]
    elif keep:
        out = _like(x)
    if out_sum is not None:
        ld_h = _rows(out_sum, "out_sum", dt, x.shape)[2]
    elif residual is not None:
        out_sum = _like(x)
    q, s = _eight_bit_rows(x) if eight else (None, None)
    dattri_rms_norm(x, ld_x, residual, ld_r, weight, eps, out, ld_y, out_sum, ld_h, q, 0, s, 0, n, d, code)
    if given:
        _changed(given)
    got = ([(q, s)] if eight else []) + [t for t in (out, out_sum) if t is not None]
    return got[0] if len(got) == 1 else tuple(got)


def rms_norm_grad(g, h, weight, eps=1e-6, residual=None, weight_grad=True, out=None, out_weight=None, accumulate=False,
                  stream=None):
    """(gradient of h, float32 gradient of the weight) from the gradient g of
    rms_norm's y and its input h (x, or the sum); residual is the gradient that
    reaches h by other ways and is added.  weight_grad=False returns the first
    alone.  accumulate=True adds to out_weight.  `out` may be the residual."""
    _on_gpu(g, h, weight, residual, out, out_weight)
    ctx = _elsewhere(g, stream)
    if ctx is not None:
        with ctx:
            return rms_norm_grad(g, h, weight, eps, residual, weight_grad, out, out_weight, accumulate)
    code, dt = _code(g, "g"), g.dtype
    n, d, ld_g = _rows(g, "g")
    ld_h = _rows(h, "h", dt, g.shape)[2]
    _vector(weight, "weight", d, dt)
    ld_p = _rows(residual, "residual", dt, g.shape)[2] if residual is not None else 0
    if accumulate and (out_weight is None or not weight_grad):
        raise ValueError("accumulate needs out_weight")
    given = [t for t in (out, out_weight if weight_grad else None) if t is not None]
    ld_d = 0
    if out is None:
        out = _like(g)
    else:
        ld_d = _rows(out, "out", dt, g.shape)[2]
    if weight_grad:
        if out_weight is None:
            out_weight = weight.new_empty((d,), dtype=torch.float32)
        else:
            _vector(out_weight, "out_weight", d, torch.float32)
    ws_bytes = dattri_rms_norm_grad_workspace_bytes(n, d, code, weight_grad)
    dattri_rms_norm_grad(g, ld_g, h, ld_h, weight, eps, residual, ld_p, out, ld_d, out_weight if weight_grad else None,
                         accumulate, n, d, code, _workspace(ws_bytes, g.device), ws_bytes)
    if given:
        _changed(given)
    return (out, out_weight) if weight_grad else out


def _groups(d):
    return -(-d // 128)


def _eight_bit_rows(x):
    """Empty 8-bit rows of x's shape and their scales."""
    return (torch.empty_like(x, dtype=torch.float8_e4m3fn, memory_format=torch.contiguous_format),
            x.new_empty((*x.shape[:-1], _groups(x.shape[-1])), dtype=torch.float32))


def quantize_rows(x, stream=None):
    """Rows in 8 bits: (values [..., d] float8_e4m3fn, scales [..., ceil(d / 128)]
    float32), value times its group's scale standing for x."""
    _on_gpu(x)
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return quantize_rows(x)
    code = _code(x, "x")
    n, d, ld = _rows(x, "x")
    q, s = _eight_bit_rows(x)
    dattri_quantize_rows(x, ld, n, d, code, q, 0, s, 0)
    return q, s


def quantize_weight(weight, stream=None):
    """A weight in 8 bits: (values [d_out, d_in] float8_e4m3fn, scales
    [ceil(d_out / 128), ceil(d_in / 128)] float32 of its 128 x 128 blocks)."""
    _on_gpu(weight)
    ctx = _elsewhere(weight, stream)
    if ctx is not None:
        with ctx:
            return quantize_weight(weight)
    code = _code(weight, "weight")
    _matrix(weight, "weight", weight.dtype)
    d_out, d_in = weight.shape
    ld = _rows(weight, "weight")[2]
    q = torch.empty((d_out, d_in), dtype=torch.float8_e4m3fn, device=weight.device)
    s = torch.empty((_groups(d_out), _groups(d_in)), dtype=torch.float32, device=weight.device)
    dattri_quantize_weight(weight, ld, d_out, d_in, code, q, 0, s, 0)
    return q, s


def transpose_8bit(weight, stream=None):
    """The transposed 8-bit weight, with which ``linear_8bit`` carries a gradient
    back through the layer.  Laid out once, beside the weight: torch's copies,
    which compute nothing, into memory of its own."""
    q, s = weight
    if q.dtype != torch.float8_e4m3fn or q.dim() != 2 or s.shape != (_groups(q.shape[0]), _groups(q.shape[1])):
        raise ValueError("weight must be float8_e4m3fn of two axes with a scale for each 128 x 128 block")
    if q.is_cuda or s.is_cuda or stream is not None:
        _on_gpu(q, s)
        ctx = _elsewhere(q, stream)
        if ctx is not None:
            with ctx:
                return transpose_8bit(weight)
    return _transposed(q.view(torch.uint8)).view(torch.float8_e4m3fn), _transposed(s)


def _transposed(t):
    """A dense copy (t() of a single row or column may be t's own memory, dense already)."""
    return torch.empty((t.shape[1], t.shape[0]), dtype=t.dtype, device=t.device).copy_(t.detach().t())


def linear_8bit(x, weight, bias=None, act="none", residual=None, keep_preact=False, dtype=torch.bfloat16, out=None,
                stream=None):
    """y = act(x weight^T + bias) + residual of 8-bit rows x = (values, scales)
    and an 8-bit weight = (values, scales), as the functions above make them;
    with keep_preact (y, z).  bias, residual and results are of `dtype`; `out`
    may be the residual.  bf16 results lose, of eight products of neighbouring
    columns, the bits below 2^-13 of the largest, which shows beside bf16's own
    rounding where large terms cancel; float32 results keep all (half the rate)."""
    (x, sx), (weight, sw) = x, weight
    _on_gpu(x, sx, weight, sw, bias, residual, out)
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return linear_8bit((x, sx), (weight, sw), bias, act, residual, keep_preact, dtype, out)
    if dtype not in _CODES:
        raise ValueError(f"dtype must be float32 or bfloat16, not {dtype}")
    code = _CODES[dtype]
    d_out, d_in, ld_w = _matrix(weight, "weight", torch.float8_e4m3fn)
    n, _, ld_x = _rows(x, "x", torch.float8_e4m3fn, width=d_in)
    ld_sx = _rows(sx, "scales of x", torch.float32, x.shape[:-1] + (_groups(d_in),))[2]
    ld_sw = _matrix(sw, "scales of the weight", torch.float32, shape=(_groups(d_out), _groups(d_in)))[2]
    shape = x.shape[:-1] + (d_out,)
    if bias is not None:
        _vector(bias, "bias", d_out, dtype)
    ld_r = _rows(residual, "residual", dtype, shape)[2] if residual is not None else 0
    given, ld_y = out, 0
    if out is None:
        out = x.new_empty(shape, dtype=dtype)
    else:
        ld_y = _rows(out, "out", dtype, shape)[2]
    z = _like(out) if keep_preact else None
    ws_bytes = dattri_linear_scaled_workspace_bytes(n, d_in, d_out, code, _on_16(x, ld_x) and _on_16(weight, ld_w))
    dattri_linear_scaled(x, ld_x, sx, ld_sx, weight, ld_w, sw, ld_sw, bias, _act(act), residual, ld_r, out, ld_y, z, 0, n,
                       d_in, d_out, code, _workspace(ws_bytes, x.device), ws_bytes)
    _changed(given)
    return (out, z) if keep_preact else out


def _experts(weight, offsets, dtype):
    """(experts, d_out, d_in, row stride) of a weight [experts, d_out, d_in] and
    the offsets [experts + 1] of its experts' rows."""
    if weight.dim() != 3:
        raise ValueError("weight must have three axes")
    e, d_out, d_in = weight.shape
    ld = _rows(weight, "weight", dtype)[2]
    return e, d_out, d_in, ld, _offsets(offsets, e)


def _offsets(offsets, experts=None):
    if offsets.dtype not in (torch.int32, torch.int64):
        raise ValueError("offsets must be int32 or int64")
    if offsets.dim() != 1 or offsets.numel() < 2 or (experts is not None and offsets.numel() != experts + 1):
        raise ValueError("offsets must be a vector of one more than the experts")
    return offsets if offsets.is_contiguous() else offsets.contiguous()


def _bias_rows(t, what, experts, d_out, dtype):
    if t.dtype != dtype or t.shape != (experts, d_out) or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} of {experts} x {d_out}")


def expert_linear(x, weight, offsets, bias=None, act="none", residual=None, keep_preact=False, out=None, stream=None):
    """``linear`` with a weight for each expert: rows offsets[e] .. offsets[e + 1]
    - 1 of x [n, d_in] (all leading axes as one) meet weight[e], weight
    [experts, d_out, d_in], bias [experts, d_out].  offsets (int32 or int64, on
    the GPU, ascending within [0, n]) are not read on the host.  Rows of no
    expert, in front of offsets[0] and from offsets[-1] on, come out as with
    zero weights and bias: y = residual, z = 0."""
    _on_gpu(x, weight, offsets, bias, residual, out)
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return expert_linear(x, weight, offsets, bias, act, residual, keep_preact, out)
    code, dt = _code(x, "x"), x.dtype
    e, d_out, d_in, ld_w, offsets = _experts(weight, offsets, dt)
    n, _, ld_x = _rows(x, "x", width=d_in)
    shape = x.shape[:-1] + (d_out,)
    if bias is not None:
        _bias_rows(bias, "bias", e, d_out, dt)
    ld_r = _rows(residual, "residual", dt, shape)[2] if residual is not None else 0
    given, ld_y = out, 0
    if out is None:
        out = x.new_empty(shape)
    else:
        ld_y = _rows(out, "out", dt, shape)[2]
    z = _like(out) if keep_preact else None
    ws_bytes = dattri_expert_linear_workspace_bytes(DATTRI_LINEAR_FORWARD, n, e, d_in, d_out, code,
                                                    _on_16(x, ld_x) and _on_16(weight, ld_w))
    dattri_expert_linear(x, ld_x, weight, ld_w, bias, offsets, offsets.element_size(), _act(act), residual, ld_r, out,
                         ld_y, z, 0, n, e, d_in, d_out, code, _workspace(ws_bytes, x.device), ws_bytes)
    _changed(given)
    return (out, z) if keep_preact else out


def expert_linear_input_grad(g, weight, offsets, residual=None, act="none", preact=None, both=False, out=None,
                             stream=None):
    """``linear_input_grad`` with a weight for each expert, rows as for
    ``expert_linear``: (g weight[e] + residual) * act'(preact)."""
    _on_gpu(g, weight, offsets, residual, preact, out)
    ctx = _elsewhere(g, stream)
    if ctx is not None:
        with ctx:
            return expert_linear_input_grad(g, weight, offsets, residual, act, preact, both, out)
    code, dt = _code(g, "g"), g.dtype
    e, d_out, d_in, ld_w, offsets = _experts(weight, offsets, dt)
    n, _, ld_g = _rows(g, "g", width=d_out)
    shape = g.shape[:-1] + (d_in,)
    a = _act(act)
    if a != DATTRI_ACT_NONE and preact is None:
        raise ValueError(f"act={act!r} needs preact")
    ld_r = _rows(residual, "residual", dt, shape)[2] if residual is not None else 0
    ld_z = _rows(preact, "preact", dt, shape)[2] if preact is not None else 0
    given, ld_p = out, 0
    if out is None:
        out = g.new_empty(shape)
    else:
        ld_p = _rows(out, "out", dt, shape)[2]
    d = _like(out) if both else None
    ws_bytes = dattri_expert_linear_workspace_bytes(DATTRI_LINEAR_INPUT_GRAD, n, e, d_in, d_out, code,
                                                    _on_16(g, ld_g) and _on_16(weight, ld_w))
    dattri_expert_linear_input_grad(g, ld_g, weight, ld_w, offsets, offsets.element_size(), residual, ld_r, a, preact,
                                    ld_z, d, 0, out, ld_p, n, e, d_in, d_out, code, _workspace(ws_bytes, g.device),
                                    ws_bytes)
    _changed(given)
    return (d, out) if both else out


def expert_linear_weight_grad(g, x, offsets, bias=False, out=None, out_bias=None, accumulate=False, stream=None):
    """``linear_weight_grad`` of every expert from its rows: float32 [experts,
    d_out, d_in], with bias=True also [experts, d_out].  Experts without rows
    get zeros, or with accumulate=True keep what is there."""
    _on_gpu(g, x, offsets, out, out_bias)
    ctx = _elsewhere(g, stream)
    if ctx is not None:
        with ctx:
            return expert_linear_weight_grad(g, x, offsets, bias, out, out_bias, accumulate)
    code = _code(g, "g")
    offsets = _offsets(offsets)
    e = offsets.numel() - 1
    n, d_out, ld_g = _rows(g, "g")
    if x.shape[:-1] != g.shape[:-1]:
        raise ValueError(f"x is {tuple(x.shape)} for g of {tuple(g.shape)}")
    _, d_in, ld_x = _rows(x, "x", g.dtype)
    if accumulate and (out is None or (bias and out_bias is None)):
        raise ValueError("accumulate needs out (and out_bias)")
    given = [t for t in (out, out_bias if bias else None) if t is not None]
    if out is None:
        out = torch.empty((e, d_out, d_in), dtype=torch.float32, device=g.device)
    ld_dw = _rows(out, "out", torch.float32, (e, d_out, d_in))[2]
    if bias and out_bias is None:
        out_bias = torch.empty((e, d_out), dtype=torch.float32, device=g.device)
    if bias:
        _bias_rows(out_bias, "out_bias", e, d_out, torch.float32)
    ws_bytes = dattri_expert_linear_workspace_bytes(DATTRI_LINEAR_WEIGHT_GRAD, n, e, d_in, d_out, code,
                                                    _on_16(g, ld_g) and _on_16(x, ld_x))
    dattri_expert_linear_weight_grad(g, ld_g, x, ld_x, offsets, offsets.element_size(), out, ld_dw,
                                     out_bias if bias else None, accumulate, n, e, d_in, d_out, code,
                                     _workspace(ws_bytes, g.device), ws_bytes)
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
