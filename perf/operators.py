"""Performance cases of the model-side operators: the step of the attributed model that makes the factor blocks.

Each case is one pass through one operator on seeded synthetic inputs that are already on the GPU:

* ``linear``     Y = act(X W^T + b) + R, with the pre-activation kept where a backward pass will want it
* ``backward``   the products behind it: the gradient of the layer's input times the derivative of the activation
                 below (the factor block of the layer below), and the weight and bias gradients
* ``embedding``  rows of a table looked up by token and scaled
* ``embgrad``    the gradient of that table: rows summed by token
* ``clip``       the norm of all gradients of a model together, and the gradients scaled to a largest norm

``listed`` names the cases, ``draw`` makes more from the same ranges, ``exact`` is the same in float64.  Where ``own``
is false ``run`` computes the operators with elementary torch operations in float32, rounded once at the end.
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
ELT = {"f32": 4, "bf16": 2}

# Weight shapes of one transformer block, [d_out, d_in], whose gradients are clipped together.
FAMILIES = {
    "adapters": [(8, 4096), (4096, 8), (8, 4096), (1024, 8), (8, 4096), (14336, 8), (8, 14336), (4096, 8)],
    "pythia410m": [(1024, 1024), (1024,), (1024, 4096), (1024,), (4096, 1024), (4096,), (1024,), (1024,)],
    "llama8b": [(4096, 4096), (1024, 4096), (1024, 4096), (4096, 4096), (14336, 4096), (14336, 4096), (4096, 14336),
                (4096,), (4096,)],
    "odd": [(257, 129), (1,), (33, 65), (0,), (1023,), (77, 501)],
}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # One token through a wide layer while serving: the weights are read once, nothing else counts.
        {"name": "linear one token bf16", "op": "linear", "rows": 1, "d_in": 4096, "d_out": 14336, "dtype": "bf16",
         "bias": True, "act": "silu", "residual": False, "keep": False},
        # The down projection over a capture batch of 8 sequences of 2048 tokens, bf16: the largest product.
        {"name": "linear batch bf16", "op": "linear", "rows": 16384, "d_in": 14336, "d_out": 4096, "dtype": "bf16",
         "bias": True, "act": "none", "residual": True, "keep": False},
        # A small model's layer in float32 with a ragged batch and widths that no tile divides; kept for backward.
        {"name": "linear odd sizes f32", "op": "linear", "rows": 999, "d_in": 769, "d_out": 2305, "dtype": "f32",
         "bias": True, "act": "gelu", "residual": False, "keep": True},
        # The backward products of a wide layer of a training batch, bf16 with float32 weight gradients.
        {"name": "backward batch bf16", "op": "backward", "rows": 8192, "d_in": 4096, "d_out": 14336, "dtype": "bf16",
         "act": "gelu_tanh", "residual": True},
        # The same for a small model in float32, the precision of fidelity runs, with a ragged number of tokens.
        {"name": "backward ragged f32", "op": "backward", "rows": 1531, "d_in": 1024, "d_out": 4096, "dtype": "f32",
         "act": "gelu", "residual": True},
        # One token's embedding while serving: the call itself.
        {"name": "embedding one token bf16", "op": "embedding", "tokens": 1, "vocab": 128000, "d": 4096,
         "dtype": "bf16", "scale": 64.0},
        # A capture batch's lookup, with padding among the tokens.
        {"name": "embedding batch bf16", "op": "embedding", "tokens": 16384, "vocab": 128000, "d": 4096,
         "dtype": "bf16", "scale": 64.0},
        # The table gradient of one short sequence of a small model, float32, odd sizes.
        {"name": "embedding gradient short f32", "op": "embgrad", "tokens": 509, "vocab": 10007, "d": 769,
         "dtype": "f32", "scale": 1.0},
        # The table gradient of a whole batch: few tokens are most of it, and most rows of the table have none.
        {"name": "embedding gradient batch bf16", "op": "embgrad", "tokens": 16384, "vocab": 128000, "d": 4096,
         "dtype": "bf16", "scale": 64.0},
        # An adapter's many small gradients, clipped: launches and latency.
        {"name": "clip adapters f32", "op": "clip", "family": "adapters", "blocks": 32, "dtype": "f32",
         "clipped": True, "into": "f32"},
        # A small model whose norm stays below the bound, as in most steps: the gradients are left as they are.
        {"name": "clip small model in place bf16", "op": "clip", "family": "pythia410m", "blocks": 24, "dtype": "bf16",
         "clipped": False, "into": "self"},
        # Blocks of an 8B model, bf16 gradients clipped into the optimizer's float32 ones.
        {"name": "clip large blocks bf16 to f32", "op": "clip", "family": "llama8b", "blocks": 4, "dtype": "bf16",
         "clipped": True, "into": "f32"},
    ]


# ------------------------------------------------------------------- drawing
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log_int(rng, lo, hi)
    return max(8, d // 8 * 8) if rng.random() < 0.7 else d  # most models' widths are multiples of 8


def draw(rng):
    op = rng.choice(["linear", "linear", "backward", "backward", "embedding", "embgrad", "clip"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("linear", "backward"):
        most = {"bf16": 1.9e12, "f32": 2e11}[dtype] / (2 if op == "backward" else 1)
        while True:
            rows = _log_int(rng, 1, 64) if rng.random() < 0.3 else _log_int(rng, 64, 16384)
            c = {"op": op, "rows": rows, "d_in": _width(rng, 8, 16384), "d_out": _width(rng, 8, 16384),
                 "dtype": dtype, "act": rng.choice(ACTS), "residual": rng.random() < 0.5}
            if op == "linear":
                c.update(bias=rng.random() < 0.7, keep=rng.random() < 0.4)
            if 2 * rows * c["d_in"] * c["d_out"] <= most:
                return c
    if op in ("embedding", "embgrad"):
        while True:
            c = {"op": op, "tokens": _log_int(rng, 1, 65536), "vocab": _log_int(rng, 64, 200000),
                 "d": _width(rng, 32, 8192), "dtype": dtype, "scale": rng.choice([1.0, 0.5, 32.0])}
            if c["vocab"] * c["d"] <= 128000 * 4096 and c["tokens"] * c["d"] <= 1.4e8:
                return c
    family = rng.choice(list(FAMILIES))
    blocks = _log_int(rng, 1, {"adapters": 64, "pythia410m": 24, "llama8b": 4, "odd": 64}[family])
    return {"op": "clip", "family": family, "blocks": blocks, "dtype": dtype, "clipped": rng.random() < 0.6,
            "into": rng.choice(["f32", "same"])}


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + 17) & ((1 << 62) - 1))
    return g


def _tokens(g, n, vocab):
    """Ids with frequencies of about 1 / rank, one in fifty outside the table (padding)."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    ids = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
    if n > 1:
        ids = torch.where(torch.rand(n, generator=g, device=DEV) < 0.02, torch.full_like(ids, -100), ids)
    return ids


def _shapes(c):
    return [s for _ in range(c["blocks"]) for s in FAMILIES[c["family"]]]


def _bucket(c):
    """Where each gradient starts in its bucket, and the bucket's size: on 64 elements, or back to back."""
    step = 1 if c["family"] == "odd" else 64
    offsets, at = [], 0
    for s in _shapes(c):
        offsets.append(at)
        at += -(-math.prod(s) // step) * step
    return offsets, at


def _views(c, bucket):
    return [bucket[at:at + math.prod(s)].view(s) for s, at in zip(_shapes(c), _bucket(c)[0])]


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = TORCH[c["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(dt)

    if c["op"] == "linear":
        n, i, o = c["rows"], c["d_in"], c["d_out"]
        return {"case": c, "x": normal(n, i), "w": normal(o, i, std=1.0 / math.sqrt(i)),
                "b": normal(o, std=0.2) if c["bias"] else None, "r": normal(n, o) if c["residual"] else None}
    if c["op"] == "backward":
        n, i, o = c["rows"], c["d_in"], c["d_out"]
        return {"case": c, "g": normal(n, o, std=1e-3), "x": normal(n, i), "w": normal(o, i, std=1.0 / math.sqrt(o)),
                "z": normal(n, i) if c["act"] != "none" else None,
                "r": normal(n, i, std=1e-3) if c["residual"] else None}
    if c["op"] == "embedding":
        return {"case": c, "table": normal(c["vocab"], c["d"], std=0.02), "ids": _tokens(g, c["tokens"], c["vocab"])}
    if c["op"] == "embgrad":
        return {"case": c, "g": normal(c["tokens"], c["d"], std=1e-3), "ids": _tokens(g, c["tokens"], c["vocab"])}
    # a bucket of gradients, each tensor a view of it, as data-parallel training keeps them
    offsets, size = _bucket(c)
    bucket = torch.zeros(size, dtype=dt, device=DEV)
    for s, at in zip(_shapes(c), offsets):
        bucket[at:at + math.prod(s)] = normal(math.prod(s), std=1e-3)
    total = sum(math.prod(s) for s in _shapes(c))
    bound = 1e-3 * math.sqrt(total) * (0.25 if c["clipped"] else 4.0)
    into = bucket if c["into"] == "self" else torch.zeros(size, dtype=torch.float32 if c["into"] == "f32" else dt,
                                                          device=DEV)
    return {"case": c, "grads": _views(c, bucket), "bound": bound, "out": _views(c, into), "into": into}


# ----------------------------------------------------------------- operators
def _act(z, kind):
    if kind == "relu":
        return z.clamp_min(0)
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if kind == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain(s):
    c = s["case"]
    dt = TORCH[c["dtype"]]
    if c["op"] == "linear":
        z = torch.matmul(s["x"].float(), s["w"].float().t())
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z, c["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return (y.to(dt), z.to(dt)) if c["keep"] else y.to(dt)
    if c["op"] == "backward":
        g = s["g"].float()
        d = torch.matmul(g, s["w"].float())
        if s["r"] is not None:
            d = d + s["r"].float()
        if s["z"] is not None:
            d = d * _act_slope(s["z"].float(), c["act"])
        return d.to(dt), torch.matmul(g.t(), s["x"].float()), g.sum(0)
    if c["op"] == "embedding":
        ok = (s["ids"] >= 0) & (s["ids"] < c["vocab"])
        rows = s["table"][torch.where(ok, s["ids"], 0)].float() * c["scale"]
        return torch.where(ok[:, None], rows, 0.0).to(dt)
    if c["op"] == "embgrad":
        ok = (s["ids"] >= 0) & (s["ids"] < c["vocab"])
        out = torch.zeros(c["vocab"] + 1, c["d"], device=DEV)  # the last row takes the ids outside the table
        out.index_add_(0, torch.where(ok, s["ids"], c["vocab"]), s["g"].float() * c["scale"])
        return out[:-1]
    norm = torch.sqrt(torch.stack([(t.float() * t.float()).sum() for t in s["grads"]]).sum())
    coef = (s["bound"] / (norm + 1e-6)).clamp_max(1.0)
    torch._foreach_copy_(s["out"], [t.float() * coef for t in s["grads"]])
    return {"out": s["into"], "norm": norm}


def run(state):
    if not own:
        return _plain(state)
    from paper_2609_38767_amd import layers
    s, c = state, state["case"]
    if c["op"] == "linear":
        return layers.linear(s["x"], s["w"], s["b"], act=c["act"], residual=s["r"], keep_preact=c["keep"])
    if c["op"] == "backward":
        d = layers.linear_input_grad(s["g"], s["w"], residual=s["r"], act=c["act"], preact=s["z"])
        dw, db = layers.linear_weight_grad(s["g"], s["x"], bias=True)
        return d, dw, db
    if c["op"] == "embedding":
        return layers.embedding(s["table"], s["ids"], scale=c["scale"])
    if c["op"] == "embgrad":
        return layers.embedding_grad(s["g"], s["ids"], c["vocab"], scale=c["scale"])
    norm, _ = layers.clip_gradients(s["grads"], s["bound"], out=s["out"])
    return {"out": s["into"], "norm": norm}


# --------------------------------------------------------------- what it takes
def _distinct(tokens, vocab):
    """Expected number of distinct ids among `tokens` draws with frequencies log((k+2)/(k+1)) / log(vocab+1)."""
    k = torch.arange(vocab, dtype=torch.float64)
    p = 0.98 * torch.log((k + 2) / (k + 1)) / math.log(vocab + 1.0)
    return float((1 - torch.exp(tokens * torch.log1p(-p))).sum())


def work(case):
    c = case
    e = ELT[c["dtype"]]
    if c["op"] == "linear":
        n, i, o = c["rows"], c["d_in"], c["d_out"]
        outs = n * o * (1 + bool(c["keep"]) + bool(c["residual"]))
        return {"bytes": e * (n * i + i * o + o * bool(c["bias"]) + outs), "flops": 2 * n * i * o}
    if c["op"] == "backward":
        n, i, o = c["rows"], c["d_in"], c["d_out"]
        below = n * i * (2 + (c["act"] != "none") + bool(c["residual"]))  # X in, the gradient out, Z and R in
        return {"bytes": e * (n * o + i * o + below) + 4 * (i * o + o), "flops": 4 * n * i * o + n * o}
    if c["op"] == "embedding":
        return {"bytes": int(e * c["d"] * (_distinct(c["tokens"], c["vocab"]) + c["tokens"]) + 8 * c["tokens"]),
                "flops": c["tokens"] * c["d"]}
    if c["op"] == "embgrad":
        return {"bytes": c["tokens"] * (e * c["d"] + 8) + 4 * c["vocab"] * c["d"], "flops": c["tokens"] * c["d"]}
    total = sum(math.prod(s) for s in _shapes(c))
    written = {"f32": 4, "same": e, "self": e if c["clipped"] else 0}[c["into"]]
    return {"bytes": total * (e + written), "flops": 2 * total + (total if written else 0)}


# ----------------------------------------------------------------- in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "linear":
        z = s["x"].double() @ s["w"].double().mT
        z = z if s["b"] is None else z.add_(s["b"].double())
        y = {"none": lambda v: v.clone(), "relu": lambda v: torch.where(v > 0, v, 0.0),
             "gelu": lambda v: v * torch.special.ndtr(v),
             "gelu_tanh": lambda v: v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)),
             "silu": lambda v: v * torch.sigmoid(v)}[c["act"]](z)
        y = y if s["r"] is None else y.add_(s["r"].double())
        return (y, z) if c["keep"] else y
    if c["op"] == "backward":
        g = s["g"].double()
        d = g @ s["w"].double()
        d = d if s["r"] is None else d.add_(s["r"].double())
        if s["z"] is not None:
            z = s["z"].double()
            if c["act"] == "relu":
                d = torch.where(z > 0, d, 0.0)
            elif c["act"] == "gelu":  # Phi(z) + z phi(z)
                d = d * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
            elif c["act"] == "gelu_tanh":  # z sigma(2u): sigma + 2 z u' sigma (1 - sigma)
                a = math.sqrt(2 / math.pi)
                q = torch.sigmoid(2 * a * (z + 0.044715 * z ** 3))
                d = d * (q + 2 * z * a * (1 + 0.134145 * z ** 2) * q * (1 - q))
            else:
                q = torch.sigmoid(z)
                d = d * (q + z * q * (1 - q))
        return d, g.mT.contiguous() @ s["x"].double(), g.sum(0)
    if c["op"] == "embedding":
        padded = torch.cat([s["table"].double() * c["scale"], torch.zeros(1, c["d"], device=DEV, dtype=torch.float64)])
        return padded[torch.where((s["ids"] < 0) | (s["ids"] >= c["vocab"]), c["vocab"], s["ids"])]
    if c["op"] == "embgrad":
        keep = (s["ids"] >= 0) & (s["ids"] < c["vocab"])
        out = torch.zeros(c["vocab"], c["d"], device=DEV, dtype=torch.float64)
        return out.index_put_((s["ids"][keep],), s["g"][keep].double() * c["scale"], accumulate=True)
    squares = sum(float(t.double().pow(2).sum()) for t in s["grads"])
    norm = math.sqrt(squares)
    coef = min(1.0, s["bound"] / (norm + 1e-6))
    out = torch.zeros(s["into"].numel(), dtype=torch.float64, device=DEV)
    for at, t in zip(_bucket(c)[0], s["grads"]):
        out[at:at + t.numel()] = t.reshape(-1).double() * coef
    return {"out": out, "norm": torch.tensor(norm, dtype=torch.float64, device=DEV)}
