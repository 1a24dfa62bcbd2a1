"""Train a small residual language model with the model-side operators, then
attribute its predictions to its training sequences.

    python examples/attribute_mlp.py [--steps 30] [--dtype bf16]

The model is embedding -> blocks of two linear layers around a residual ->
output layer.  Its forward and backward passes are made of the library's
calls, so the blocks that attribution needs (each linear layer's input A and
the gradient B of its pre-activation) are there when the pass is over and are
captured where they lie.  The data are synthetic: sequences of a few "topics",
each a random cycle of tokens; the training sequences most responsible for a
query should be those of its topic.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_38767_amd import layers as L  # noqa: E402
from paper_2609_38767_amd.session import ProjectionSession, score  # noqa: E402


class Model:
    """Weights in the compute type with float32 masters; `passes` keeps what attribution reads."""

    def __init__(self, vocab, d, hidden, blocks, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.vocab = dtype, vocab

        def make(o, i):
            return torch.randn(o, i, generator=g, device="cuda") / math.sqrt(i)

        self.master = {"table": torch.randn(vocab, d, generator=g, device="cuda") / math.sqrt(d)}
        for b in range(blocks):
            self.master[f"up{b}"], self.master[f"up{b}.bias"] = make(hidden, d), torch.zeros(hidden, device="cuda")
            self.master[f"down{b}"] = make(d, hidden)
        self.master["out"] = make(vocab, d)
        self.blocks, self.scale = blocks, math.sqrt(d)
        self.sync()

    def sync(self):
        self.w = {k: v.to(self.dtype) for k, v in self.master.items()}

    def forward(self, tokens):
        """Logits [n, T, vocab] and the inputs and pre-activations of every layer."""
        w, kept = self.w, {}
        h = L.embedding(w["table"], tokens, scale=self.scale)
        for b in range(self.blocks):
            kept[f"up{b}"] = h
            u, kept[f"z{b}"] = L.linear(h, w[f"up{b}"], w[f"up{b}.bias"], act="gelu", keep_preact=True)
            kept[f"down{b}"] = u
            h = L.linear(u, w[f"down{b}"], residual=h)
        kept["out"] = h
        return L.linear(h, w["out"]), kept

    def backward(self, g_out, kept, tokens, weights=True):
        """From the logits' gradient: each linear layer's (A, B), and the weight gradients if asked for."""
        w, pairs, grads = self.w, {"out": (kept["out"], g_out)}, {}
        d = L.linear_input_grad(g_out, w["out"])
        for b in reversed(range(self.blocks)):
            pairs[f"down{b}"] = (kept[f"down{b}"], d)
            g = L.linear_input_grad(d, w[f"down{b}"], act="gelu", preact=kept[f"z{b}"])
            pairs[f"up{b}"] = (kept[f"up{b}"], g)
            d = L.linear_input_grad(g, w[f"up{b}"], residual=d)
        if weights:
            for name, (a, g) in pairs.items():
                if name.startswith("up"):
                    grads[name], grads[name + ".bias"] = L.linear_weight_grad(g, a, bias=True)
                else:
                    grads[name] = L.linear_weight_grad(g, a)
            grads["table"] = L.embedding_grad(d, tokens, self.vocab, scale=self.scale)
        return pairs, grads


def loss_and_gradient(logits, targets):
    """Summed next-token loss per sequence, and its gradient with respect to the logits."""
    p = torch.softmax(logits.float(), -1)
    nll = -torch.log(p.gather(-1, targets[..., None]).clamp_min(1e-30))[..., 0]
    p.scatter_add_(-1, targets[..., None], torch.full_like(nll, -1.0)[..., None])
    return nll.sum(1), p.to(logits.dtype)


def sequences(n, T, vocab, topics, seed):
    """n sequences of T + 1 tokens; topic i % topics is one fixed cycle through 12 tokens, entered anywhere."""
    g = torch.Generator().manual_seed(1)
    cycles = torch.stack([torch.randperm(vocab, generator=g)[:12] for _ in range(topics)])
    start = torch.randint(0, 12, (n,), generator=torch.Generator().manual_seed(seed))
    at = (start[:, None] + torch.arange(T + 1)[None]) % 12
    topic = torch.arange(n) % topics
    return cycles[topic].gather(1, at).cuda(), topic


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    ap.add_argument("--lr", type=float, default=0.3)
    a = ap.parse_args(argv)
    vocab, d, hidden, blocks, T, topics = 509, 64, 256, 2, 32, 8
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype]
    model = Model(vocab, d, hidden, blocks, dtype)
    train, topic = sequences(64, T, vocab, topics, seed=2)
    x, y = train[:, :-1].contiguous(), train[:, 1:]
    names = [n for b in range(blocks) for n in (f"up{b}", f"down{b}")] + ["out"]
    n_tokens = x.numel()
    losses = []
    for step in range(a.steps):
        logits, kept = model.forward(x)
        loss, g = loss_and_gradient(logits, y)
        _, grads = model.backward(g / n_tokens, kept, x)
        norm, _ = L.clip_gradients(list(grads.values()), 1.0)
        for k, v in grads.items():
            model.master[k].add_(v, alpha=-a.lr)
        model.sync()
        losses.append(loss.sum().item() / n_tokens)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step:3d}: loss {losses[-1]:.3f} per token, gradient norm {norm.item():.3f}")

    # projected gradients of queries and training sequences, by capture of the same pass
    dims = [dict(name=n, d_in=model.w[n].shape[1], d_out=model.w[n].shape[0], k_in=16, k_out=16) for n in names]
    session = ProjectionSession(dims, dtype=a.dtype, seed=0)

    def features(tokens):
        logits, kept = model.forward(tokens[:, :-1].contiguous())
        _, g = loss_and_gradient(logits, tokens[:, 1:])
        pairs, _ = model.backward(g, kept, tokens[:, :-1].contiguous(), weights=False)
        for i, n in enumerate(names):
            session.capture(i, *pairs[n])
        phi = session.project(tokens.shape[0])
        torch.cuda.synchronize()
        session.clear()
        return phi

    queries, q_topic = sequences(16, T, vocab, topics, seed=3)
    _, idx, _ = score(features(queries), features(train), topk=8, want_scores=False, cosine=True)
    hits = (topic.cuda()[idx.long()] == q_topic.cuda()[:, None]).float().mean().item()
    print(f"of each query's 8 most similar training sequences, {100 * hits:.0f}% share its topic "
          f"({100 / topics:.0f}% by chance)")
    return losses, hits


if __name__ == "__main__":
    main()
