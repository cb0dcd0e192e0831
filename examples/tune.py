"""Weak-column tuning of a small language model: its dense weights stay as they are packed, the weak columns are trained.

    python examples/tune.py [--steps 8]

Every block is: norm, up projection, relu, down projection (OwqLinear), then in one call the norm of what the block gives, a
gate, dropout, the residual sum and the next block's norm (residual_norm).  The loss is the mean of -log p of the next tokens
(token_logprobs), and the gradients go back through token_logprobs_backward, OwqLinear.backward and residual_norm_backward; the
random bits of dropout are drawn again there from (seed, step).  The residual is held in fp32.  Weights are random, quantised by
the library's own configuration search (4 bits, groups of 128, a few weak columns in fp16), and so are the tokens.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_02272_amd import binding as B  # noqa: E402

WEAK = (1, 40, 77, 200)
SCALE = 256.0             # of the loss, so that fp16 gradients stay in range


class Low:
    """A low-bit layer and its weak columns."""

    def __init__(self, d_in, d_out, g):
        w = (torch.randn(d_out, d_in, generator=g, device="cuda") * d_in ** -0.5).half()
        idx = torch.tensor(WEAK, dtype=torch.int32, device="cuda")
        scale, zero, codes, _, _ = B.search_config(w, idx, bits=4, group_size=128, n_lo=4, n_hi=4, shrink=0.2, want_err=False)

        class Layer:
            pass
        Layer.d_out, Layer.d_in, Layer.bits, Layer.group_size, Layer.k = d_out, d_in, 4, 128, len(WEAK)
        Layer.codes, Layer.scale, Layer.zero = codes.cpu().numpy(), scale.cpu().numpy(), zero.cpu().numpy()
        self.weak = w[:, idx.long()].contiguous()
        Layer.weak_idx, Layer.weak_w = idx.cpu().numpy(), self.weak.cpu().numpy()
        self.layer = Layer
        self.linear = B.OwqLinear(Layer, layout=B.OWQ_LAYOUT_TILE)

    def __call__(self, x):
        return self.linear(x)

    def update(self, weak):
        self.weak = weak.half().contiguous()
        B.owq_update_weak(self.linear.handle, self.weak.cpu().numpy(), B._current_stream(torch))


class Model:
    def __init__(self, blocks=2, width=256, inner=512, vocab=1000, p=0.1, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.p = p
        self.embed = torch.randn(vocab, width, generator=g, device="cuda")
        self.head = Low(width, vocab, g)

        def vector(about=1.0):
            return (about + 0.1 * torch.randn(width, generator=g, device="cuda")).half()
        self.first = vector()
        self.blocks = [{"up": Low(width, inner, g), "down": Low(inner, width, g), "post": vector(), "gate": vector(0.5), "norm": vector()}
                       for _ in range(blocks)]

    def layers(self):
        return [b[k] for b in self.blocks for k in ("up", "down")] + [self.head]

    def _options(self, i, rng):
        b = self.blocks[i]
        return dict(gate=b["gate"], post="rms", post_weight=b["post"], norm="rms", weight=b["norm"], rng=rng, p=self.p, site=i)

    def forward(self, tokens, rng):
        """Logits, and what the gradients need."""
        h = self.embed[tokens.long()]
        total, y = B.residual_norm(h, weight=self.first)
        kept = []
        for i, b in enumerate(self.blocks):
            a = b["up"](y)
            r = torch.relu(a)
            o = b["down"](r)
            into = y
            total, y = B.residual_norm(total, o, **self._options(i, rng))
            kept.append((into, r, o, total))
        return self.head(y), (h, y, kept)

    def loss(self, tokens, targets, rng):
        lp = B.token_logprobs(self.forward(tokens, rng)[0], targets)[0]
        return -lp.sum().item() / max(1, int((targets >= 0).sum()))

    def step(self, tokens, targets, count, rng):
        """(log-probabilities, gradients of SCALE times the loss: of the layers' weak columns in the order of layers(), of the vectors, of
        the embedded tokens), where `count` targets are counted.  Waits for nothing, so that a graph can hold it."""
        logits, (h, y, kept) = self.forward(tokens, rng)
        lp, _, _, stats = B.token_logprobs(logits, targets)
        dlp = torch.full_like(lp, -SCALE / count)
        dlogits = B.token_logprobs_backward(dlp, None, logits, targets, stats, out=logits)
        dy, dhead = self.head.linear.backward(dlogits, y)
        weak, vectors = [dhead], {}
        dtotal = None
        for i in reversed(range(len(self.blocks))):
            b, (into, r, o, total) = self.blocks[i], kept[i]
            dtotal, do, dgate, dpost, _, dnorm, _ = B.residual_norm_backward(dy, dtotal, total, o, **self._options(i, rng))
            dr, ddown = b["down"].linear.backward(do, r)
            dy, dup = b["up"].linear.backward(dr * (r > 0), into)
            weak = [dup, ddown] + weak
            vectors[i] = {"gate": dgate, "post": dpost, "norm": dnorm}
        dh, *_, dfirst, _ = B.residual_norm_backward(dy, dtotal, h, weight=self.first)
        vectors["first"] = dfirst
        return lp, weak, vectors, dh

    def gradients(self, tokens, targets, rng):
        """(loss, its gradients in the order of step())."""
        count = max(1, int((targets >= 0).sum()))
        lp, weak, vectors, dh = self.step(tokens, targets, count, rng)
        unscaled = {i: v / SCALE if torch.is_tensor(v) else {k: g / SCALE for k, g in v.items()} for i, v in vectors.items()}
        return -lp.sum().item() / count, [g / SCALE for g in weak], unscaled, dh / SCALE


def batch(model, rows=96, seed=1):
    """Tokens, the ones that follow them, a tenth not counted."""
    g = torch.Generator("cuda").manual_seed(seed)
    tokens = torch.randint(0, model.embed.shape[0], (rows,), generator=g, device="cuda", dtype=torch.int32)
    targets = tokens.roll(-1)
    targets[torch.rand(rows, generator=g, device="cuda") < 0.1] = -100
    return tokens, targets


def train(model, steps, rate=0.5):
    tokens, targets = batch(model)
    rng = torch.tensor([7, 0], dtype=torch.int64, device="cuda")
    losses = []
    for _ in range(steps):
        loss, weak, _, _ = model.gradients(tokens, targets, rng)
        for layer, g in zip(model.layers(), weak):
            layer.update(layer.weak.float() - rate * g)
        rng[1] += 1                      # other elements are dropped in the next step
        losses.append(loss)
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=8)
    for i, loss in enumerate(train(Model(), parser.parse_args().steps)):
        print(f"step {i}: loss {loss:.4f}")
