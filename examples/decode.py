"""A small decoder whose layers are low-bit and whose cache is 4-bit, from prompt tokens to sampled ones.

    python examples/decode.py [--steps 16]

Every block is: norm, one projection for queries, keys and values (OwqLinear), norm of the heads with rotation
(qk_norm_rope), the keys and values into the cache (cache_append), attention over it (cache_attention), output projection,
norm, feed-forward pair.  A prompt and a single token take the same path.  Weights are random, quantised by the library's
own configuration search (4 bits, groups of 128, a few weak columns in fp16), so the text means nothing.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_02272_amd import binding as B  # noqa: E402

WEAK = (3, 64, 200)


def low_bit(d_in, d_out, g):
    """A random layer of fp16 weights, searched and packed (tile layout: batches and single tokens)."""
    w = (torch.randn(d_out, d_in, generator=g, device="cuda") * d_in ** -0.5).half()
    idx = torch.tensor(WEAK, dtype=torch.int32, device="cuda")
    scale, zero, codes, _, _ = B.search_config(w, idx, bits=4, group_size=128, n_lo=4, n_hi=4, shrink=0.2, want_err=False)

    class Layer:
        pass
    Layer.d_out, Layer.d_in, Layer.bits, Layer.group_size, Layer.k = d_out, d_in, 4, 128, len(WEAK)
    Layer.codes, Layer.scale, Layer.zero = codes.cpu().numpy(), scale.cpu().numpy(), zero.cpu().numpy()
    Layer.weak_idx, Layer.weak_w = idx.cpu().numpy(), w[:, idx.long()].cpu().numpy()
    return B.OwqLinear(Layer, layout=B.OWQ_LAYOUT_TILE)


def rms(x):
    return torch.nn.functional.rms_norm(x.float(), x.shape[-1:]).half()


class Decoder:
    def __init__(self, blocks=2, q_heads=8, kv_heads=2, dim=64, vocab=1000, page=64, pages=64, positions=2048, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.hq, self.hk, self.dim, self.vocab = q_heads, kv_heads, dim, vocab
        d = q_heads * dim
        self.embed = torch.randn(vocab, d, generator=g, device="cuda").half()
        self.head = low_bit(d, vocab, g)
        self.blocks = []
        for _ in range(blocks):
            self.blocks.append({
                "qkv": low_bit(d, (q_heads + 2 * kv_heads) * dim, g), "out": low_bit(d, d, g),
                "up": low_bit(d, 4 * d, g), "down": low_bit(4 * d, d, g),
                "wq": (1 + 0.1 * torch.randn(dim, generator=g, device="cuda")).half(),
                "wk": (1 + 0.1 * torch.randn(dim, generator=g, device="cuda")).half(),
                "cache": B.cache_empty(pages, page, kv_heads, dim)})
        angle = torch.arange(positions, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, device="cuda") / dim)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def forward(self, tokens, positions, table, starts, lengths, max_new, max_len):
        """tokens, positions [rows]: the new tokens of all sequences one after the other, sequence b's from starts[b] on;
        lengths: the sequences' tokens with these.  Returns the logits of every sequence's last token."""
        x = self.embed[tokens.long()]
        rows = x.shape[0]
        for b in self.blocks:
            qkv = b["qkv"](rms(x)).view(rows, self.hq + 2 * self.hk, self.dim)
            q, k = B.qk_norm_rope(qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hk], self.cos, self.sin, positions, b["wq"], b["wk"])
            B.cache_append(b["cache"], table, starts, lengths, k, qkv[:, self.hq + self.hk:], max_new=max_new)
            a = B.cache_attention(q, b["cache"], table, starts, lengths, max_new=max_new, max_len=max_len)
            x = x + b["out"](a.view(rows, -1))
            x = x + b["down"](torch.relu(b["up"](rms(x))))
        return self.head(rms(x[starts[1:].long() - 1]))


def int32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def generate(model, prompts, steps, temperature=0.8, top_k=40, top_p=0.95, page=64, seed=1):
    """Token lists, each prompt followed by `steps` sampled tokens."""
    g = torch.Generator("cuda").manual_seed(seed)
    n = len(prompts)
    per = [(len(p) + steps + page - 1) // page for p in prompts]
    table = torch.full((n, max(per)), -1, dtype=torch.int32)
    at = 0
    for b in range(n):                                   # a page is any page: hand them out in turn
        table[b, :per[b]] = torch.arange(at, at + per[b])
        at += per[b]
    table = table.cuda()
    out = [list(p) for p in prompts]
    tokens = int32([t for p in prompts for t in p])
    positions = int32([i for p in prompts for i in range(len(p))])
    lengths = [len(p) for p in prompts]
    starts = int32([sum(lengths[:b]) for b in range(n + 1)])
    t, k, p = torch.full((n,), temperature, device="cuda"), int32([top_k] * n), torch.full((n,), top_p, device="cuda")
    max_new = max(lengths)
    for _ in range(steps):
        logits = model.forward(tokens, positions, table, starts, int32(lengths), max_new, max(lengths))
        noise = torch.empty(n, model.vocab, device="cuda").exponential_(generator=g)
        tokens, _ = B.sample(logits, noise, t, k, p)
        for b, token in enumerate(tokens.tolist()):
            out[b].append(token)
        positions = int32(lengths)
        lengths = [m + 1 for m in lengths]
        starts, max_new = torch.arange(n + 1, dtype=torch.int32, device="cuda"), 1
    return out


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=16)
    for line in generate(Decoder(), [list(range(5, 45)), [7], list(range(100, 230))], parser.parse_args().steps):
        print(line)
