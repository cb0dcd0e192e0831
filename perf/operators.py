"""The operators between two low-bit linear layers of a decoder, as cases that can be timed and compared.

  path "rope"      norm of every query and key head and the position rotation, one pass
  path "rope_bwd"  its gradients: of the queries, the keys and the two norm weights
  path "append"    new keys and values into the 4-bit cache, and the cache's contents read back as fp16
  path "attend"    attention of new queries over the 4-bit cache: single tokens, several per sequence, whole prompts
  path "sample"    from logits and given exponential variates to token indices and log-probabilities

`run` computes them from elementary torch operations in 32 bits, or, where `own` is true, by the library's calls.

The cache is a tensor of bytes [pages, key/value heads, page tokens / 32, 32 P + 256], P = the head size rounded up to
32: for 32 tokens of one head first the keys' codes, then the values', then 32 keys' and 32 values' (step size, least
value) pairs in fp16.  The codes lie as matrix-core operands: keys [P/32][4][16][2] words, word (s, q, r, h) = key
16 h + r at columns 32 s + 8 q + e; values [P/32][4][16][2] words, word (s, q, r, j) = column 32 s + 16 j + r of keys
16 (e / 4) + 4 q + e % 4; e = 0..7 sits at nibble e / 2 + 4 (e % 2) of its word.
"""
from __future__ import annotations

import math

import torch

own = False

GOLDEN = 0.6180339887498949
NIBBLE_OF = [0, 4, 1, 5, 2, 6, 3, 7]          # where element e of a word sits
ELEMENT_AT = [0, 2, 4, 6, 1, 3, 5, 7]         # and the element at nibble n


def _rope(tokens, q_heads, kv_heads, dim, rotary, norm=True, interleaved=False, dtype="float16", path="rope"):
    return {"path": path, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary,
            "norm": norm, "interleaved": interleaved, "dtype": dtype}


def _append(seqs, new, shortest, longest, kv_heads, dim, page, dtype="float16"):
    return {"path": "append", "seqs": seqs, "new": new, "shortest": shortest, "longest": longest, "kv_heads": kv_heads,
            "dim": dim, "page": page, "dtype": dtype}


def _attend(seqs, new, shortest, longest, q_heads, kv_heads, dim, page, window=0, sinks=0, dtype="float16"):
    return {"path": "attend", "seqs": seqs, "new": new, "shortest": shortest, "longest": longest, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "window": window, "sinks": sinks, "dtype": dtype}


def _sample(rows, vocab, top_k, top_p, min_p, temperature, dtype="float16"):
    return {"path": "sample", "rows": rows, "vocab": vocab, "top_k": top_k, "top_p": top_p, "min_p": min_p,
            "temperature": temperature, "dtype": dtype}


def listed():
    return [
        # one token of a decoder with 40 heads of 128: what a call costs at least
        dict(_rope(1, 40, 40, 128, 128, norm=False), name="rope_token"),
        # a prompt's chunk of 4096 tokens, 32 query heads on 8 key heads, heads normalised
        dict(_rope(4096, 32, 8, 128, 128), name="rope_prompt"),
        # the gradients for a training batch of 2048 tokens with 72 heads
        dict(_rope(2048, 72, 72, 128, 128, path="rope_bwd"), name="rope_backward"),
        # bfloat16, part of an 80-wide head rotated by neighbours, a number of tokens that divides by nothing
        dict(_rope(1021, 32, 32, 80, 32, interleaved=True, dtype="bfloat16", path="rope_bwd"), name="rope_backward_part"),
        # 64 requests, a token each, on short contexts
        dict(_append(64, 1, 1, 90, 8, 128, 64), name="append_tokens"),
        # four prompts of uneven lengths, 40 heads
        dict(_append(4, 2500, 900, 2500, 40, 128, 128), name="append_prompts"),
        # a single request of one token, every head with keys of its own
        dict(_attend(1, 1, 4001, 4001, 40, 40, 128, 128), name="attend_token"),
        # 64 requests decoded together on contexts up to 8192 tokens, four query heads to a key head
        dict(_attend(64, 1, 300, 8192, 32, 8, 128, 64), name="attend_batch"),
        # window of 1024 with 4 first tokens kept, long contexts, three drafted tokens per request, bfloat16 heads of 64
        dict(_attend(16, 3, 2000, 30000, 32, 32, 64, 256, window=1024, sinks=4, dtype="bfloat16"), name="attend_window"),
        # 2048 more tokens of a prompt of which 4100 are in the cache
        dict(_attend(1, 2048, 6148, 6148, 32, 8, 128, 128), name="attend_prompt"),
        # one request's next token from 32000 logits
        dict(_sample(1, 32000, 50, 0.95, 0.0, 0.8), name="sample_token"),
        # 256 requests over the larger vocabulary, float32 logits, wide nucleus
        dict(_sample(256, 50272, 0, 0.9, 0.02, 1.0, dtype="float32"), name="sample_batch"),
    ]


def _log_int(rng, lo, hi):
    n = int(round(lo * (hi / lo) ** rng.random()))
    return n + 1 if n == 3072 else n


HEADS = ((32, 32), (32, 8), (40, 40), (12, 12), (64, 8), (8, 1), (72, 72), (28, 4), (5, 5))


def draw(rng):
    path = rng.choice(("rope", "rope_bwd", "append", "attend", "attend", "attend", "sample", "sample"))
    q_heads, kv_heads = rng.choice(HEADS)
    dtype = rng.choice(("float16", "float16", "bfloat16"))
    if path in ("rope", "rope_bwd"):
        dim = rng.choice((64, 80, 96, 128, 128, 256))
        tokens = _log_int(rng, 1, max(2, min(8192, (2048 * 144 * 128) // (2 * (q_heads + kv_heads) * dim))))
        rotary = dim if rng.random() < 0.6 else dim // 32 * 16
        return _rope(tokens, q_heads, kv_heads, dim, rotary, rng.random() < 0.7, rng.random() < 0.3, dtype, path)
    dim = rng.choice((64, 64, 80, 96, 128, 128, 128))
    page = rng.choice((32, 64, 128, 256))
    if path == "append":
        longest = _log_int(rng, 40, 2500)
        seqs = _log_int(rng, 1, max(1, min(64, 300000 // (longest * kv_heads))))
        new = rng.choice((1, 1, 2, 7, longest))
        return _append(seqs, new, max(1, longest // rng.choice((1, 2, 9))), longest, kv_heads, dim, page, dtype)
    if path == "attend":
        kind = rng.choice(("one", "batch", "batch", "prompt"))
        window, sinks = rng.choice(((0, 0), (0, 0), (513, 4), (2000, 0)))
        if kind == "prompt":
            new = _log_int(rng, 40, 2048)
            longest = new + _log_int(rng, 1, 3000)
            return _attend(1 if new > 500 else 3, new, longest - new // 3, longest, min(q_heads, 32), min(kv_heads, 32) if q_heads <= 32 else 8, dim, page, window, sinks, dtype)
        longest = _log_int(rng, 20, 30000)
        seqs = 1 if kind == "one" else max(1, min(64, _log_int(rng, 2, 64), 1500000 // (longest * kv_heads)))
        return _attend(seqs, rng.choice((1, 1, 1, 2, 4)), max(4, longest // rng.choice((1, 3, 20))), longest, q_heads, kv_heads, dim, page, window, sinks, dtype)
    return _sample(_log_int(rng, 1, 256), rng.choice((32000, 50272, _log_int(rng, 300, 50000))), rng.choice((0, 0, 1, 20, 50, 1000)),
                   rng.choice((1.0, 0.95, 0.9, 0.5)), rng.choice((0.0, 0.0, 0.05)), rng.choice((0.0, 0.7, 1.0, 1.3)),
                   rng.choice(("float16", "bfloat16", "float32")))


def _dtype(case):
    return getattr(torch, case["dtype"])


def _lengths(case):
    """Tokens of every sequence, new ones among them: spread over the case's range, the first the longest."""
    lo, hi = case["shortest"], case["longest"]
    return [hi - int((hi - lo) * ((b * GOLDEN) % 1.0)) for b in range(case["seqs"])]


def _news(case):
    return [min(case["new"], n) for n in _lengths(case)]


def _padded(dim):
    return (dim + 31) // 32 * 32


def work(case):
    path = case["path"]
    if path in ("rope", "rope_bwd"):
        n = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        table = case["tokens"] * (4 * case["rotary"] + 4)
        passes = 2 if path == "rope" else 3 if case["norm"] else 2
        return {"bytes": 2 * passes * n + table, "flops": (8 if path == "rope" else 16) * n}
    if path == "append":
        row = case["kv_heads"] * (case["dim"] + 8)
        new, whole = sum(_news(case)), sum(_lengths(case))
        values = case["kv_heads"] * case["dim"] * 4
        return {"bytes": new * (values + row) + whole * (row + values), "flops": 8 * new * case["kv_heads"] * case["dim"]}
    if path == "attend":
        window, sinks = case["window"], case["sinks"]
        read = pairs = 0
        for n, m in zip(_lengths(case), _news(case)):
            first = n - m
            low = max(0, first - window + 1) if window else 0
            read += n - low + min(low, sinks)
            for p in range(first, n):
                at = max(0, p - window + 1) if window else 0
                pairs += p + 1 - at + min(at, sinks)
        tokens = sum(_news(case))
        return {"bytes": read * case["kv_heads"] * (case["dim"] + 8) + 4 * tokens * case["q_heads"] * case["dim"],
                "flops": 4 * pairs * case["q_heads"] * case["dim"]}
    size = 4 if case["dtype"] == "float32" else 2
    kept = case["top_k"] if case["top_k"] else case["vocab"]
    if case["temperature"] == 0.0:
        kept = 0
    return {"bytes": case["rows"] * (case["vocab"] * size + min(kept, case["vocab"]) * 4 + 8), "flops": 10 * case["rows"] * case["vocab"]}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _quantise(x):
    """Rows of x (last axis) to codes, step size and least value, each step one binary32 operation."""
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = ((high - low) * (1.0 / 15.0)).clamp(2.0 ** -24, 65504.0).half()
    low = low.clamp(-65504.0, 65504.0).half()
    codes = ((x - low.float()) / step.float()).round().clamp(0, 15).to(torch.uint8)
    return codes, step.squeeze(-1), low.squeeze(-1)


def _to_bytes(words):
    """[..., 8] codes in element order to the 4 bytes of their word."""
    n = words[..., torch.tensor(ELEMENT_AT, device=words.device)]
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _pages_of(k, v, tokens_per_page):
    """Keys and values [tokens (whole pages), heads, dim] to cache pages."""
    t, heads, dim = k.shape
    pad = _padded(dim)
    steps, tiles = pad // 32, t // 32
    parts = []
    for x, axes in ((k, "k"), (v, "v")):
        codes, step, low = _quantise(x)
        codes = torch.nn.functional.pad(codes, (0, pad - dim))
        if axes == "k":       # tile, h, r, head, s, q, e
            c = codes.view(tiles, 2, 16, heads, steps, 4, 8).permute(0, 3, 4, 5, 2, 1, 6)
        else:                 # tile, e / 4, q, e % 4, head, s, j, r
            c = codes.view(tiles, 2, 4, 4, heads, steps, 2, 16).permute(0, 4, 5, 2, 7, 6, 1, 3).reshape(tiles, heads, steps, 4, 16, 2, 8)
        meta = torch.stack((step, low), -1).view(tiles, 32, heads, 2).permute(0, 2, 1, 3).contiguous()
        parts.append((_to_bytes(c).reshape(tiles, heads, -1), meta.view(torch.uint8).reshape(tiles, heads, -1)))
    tile = torch.cat((parts[0][0], parts[1][0], parts[0][1], parts[1][1]), -1)
    per = tokens_per_page // 32
    return tile.view(t // tokens_per_page, per, heads, -1).permute(0, 2, 1, 3).contiguous()


def _cache(case, g, device, lengths):
    """Pages with every sequence's tokens in them, handed out in no order, and the table of their indices."""
    page, heads, dim = case["page"], case["kv_heads"], case["dim"]
    per = [(n + page - 1) // page for n in lengths]
    total = sum(per)
    k = torch.randn(total * page, heads, dim, generator=g, device=device)
    k *= torch.where(torch.rand(heads, dim, generator=g, device=device) < 0.03, 5.0, 1.0)     # keys have columns of large values
    v = torch.randn(total * page, heads, dim, generator=g, device=device)
    order = torch.randperm(total, generator=g, device=device)
    pages = torch.empty_like(made := _pages_of(k.half(), v.half(), page))
    pages[order] = made
    table = torch.full((len(lengths), max(per)), -1, dtype=torch.int32)
    at, where = 0, order.to("cpu", torch.int32)
    for b, n in enumerate(per):
        table[b, :n] = where[at:at + n]
        at += n
    return pages, table.to(device)


def _offsets(counts, device):
    return torch.tensor([0] + counts, dtype=torch.int64).cumsum(0).to(device, torch.int32)


def prepare(case, seed):
    device = torch.device("cuda")
    g = torch.Generator(device).manual_seed(seed)
    path, dtype = case["path"], None if case["path"] == "sample" else _dtype(case)
    s = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=device)

    if path in ("rope", "rope_bwd"):
        t, hq, hk, d, rot = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"], case["rotary"]
        qkv = normal(t, hq + 2 * hk, d).to(dtype)          # what a fused projection leaves: queries, keys, values of a token in a row
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        angle = torch.arange(t + 100, device=device, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=device, dtype=torch.float64) / rot)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["positions"] = torch.arange(t, device=device, dtype=torch.int32) + int(seed % 100)
        s["wq"], s["wk"] = ((1 + 0.2 * normal(d)).to(dtype), (1 + 0.2 * normal(d)).to(dtype)) if case["norm"] else (None, None)
        if path == "rope_bwd":
            s["dq"], s["dk"] = (0.05 * normal(t, hq, d)).to(dtype), (0.05 * normal(t, hk, d)).to(dtype)
    elif path in ("append", "attend"):
        lengths, news = _lengths(case), _news(case)
        s["pages"], s["table"] = _cache(case, g, device, lengths)
        s["starts"] = _offsets(news, device)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=device)
        s["max_new"], s["max_len"], s["total"] = max(news), max(lengths), sum(lengths)
        if path == "append":
            qkv = normal(sum(news), 2 * case["kv_heads"], case["dim"]).to(dtype)
            s["k"], s["v"] = qkv[:, :case["kv_heads"]], qkv[:, case["kv_heads"]:]
            s["rows"] = _offsets(lengths, device)
        else:
            s["q"] = normal(sum(news), case["q_heads"], case["dim"]).to(dtype)
    else:
        r, n = case["rows"], case["vocab"]
        dtype = _dtype(case)
        # a few likely tokens above a broad rest, as a trained model's logits are
        s["logits"] = (normal(r, n) * 2 + 9 * torch.rand(r, n, generator=g, device=device) ** 40).to(dtype)
        s["noise"] = torch.empty(r, n, device=device).exponential_(generator=g)
        s["temperature"] = torch.full((r,), case["temperature"], device=device)
        s["top_k"] = torch.full((r,), case["top_k"], dtype=torch.int32, device=device) if case["top_k"] else None
        s["top_p"] = torch.full((r,), case["top_p"], device=device) if case["top_p"] < 1.0 else None
        s["min_p"] = torch.full((r,), case["min_p"], device=device) if case["min_p"] > 0.0 else None
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _pairs(x, rot, interleaved):
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2]
    return x[..., :rot // 2], x[..., rot // 2:rot]


def _joined(a, b, x, rot, interleaved):
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _turn(x, cos, sin, rot, interleaved):
    a, b = _pairs(x, rot, interleaved)
    return _joined(a * cos - b * sin, b * cos + a * sin, x, rot, interleaved)


EPS = 1e-6


def _rope_plain(s):
    case = s["case"]
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        return _turn(y, cos, sin, case["rotary"], case["interleaved"]).to(x.dtype)
    return one(s["q"], s["wq"]), one(s["k"], s["wk"])


def _rope_bwd_plain(s):
    case = s["case"]
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]

    def one(dy, x, w):
        g = _turn(dy.float(), cos, -sin, case["rotary"], case["interleaved"])
        if w is None:
            return g.to(x.dtype), None
        y = x.float()
        r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        h = g * w.float()
        dx = r * (h - y * (r * r) * (h * y).mean(-1, keepdim=True))
        return dx.to(x.dtype), (g * y * r).sum((0, 1))
    (dq, dwq), (dk, dwk) = one(s["dq"], s["q"], s["wq"]), one(s["dk"], s["k"], s["wk"])
    return [t for t in (dq, dk, dwq, dwk) if t is not None]


def _unpacked(tiles, dim):
    """Cache tiles [..., 32 P + 256] bytes to keys and values [..., 32, dim] in 32 bits."""
    pad = _padded(dim)
    lead, steps = tiles.shape[:-1], pad // 32
    where = torch.tensor(NIBBLE_OF, device=tiles.device)

    def codes(b):
        n = torch.stack((b & 15, b >> 4), -1).flatten(-2)           # nibbles of 4-byte words
        return n.view(-1, steps, 4, 16, 2, 8)[..., where]
    k = codes(tiles[..., :16 * pad]).permute(0, 4, 3, 1, 2, 5).reshape(*lead, 32, pad)
    v = codes(tiles[..., 16 * pad:32 * pad]).reshape(-1, steps, 4, 16, 2, 2, 4).permute(0, 5, 2, 6, 1, 4, 3).reshape(*lead, 32, pad)
    meta = tiles[..., 32 * pad:].contiguous().view(torch.float16).float().view(*lead, 2, 32, 2, 1)
    return (meta[..., 0, :, 0, :] * k[..., :dim] + meta[..., 0, :, 1, :], meta[..., 1, :, 0, :] * v[..., :dim] + meta[..., 1, :, 1, :])


def _contents(s):
    """Keys and values of every sequence, padded to the longest: [sequences, tokens, heads, dim] in 32 bits."""
    case = s["case"]
    got = s["pages"][s["table"].clamp(min=0).long()]                # sequence, page, head, tile, bytes
    k, v = _unpacked(got, case["dim"])
    return [x.permute(0, 1, 3, 4, 2, 5).flatten(1, 3) for x in (k, v)]


def _append_plain(s):
    case = s["case"]
    old_k, old_v = _contents(s)
    lengths, starts = s["lengths"].long(), s["starts"].long()
    at = torch.arange(s["total"], device=lengths.device)
    seq = torch.searchsorted(s["rows"].long(), at, right=True) - 1
    place = at - s["rows"].long()[seq]
    new = starts[seq] + place - (lengths[seq] - (starts[seq + 1] - starts[seq]))       # row of the new token, below starts[seq] for old ones
    out = []
    for x, old in ((s["k"], old_k), (s["v"], old_v)):
        codes, step, low = _quantise(x)
        value = step.float()[..., None] * codes.float() + low.float()[..., None]
        is_new = new >= starts[seq]
        out.append(torch.where(is_new[:, None, None], value[new.clamp(min=0)], old[seq, place]).half())
    return out


def _attend_plain(s):
    case = s["case"]
    k, v = _contents(s)
    b, n, hk, d = k.shape
    hq, m = case["q_heads"], s["max_new"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    step = torch.arange(m, device=k.device)
    row = (starts[:-1, None] + step).clamp(max=starts[-1] - 1)
    q = s["q"][row].float().view(b, m, hk, hq // hk, d).permute(0, 2, 1, 3, 4).reshape(b, hk, m * (hq // hk), d)
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).view(b, hk, m, hq // hk, n) * d ** -0.5
    pos = (lengths - (starts[1:] - starts[:-1]))[:, None] + step                          # [b, m]
    key = torch.arange(n, device=k.device)
    seen = key <= pos[..., None]
    if case["window"]:
        seen &= (key > pos[..., None] - case["window"]) | (key < case["sinks"])
    x = x.masked_fill(~seen[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v.permute(0, 2, 1, 3).contiguous()).view(b, hk, m, hq // hk, d)
    o = torch.where(total > 0, o / total, torch.zeros((), device=k.device))
    o = o.permute(0, 2, 1, 3, 4).reshape(b, m, hq, d)
    tokens = torch.arange(s["q"].shape[0], device=k.device)
    seq = torch.searchsorted(starts, tokens, right=True) - 1
    return o[seq, tokens - starts[seq]].to(s["q"].dtype)


def _sample_plain(s):
    x = s["logits"].float()
    t = s["temperature"][:, None]
    z = x / torch.where(t > 0, t, torch.ones_like(t))
    total = torch.logsumexp(z, -1)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    z_sorted = z.gather(1, order)
    rank = torch.arange(z.shape[1], device=z.device)
    keep = torch.ones_like(z, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= rank < s["top_k"][:, None]
    if s["top_p"] is not None:
        mass = torch.exp(z_sorted - z_sorted[:, :1]) * keep
        before = mass.cumsum(-1) - mass
        keep &= before < s["top_p"][:, None] * mass.sum(-1, keepdim=True)
    if s["min_p"] is not None:
        keep &= z_sorted >= z_sorted[:, :1] + torch.log(s["min_p"])[:, None]
    key = torch.where(keep, z_sorted - torch.log(s["noise"].gather(1, order)), -math.inf)
    token = order.gather(1, torch.where(t > 0, key.argmax(-1, keepdim=True), 0))
    return token[:, 0].int(), z.gather(1, token)[:, 0] - total


def run(s):
    case = s["case"]
    path = case["path"]
    if own:
        from paper_2306_02272_amd import binding as B
        if path == "rope":
            return B.qk_norm_rope(s["q"], s["k"], s["cos"], s["sin"], s["positions"], s["wq"], s["wk"], EPS, case["interleaved"])
        if path == "rope_bwd":
            got = B.qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["cos"], s["sin"], s["positions"], s["wq"], s["wk"], EPS,
                                          case["interleaved"])
            return [t for t in got if t is not None]
        if path == "append":
            B.cache_append(s["pages"], s["table"], s["starts"], s["lengths"], s["k"], s["v"], max_new=s["max_new"])
            return B.cache_read(s["pages"], s["table"], s["rows"], s["total"], case["dim"], max_len=s["max_len"])
        if path == "attend":
            return B.cache_attention(s["q"], s["pages"], s["table"], s["starts"], s["lengths"], window=case["window"], sinks=case["sinks"],
                                   max_new=s["max_new"], max_len=s["max_len"])
        return B.sample(s["logits"], s["noise"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    return {"rope": _rope_plain, "rope_bwd": _rope_bwd_plain, "append": _append_plain, "attend": _attend_plain,
            "sample": _sample_plain}[path](s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_head(x, w, cos, sin, rot, interleaved):
    y = x.double()
    if w is not None:
        y = y / (y.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    out = y.clone()
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, n = cos[:, None, j].double(), sin[:, None, j].double()
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * n, y[..., b] * c + y[..., a] * n
    return out


def _exact_sequence(pages, table, n, dim):
    """Keys and values [n, heads, dim] of one sequence, from the words of its pages."""
    pad = _padded(dim)
    got = pages[table[:(n + pages.shape[2] * 32 - 1) // (pages.shape[2] * 32)].long()]
    tiles = got.transpose(1, 2).flatten(0, 1)                       # tile, head, bytes
    words = tiles[..., :32 * pad].contiguous().view(torch.int32).long() & 0xffffffff
    meta = tiles[..., 32 * pad:].contiguous().view(torch.float16).double().view(*tiles.shape[:2], 2, 32, 2)
    k = torch.zeros(*tiles.shape[:2], 32, pad, dtype=torch.float64, device=pages.device)
    v = torch.zeros_like(k)
    half = words.shape[-1] // 2
    index = torch.arange(half, device=pages.device)
    second, r, q, s = index % 2, index // 2 % 16, index // 32 % 4, index // 128
    for e in range(8):
        shift = 4 * (e // 2 + 4 * (e % 2))
        code = (words >> shift & 15).double()
        k[:, :, 16 * second + r, 32 * s + 8 * q + e] = code[..., :half]
        v[:, :, 16 * (e // 4) + 4 * q + e % 4, 32 * s + 16 * second + r] = code[..., half:]
    out = []
    for x, m in ((k, meta[:, :, 0]), (v, meta[:, :, 1])):
        x = x * m[..., :1] + m[..., 1:]
        out.append(x.transpose(1, 2).flatten(0, 1)[:n, :, :dim])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path in ("rope", "rope_bwd"):
        at = s["positions"].long()
        cos, sin = s["cos"][at], s["sin"][at]
        rot, inter = case["rotary"], case["interleaved"]
        if path == "rope":
            return tuple(_exact_head(s[n], s["w" + n], cos, sin, rot, inter) for n in "qk")
        grads = []
        for n in "qk":                      # by differentiation of the definition
            x = s[n].double().requires_grad_(True)
            w = s["w" + n].double().requires_grad_(True) if case["norm"] else None
            y = x if w is None else x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
            a, b = _pairs(y, rot, inter)
            c, d = cos[:, None].double(), sin[:, None].double()
            (_joined(a * c - b * d, b * c + a * d, y, rot, inter) * s["d" + n].double()).sum().backward()
            grads.append((x.grad, None if w is None else w.grad))
        return [t for t in (grads[0][0], grads[1][0], grads[0][1], grads[1][1]) if t is not None]
    if path == "append":
        out = ([], [])
        for b, (n, m) in enumerate(zip(_lengths(case), _news(case))):
            old = _exact_sequence(s["pages"], s["table"][b], n, case["dim"])
            at = int(s["starts"][b])
            for o, x, dst in zip(old, (s["k"], s["v"]), out):
                x = x[at:at + m].double()
                low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
                step, low = ((high - low) / 15).clamp(2.0 ** -24, 65504.0).half().double(), low.clamp(-65504.0, 65504.0).half().double()
                o[n - m:] = torch.round((x - low) / step).clamp(0, 15) * step + low
                dst.append(o)
        return [torch.cat(o) for o in out]
    if path == "attend":
        out = []
        group = case["q_heads"] // case["kv_heads"]
        for b, (n, m) in enumerate(zip(_lengths(case), _news(case))):
            k, v = _exact_sequence(s["pages"], s["table"][b], n, case["dim"])
            at = int(s["starts"][b])
            q = s["q"][at:at + m].double()
            pos, key = torch.arange(n - m, n, device=q.device)[:, None], torch.arange(n, device=q.device)
            seen = key <= pos
            if case["window"]:
                seen = seen & ((key + case["window"] > pos) | (key < case["sinks"]))
            o = torch.empty_like(q)
            for h in range(case["q_heads"]):
                x = q[:, h] @ k[:, h // group].t() / math.sqrt(case["dim"])
                o[:, h] = torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ v[:, h // group]
            out.append(o)
        return torch.cat(out)
    x = s["logits"].double().cpu()
    t = float(torch.tensor(case["temperature"], dtype=torch.float32))
    z = x / t if t > 0 else x
    noise = s["noise"].double().cpu()
    tokens = []
    for r in range(case["rows"]):
        order = torch.argsort(x[r], descending=True, stable=True)
        if t == 0:
            tokens.append(int(order[0]))
            continue
        if case["top_k"]:
            order = order[:case["top_k"]]
        p = torch.softmax(z[r][order], -1)
        if case["top_p"] < 1.0:
            order = order[torch.cumsum(p, 0) - p < float(torch.tensor(case["top_p"], dtype=torch.float32))]
        if case["min_p"] > 0.0:
            order = order[z[r][order] >= z[r][order[0]] + math.log(float(torch.tensor(case["min_p"], dtype=torch.float32)))]
        tokens.append(int(order[torch.argmax(z[r][order] - torch.log(noise[r][order]))]))
    token = torch.tensor(tokens, dtype=torch.int32)
    return token, z.gather(1, token.long()[:, None])[:, 0] - torch.logsumexp(z, -1)
