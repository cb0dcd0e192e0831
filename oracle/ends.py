"""The operators at the ends of a block and of a tuning step, stated plainly in binary64 numpy: dropout from Philox bits,
residual sum and norms, log-probabilities of tokens, and the gradients.  Independent of the library; include/owq.h says what
each computes."""
from __future__ import annotations

import numpy as np

LOW = 0xffffffff


def philox(counter, key):
    """Philox 4x32, ten rounds: counter of four integers, key of two -> four integers below 2^32."""
    c, k = [int(v) & LOW for v in counter], [int(v) & LOW for v in key]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & LOW, (a >> 32) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return c


def bits16(seed, step, site, rows, width):
    """The 16 bits of every element of [rows, width]: philox() over whole arrays."""
    seed, step, site = int(seed) & (2 ** 64 - 1), int(step) & LOW, int(site) & LOW
    units = -(-width // 8)
    row, unit = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange(units, dtype=np.uint64), indexing="ij")
    c = [unit, row, np.full_like(unit, step), np.full_like(unit, site)]
    k = [seed & LOW, seed >> 32]
    low, half = np.uint64(LOW), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    out = np.empty((rows, units, 8), dtype=np.int64)
    for i in range(4):
        out[:, :, 2 * i] = c[i] & np.uint64(0xffff)
        out[:, :, 2 * i + 1] = c[i] >> np.uint64(16)
    return out.reshape(rows, -1)[:, :width]


def factor(rng, p, site, rows, width):
    """0 where an element is dropped, else what it is multiplied by."""
    t = int(np.rint(np.float32(p).astype(np.float64) * 65536))
    if t == 0:
        return np.ones((rows, width))
    return np.where(bits16(*rng, site, rows, width) >= t, 65536.0 / (65536 - t), 0.0)


def times(x, f):
    """x f, 0 where f is 0 whatever x holds."""
    return np.where(f == 0, 0.0, x * np.where(f == 0, 1.0, f))


def normalised(x, kind, eps):
    """(normalised rows, 1 / size)"""
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def norm(x, kind, w, b, eps):
    if kind is None:
        return x
    y = normalised(x, kind, eps)[0]
    y = y if w is None else y * w
    return y if b is None else y + b


def residual_norm(h, branch, gate, post, post_w, post_b, kind, w, b, h_scale, branch_scale, eps, drop=None):
    """-> (total, y or None); drop = factor() of the branch, or None."""
    total = h_scale * h
    if branch is not None:
        u = norm(branch, post, post_w, post_b, eps)
        u = u if drop is None else times(u, drop)
        total = total + branch_scale * (u if gate is None else gate * u)
    return total, None if kind is None else norm(total, kind, w, b, eps)


def _norm_back(g, x, kind, w, eps):
    """-> (gradient of x, terms of the weight's, terms of the bias's gradient)"""
    n, r = normalised(x, kind, eps)
    q = g if w is None else g * w
    d = q - n * (q * n).mean(-1, keepdims=True)
    if kind == "layer":
        d = d - q.mean(-1, keepdims=True)
    return r * d, g * n, g


def residual_norm_backward(dy, dtotal, total, branch, gate, post, post_w, post_b, kind, w, h_scale, branch_scale, eps, drop=None):
    """-> dict of dh, dbranch and, per token, the terms of the gradients that are summed over tokens: gate, post_w, post_b, w, b."""
    out = {}
    d = np.zeros_like(total) if dtotal is None else dtotal
    if kind is not None and dy is not None:
        dx, out["w"], out["b"] = _norm_back(dy, total, kind, w, eps)
        d = d + dx
    out["h"] = h_scale * d
    if branch is not None:
        e = branch_scale * d
        u = norm(branch, post, post_w, post_b, eps)
        out["gate"] = e * (u if drop is None else times(u, drop))
        v = e if gate is None else e * gate
        v = v if drop is None else times(v, drop)
        out["branch"] = v
        if post is not None:
            out["branch"], out["post_w"], out["post_b"] = _norm_back(v, branch, post, post_w, eps)
    return out


def token_logprobs(logits, targets, scale, top):
    """-> dict: logprob, entropy, stats [3, rows], top_token, top_logprob; spread [rows], the mean of |z - max z| under the softmax."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    with np.errstate(all="ignore"):
        m = x.max(-1)
        good = np.isfinite(m) & ~np.isnan(x).any(-1)
        d = np.where(good[:, None], scale * (x - np.where(good, m, 0.0)[:, None]), np.nan)
        e = np.exp(d)
        s = e.sum(-1)
        p = e / s[:, None]
        pd = np.where(p > 0, p * np.where(p > 0, d, 0.0), 0.0 * p)
        log_s = np.log(s)
        out = {"stats": np.stack((np.where(good, m, np.nan), log_s, log_s - pd.sum(-1))), "spread": -pd.sum(-1),
               "spread2": np.where(p > 0, p * np.where(p > 0, d, 0.0) ** 2, 0.0).sum(-1)}
        out["entropy"] = out["stats"][2]
        if targets is not None:
            inside = (targets >= 0) & (targets < vocab)
            out["logprob"] = np.where(inside, d[np.arange(rows), np.where(inside, targets, 0)] - log_s, 0.0)
        out["top_token"] = np.full((rows, top), -1)
        out["top_logprob"] = np.full((rows, top), -np.inf)
        for r in range(rows):
            if not good[r]:
                out["top_logprob"][r] = np.nan
                continue
            order = np.argsort(-x[r], kind="stable")[:top]
            order = order[x[r][order] > -np.inf]
            out["top_token"][r, :len(order)] = order
            out["top_logprob"][r, :len(order)] = d[r][order] - log_s[r]
    return out


def token_logprobs_backward(dlogprob, dentropy, logits, targets, scale):
    """-> (dlogits, their size: what they are the sum of)"""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    zero = np.zeros(rows)
    inside = np.zeros(rows, bool) if targets is None else (targets >= 0) & (targets < vocab)
    a = np.where(inside, zero if dlogprob is None else dlogprob, 0.0)
    h = zero if dentropy is None else dentropy
    with np.errstate(all="ignore"):
        got = token_logprobs(x, None, scale, 0)
        l = scale * (x - got["stats"][0][:, None]) - got["stats"][1][:, None]
        p = np.exp(l)
        pl = np.where(p == 0, 0.0, p * l)
        d = -a[:, None] * p - h[:, None] * (pl + p * got["entropy"][:, None])
        size = np.abs(a)[:, None] * p + np.abs(h)[:, None] * (np.abs(pl) + p * got["entropy"][:, None])
    at = np.arange(rows)[inside]
    d[at, targets[inside] if targets is not None else at] += a[inside]
    none = (a == 0) & (h == 0)
    d[none], size[none] = 0.0, 0.0
    return scale * d, scale * size
