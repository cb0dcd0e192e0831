"""The operators between two low-bit layers, stated plainly in binary64 numpy: head norm with rotation and its
gradients, the 4-bit cache (quantiser, byte layout), attention over it, the choice of a token.  Independent of the
library; include/owq.h says what each computes."""
from __future__ import annotations

import math

import numpy as np


# ---- head norm and rotation -----------------------------------------------------------------------------------------

def _pair_index(rot, interleaved):
    j = np.arange(rot // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)


def norm_rope(x, w, cos, sin, positions, eps, interleaved):
    """x [tokens, heads, dim] -> the same, turned; a position outside the table makes the rotated part NaN."""
    y = np.asarray(x, np.float64).copy()
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    a, b = _pair_index(2 * cos.shape[1], interleaved)
    out = y.copy()
    for t, p in enumerate(positions):
        inside = 0 <= p < cos.shape[0]
        c = cos[p].astype(np.float64) if inside else np.full(cos.shape[1], np.nan)
        s = sin[p].astype(np.float64) if inside else np.full(cos.shape[1], np.nan)
        out[t][:, a] = y[t][:, a] * c - y[t][:, b] * s
        out[t][:, b] = y[t][:, b] * c + y[t][:, a] * s
    return out


def norm_rope_backward(dy, x, w, cos, sin, positions, eps, interleaved):
    """-> (dx, dw or None, sum of |terms| of dw or None)."""
    a, b = _pair_index(2 * cos.shape[1], interleaved)
    dy = np.asarray(dy, np.float64)
    g = dy.copy()
    for t, p in enumerate(positions):
        c, s = cos[p].astype(np.float64), sin[p].astype(np.float64)
        g[t][:, a] = dy[t][:, a] * c + dy[t][:, b] * s
        g[t][:, b] = dy[t][:, b] * c - dy[t][:, a] * s
    if w is None:
        return g, None, None
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = g * w
    dx = r * (h - x * r * r * (h * x).mean(-1, keepdims=True))
    terms = g * x * r
    return dx, terms.sum((0, 1)), np.abs(terms).sum((0, 1))


# ---- the 4-bit cache ------------------------------------------------------------------------------------------------

def quantise(x):
    """Rows (last axis) of fp16 or fp32 values -> (codes uint8, s fp16, lo fp16), every step one binary32 operation."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        hi, lo = x.max(-1), x.min(-1)
        step = np.clip((hi - lo) * np.float32(1.0 / 15.0), np.float32(2.0 ** -24), np.float32(65504)).astype(np.float16)
        low = np.clip(lo, np.float32(-65504), np.float32(65504)).astype(np.float16)
        q = np.rint((x - low.astype(np.float32)[..., None]) / step.astype(np.float32)[..., None])
        codes = np.clip(np.nan_to_num(q), 0, 15).astype(np.uint8)
    bad = ~np.isfinite(x).all(-1)
    step[bad] = low[bad] = np.uint16(0x7E00).view(np.float16)
    codes[bad] = 0
    return codes, step, low


def tile_bytes(dim):
    return 32 * (-(-dim // 32) * 32) + 256


def _word_places(dim):
    """For every code word of a tile's half (keys, values) the (token, column) of its eight elements."""
    steps = -(-dim // 32)
    S, q, r, h = np.meshgrid(np.arange(steps), np.arange(4), np.arange(16), np.arange(2), indexing="ij")
    e = np.arange(8)
    S, q, r, h = (v.reshape(-1, 1) for v in (S, q, r, h))
    keys = (16 * h + r + 0 * e, 32 * S + 8 * q + e)
    values = (16 * (e // 4) + 4 * q + e % 4 + 0 * S, 32 * S + 16 * h + r + 0 * e)
    return keys, values


SHIFTS = 4 * (np.arange(8) // 2 + 4 * (np.arange(8) % 2))


def put_tokens(tile, k, v, dim, tokens):
    """Write rows k, v [len(tokens), dim] of the given tokens into a tile's bytes (uint8 array), in place."""
    pad = -(-dim // 32) * 32
    words = tile[:32 * pad].view(np.uint32).reshape(2, -1)
    meta = tile[32 * pad:].view(np.float16).reshape(2, 32, 2)
    for half, x in enumerate((k, v)):
        codes, s, lo = quantise(x)
        full = np.zeros((32, pad), np.uint32)
        full[tokens, :dim] = codes
        mine = np.zeros(32, bool)
        mine[tokens] = True
        t, col = _word_places(dim)[half]
        mask = ((mine[t] * np.uint32(15)).astype(np.uint64) << SHIFTS.astype(np.uint64)).sum(-1).astype(np.uint32)
        new = (full[t, col].astype(np.uint64) << SHIFTS.astype(np.uint64)).sum(-1).astype(np.uint32)
        words[half] = (words[half] & ~mask) | (new & mask)
        meta[half, tokens, 0] = s
        meta[half, tokens, 1] = lo


def get_tile(tile, dim):
    """-> keys, values [32, dim] in binary64."""
    pad = -(-dim // 32) * 32
    words = tile[:32 * pad].view(np.uint32).reshape(2, -1)
    meta = tile[32 * pad:].view(np.float16).reshape(2, 32, 2).astype(np.float64)
    out = []
    for half in range(2):
        full = np.zeros((32, pad))
        t, col = _word_places(dim)[half]
        full[t, col] = (words[half][:, None] >> SHIFTS.astype(np.uint32)) & 15
        out.append(full[:, :dim] * meta[half, :, :1] + meta[half, :, 1:])
    return out


def append(pages, table, starts, lengths, k, v, dim):
    """pages uint8 [pages, heads, tiles, bytes], changed in place; k, v [rows, heads, dim]."""
    size = pages.shape[2] * 32
    for b in range(len(lengths)):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            t = lengths[b] - n + i
            if t < 0 or t // size >= table.shape[1] or not 0 <= table[b, t // size] < pages.shape[0]:
                continue
            for h in range(pages.shape[1]):
                put_tokens(pages[table[b, t // size], h, t % size // 32], k[starts[b] + i, h][None], v[starts[b] + i, h][None], dim, [t % 32])


def read(pages, table, n, dim):
    """Tokens 0..n-1 of a sequence with this row of the table -> (keys, values) [n, heads, dim]; no page: zeros, and which tokens
    lie on one."""
    size = pages.shape[2] * 32
    out = np.zeros((2, n, pages.shape[1], dim))
    there = np.zeros(n, bool)
    for t0 in range(0, n, 32):
        m = min(32, n - t0)
        if t0 // size >= len(table) or not 0 <= table[t0 // size] < pages.shape[0]:
            continue
        there[t0:t0 + m] = True
        for h in range(pages.shape[1]):
            with np.errstate(invalid="ignore"):
                k, v = get_tile(pages[table[t0 // size], h, t0 % size // 32], dim)
            out[0, t0:t0 + m, h], out[1, t0:t0 + m, h] = k[:m], v[:m]
    return out[0], out[1], there


def attention(q, pages, table, starts, lengths, scale, window=0, sinks=0):
    """-> (out, lse, bound): bound = the most that fp16 weights on values measured from code 8 may move a result, plus fp32's share."""
    rows, q_heads, dim = q.shape
    out = np.zeros((rows, q_heads, dim))
    lse = np.full((rows, q_heads), -np.inf)
    bound = np.zeros((rows, q_heads))
    group = q_heads // pages.shape[1]
    q = np.asarray(q, np.float64)
    for b in range(len(lengths)):
        n_new = starts[b + 1] - starts[b]
        k, v, there = read(pages, table[b], max(0, int(lengths[b])), dim)
        for i in range(n_new):
            pos = lengths[b] - n_new + i
            t = np.arange(len(there))
            seen = there & (t <= pos) & ((window == 0) | (t > pos - window) | (t < sinks))
            if not seen.any():
                continue
            for h in range(q_heads):
                kk, vv = k[seen, h // group], v[seen, h // group]
                y = scale * (kk @ q[starts[b] + i, h])
                with np.errstate(invalid="ignore"):
                    top = y.max()
                    p = np.exp(y - top)
                lse[starts[b] + i, h] = top + math.log(p.sum()) if np.isfinite(top) else np.nan
                out[starts[b] + i, h] = p / p.sum() @ vv
                spread = (vv.max(-1) - vv.min(-1)).max() if np.isfinite(vv).all() else np.nan
                bound[starts[b] + i, h] = 2.0 ** -11 * spread + (1e-5 + 4e-6 * np.abs(scale) * (np.abs(kk) @ np.abs(q[starts[b] + i, h])).max()) * np.abs(vv).max()
    return out, lse, bound


# ---- sampling -------------------------------------------------------------------------------------------------------

def sample_row(logits, noise, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """-> (token, log-probability)."""
    x = np.asarray(logits, np.float64)
    if np.isnan(x).any() or not np.isfinite(x.max()) or not 0 <= t < math.inf or 0 < t < 2.0 ** -126 or (t > 0 and noise is None):
        return -1, math.nan
    # beside the largest logit: at small temperatures the scaled logits themselves are so large that nothing can be added to them
    z = (x - x.max()) / (t if t > 0 else 1.0)
    total = math.log(np.exp(z).sum())
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    token = order[0]
    if t > 0:
        if 0 < top_k < len(order):
            order = order[:top_k]
        if top_p < 1:
            p = np.exp(z[order])
            keep = np.cumsum(p) - p < top_p * p.sum()
            keep[0] = True
            order = order[keep]
        if min_p > 0:
            keep = z[order] >= z[order[0]] + math.log(min_p)
            keep |= x[order] == x[order[0]]
            order = order[keep]
        with np.errstate(divide="ignore"):
            score = z[order] - np.log(np.asarray(noise, np.float64)[order])
        token = order[score == score.max()].min()
    return int(token), float(z[token] - total)
