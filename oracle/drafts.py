"""Plain references of a step of drafted tokens, numpy on the host in 64 bits: the linear layer with a step per group, norm and rotation
of heads, attention of a tree over the cache of quantized pages, log probabilities.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def nibbles(packed):
    """Codes int64 [N, K] of two's-complement nibbles uint8 [N, K / 2]."""
    p = packed.astype(np.int64)
    both = np.stack([p & 15, p >> 4], -1).reshape(p.shape[0], -1)
    return np.where(both > 7, both - 16, both)


def linear_groups(x, codes, steps, group):
    """x [M, K], codes [N, K], steps [N, K / group], in float64."""
    w = codes.astype(np.float64) * np.repeat(steps.astype(np.float64), group, 1)
    return x.astype(np.float64) @ w.T


def gelu(y):
    from scipy.special import ndtr
    return y * ndtr(y)


def rotate_heads(x, positions, frequencies, weight, eps, neighbours):
    """(output, per pair of channels the largest |a| + |b| before the rotation, spread over the channels): x [rows, heads, dim]."""
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * weight.astype(np.float64)
    out, size = y.copy(), np.abs(y)
    n = len(frequencies)
    if n:
        t = positions.astype(np.float64)[:, None] * frequencies.astype(np.float64)
        t = np.remainder(t, 2 * np.pi)[:, None]
        i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if neighbours else (slice(0, n), slice(n, 2 * n))
        a, b = y[..., i], y[..., j]
        out[..., i], out[..., j] = a * np.cos(t) - b * np.sin(t), b * np.cos(t) + a * np.sin(t)
        size[..., i] = size[..., j] = np.abs(a) + np.abs(b)
    return out, size


def attention_tree(cache, starts, kv_len, table, q, seen, scale):
    """As serving.Cache.attention, whose last two results it has too, with another mask: seen[row] is a Python integer, whose bit j says
    whether the row sees its sequence's row j."""
    rows, heads, dim = q.shape
    kh = cache.codes["k"].shape[1]
    qmax = 2.0 ** (cache.bits - 1) - 1
    out = np.zeros((rows, heads, dim))
    logit, big = np.zeros((rows, heads)), np.zeros((rows, heads))
    for s in range(len(kv_len)):
        length = min(int(kv_len[s]), cache.page * table.shape[1])
        n = int(starts[s + 1] - starts[s])
        held = int(kv_len[s]) - n
        places = [cache._place(table[s], p) for p in range(length)]
        there = np.array([p is not None for p in places], bool)
        on = np.array([p[0] if p else 0 for p in places], int)
        at = np.array([p[1] if p else 0 for p in places], int)
        if length:
            k = cache.codes["k"][on, :, at].astype(np.float64) * (cache.absmax["k"][on].astype(np.float64) / qmax)[..., None]
            v = cache.codes["v"][on, :, at].astype(np.float64) * (cache.absmax["v"][on].astype(np.float64) / qmax)[..., None]
        for i in range(n):
            row = int(starts[s]) + i
            see = there & np.array([j < held or bool(seen[row] >> (j - held) & 1) for j in range(length)], bool)
            if not see.any():
                continue
            for h in range(heads):
                kk, vv = k[see, h * kh // heads], v[see, h * kh // heads]
                x = kk @ q[row, h].astype(np.float64) * scale
                e = np.exp(x - x.max())
                out[row, h] = (e / e.sum()) @ vv
                logit[row, h] = (np.abs(kk) @ np.abs(q[row, h].astype(np.float64))).max() * abs(scale)
                big[row, h] = np.abs(vv).max()
    return out, logit, big


def token_logprobs(x, tokens, top, scale):
    """(logprob, entropy, top_logprob, top_index, spread, bend): x [rows, vocab] with finite maxima.  With d = scale (x - max) and p the
    probabilities, spread = sum p |d| and bend = sum p d^2 / sum p |d|, of which a test forms its bounds."""
    rows, vocab = x.shape
    d = (x.astype(np.float64) - x.astype(np.float64).max(1, keepdims=True)) * np.float64(np.float32(scale))
    e = np.exp(d)
    total = e.sum(1)
    log_total = np.log(total)
    p = e / total[:, None]
    finite = np.where(p > 0, d, 0.0)
    spread = (p * -finite).sum(1)
    bend = (p * finite * finite).sum(1) / np.where(spread > 0, spread, 1.0)
    entropy = log_total + spread
    logprob = np.full(rows, -np.inf)
    ok = (tokens >= 0) & (tokens < vocab)
    logprob[ok] = d[ok, tokens[ok]] - log_total[ok]
    order = np.argsort(-x.astype(np.float64), axis=1, kind="stable")[:, :top]
    best = np.full((rows, top), -np.inf)
    index = np.full((rows, top), -1)
    n = order.shape[1]
    best[:, :n] = np.take_along_axis(d, order, 1) - log_total[:, None]
    index[:, :n] = np.where(np.isneginf(best[:, :n]), -1, order)
    return logprob, entropy, best, index, spread, bend
