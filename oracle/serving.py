"""Plain references of the serving calls, numpy on the host: quantizer with a step per token, the layer on such codes,
the cache of quantized pages and attention over it in 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def constants(m, bits):
    """(scale, inv) of Eq. 1 for maxima m (float32): correctly rounded quotients, 0 for a maximum of 0 or one whose inv
    would not be finite."""
    m = np.asarray(m, np.float32)
    q = np.float32(2 ** (bits - 1) - 1)
    with np.errstate(over="ignore", divide="ignore"):
        inv = np.where(m > 0, q / np.where(m > 0, m, np.float32(1)), np.float32(0)).astype(np.float32)
    fine = np.isfinite(inv) & (m > 0)
    return np.where(fine, m / q, np.float32(0)).astype(np.float32), np.where(fine, inv, np.float32(0))


def codes_of(x, inv, bits):
    """clamp(round-half-even of the exact product)."""
    q = 2 ** (bits - 1) - 1
    return np.clip(np.rint(np.asarray(x, np.float64) * np.asarray(inv, np.float64)), -q, q).astype(np.int8)


def token_quant(x, bits):
    x = np.asarray(x, np.float32)
    scale, inv = constants(np.abs(x).max(axis=1), bits)
    return codes_of(x, inv[:, None], bits), scale


def qgemm_tokens(a_q, w_q, a_scale, w_scale):
    """fl32(fl32(acc * a_scale) * w_scale) on codes int8 [M, K], [N, K]."""
    acc = a_q.astype(np.float64) @ w_q.astype(np.float64).T  # whole numbers far below 2^53: exact
    assert np.abs(acc).max(initial=0) < 2 ** 31
    return (acc.astype(np.int32).astype(np.float32) * a_scale[:, None].astype(np.float32)) * w_scale[None].astype(np.float32)


class Cache:
    """Codes [pages][heads][page][dim] and maxima, for keys and for values; tables and lengths come with each call."""

    def __init__(self, pages, heads, page, dim, bits):
        self.page, self.bits = page, bits
        self.codes = {n: np.zeros((pages, heads, page, dim), np.int8) for n in "kv"}
        self.absmax = {n: np.zeros((pages, heads), np.float32) for n in "kv"}
        self.used = {n: np.zeros((pages, page), bool) for n in "kv"}

    def _place(self, table, p):
        if p < 0 or p >= self.page * len(table):
            return None
        on = int(table[p // self.page])
        return (on, p % self.page) if 0 <= on < self.absmax["k"].shape[0] else None

    def append(self, starts, kv_len, table, k, v):
        for s in range(len(kv_len)):
            n = int(starts[s + 1] - starts[s])
            by_page = {}
            for i in range(n):
                at = self._place(table[s], int(kv_len[s]) - n + i)
                if at is not None:
                    by_page.setdefault(at[0], []).append((at[1], int(starts[s]) + i))
            for on, rows in by_page.items():
                lo = rows[0][0]
                for name, x in (("k", k), ("v", v)):
                    codes, absmax = self.codes[name][on], self.absmax[name]
                    new = np.stack([x[r] for _, r in rows]).astype(np.float32)  # [rows, heads, dim]
                    was = absmax[on].copy() if lo > 0 else np.zeros_like(absmax[on])
                    now = np.maximum(was, np.abs(new).max(axis=(0, 2))).astype(np.float32)
                    old_scale, _ = constants(was, self.bits)
                    _, inv = constants(now, self.bits)
                    for h in range(codes.shape[0]):
                        if lo > 0 and now[h] > was[h]:
                            old = codes[h, :lo].astype(np.float32) * old_scale[h]
                            codes[h, :lo] = codes_of(old, inv[h], self.bits)
                        for (p, _), row in zip(rows, new):
                            codes[h, p] = codes_of(row[h], inv[h], self.bits)
                    absmax[on] = now
                    for p, _ in rows:
                        self.used[name][on, p] = True

    def value(self, name, table, p):
        """float32 [heads, dim] of the token at position p; None where there is none."""
        at = self._place(table, p)
        if at is None:
            return None
        scale, _ = constants(self.absmax[name][at[0]], self.bits)
        return self.codes[name][at[0], :, at[1]].astype(np.float32) * scale[:, None]

    def gather(self, starts, kv_len, table, rows):
        heads, dim = self.codes["k"].shape[1], self.codes["k"].shape[3]
        out = {n: np.zeros((rows, heads, dim), np.float32) for n in "kv"}
        for s in range(len(kv_len)):
            n = int(starts[s + 1] - starts[s])
            for i in range(n):
                for name in "kv":
                    x = self.value(name, table[s], int(kv_len[s]) - n + i)
                    if x is not None:
                        out[name][int(starts[s]) + i] = x
        return out["k"], out["v"]

    def attention(self, starts, kv_len, table, q, causal, window, scale):
        """(output, its error scale) in float64: out[row, head] and, per row and head, the largest |logit| that products
        of magnitudes give and the largest |value| seen, from which a test forms its bound."""
        rows, heads, dim = q.shape
        kh = self.codes["k"].shape[1]
        qmax = 2.0 ** (self.bits - 1) - 1
        out = np.zeros((rows, heads, dim))
        logit, big = np.zeros((rows, heads)), np.zeros((rows, heads))
        for s in range(len(kv_len)):
            length = min(int(kv_len[s]), self.page * table.shape[1])
            places = [self._place(table[s], p) for p in range(length)]
            there = np.array([p is not None for p in places], bool)
            on = np.array([p[0] if p else 0 for p in places], int)
            at = np.array([p[1] if p else 0 for p in places], int)
            if length:
                k = self.codes["k"][on, :, at].astype(np.float64) * (self.absmax["k"][on].astype(np.float64) / qmax)[..., None]
                v = self.codes["v"][on, :, at].astype(np.float64) * (self.absmax["v"][on].astype(np.float64) / qmax)[..., None]
            n = int(starts[s + 1] - starts[s])
            for i in range(n):
                p = int(kv_len[s]) - n + i
                j = np.arange(length)
                see = there.copy()
                if causal:
                    see &= j <= p
                if window:
                    see &= j > p - window
                if not see.any():
                    continue
                row = int(starts[s]) + i
                for h in range(heads):
                    kk, vv = k[see, h * kh // heads], v[see, h * kh // heads]
                    x = kk @ q[row, h].astype(np.float64) * scale
                    e = np.exp(x - x.max())
                    out[row, h] = (e / e.sum()) @ vv
                    logit[row, h] = (np.abs(kk) @ np.abs(q[row, h].astype(np.float64))).max() * abs(scale)
                    big[row, h] = np.abs(vv).max()
        return out, logit, big


def packed_values(codes):
    """[pages][heads][page][dim] in the cache's value order [pages][heads][page / 4][dim][4]."""
    p, h, t, d = codes.shape
    return np.ascontiguousarray(codes.reshape(p, h, t // 4, 4, d).transpose(0, 1, 2, 4, 3))
