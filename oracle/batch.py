"""Batches of sequences over a paged cache, and log probabilities (oracle).

The position rotation is the decoder's (rotate-half pairs i, i + hd / 2); the
attention is softmax(q k^T / sqrt(hd)) v over the visible slots; logits turn
into log probabilities, entropies and alternatives by their definitions.  The
8-bit cache holds OCP e4m3 codes (1 sign, 4 exponent bits of bias 7, 3 bits
behind the point, no infinities, S1111111 is NaN) times a power-of-two scale
for each page, head and kind.  Everything is float64.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
F8_MAX = 448.0


def _decode_table():
    t = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.ldexp(1 + m / 8, e - 7) if e else math.ldexp(m / 8, -6)
        t[c] = (-v if c & 128 else v) if c & 127 != 127 else math.nan
    return t


E4M3 = _decode_table()
_POSITIVE = E4M3[:127]                                   # codes 0 .. 126 in order


def round_e4m3(x):
    """Codes of the nearest e4m3 values (ties to the even code), saturating; NaN is code 127."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), F8_MAX)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)  # NaN sorts last
    lo = np.maximum(hi - 1, 0)
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), 127, code)
    return np.where(np.signbit(x) & ~np.isnan(x), code + 128, code).astype(np.uint8)


def block_scale(values):
    """The smallest power of two that brings the finite values to 448 or less; 1 for zeros."""
    v = np.abs(np.asarray(values, np.float64))
    top = v[np.isfinite(v)].max(initial=0.0)
    if top == 0:
        return 1.0
    k = math.ceil(math.log2(top / F8_MAX))
    while top > F8_MAX * 2.0 ** k:
        k += 1
    while top <= F8_MAX * 2.0 ** (k - 1):
        k -= 1
    return 2.0 ** k


def page_bytes(G, hd):
    return -(-(2 * G * PAGE * hd + 8 * G) // 128) * 128


def key_offset(t, i, hd):
    """Byte of the key of token t, dim i inside its head's 64 hd codes."""
    lane, b = t % 16 + 16 * (i // (hd // 4)), (t // 16) * (hd // 4) + i % (hd // 4)
    return (b // 16) * 1024 + lane * 16 + b % 16


def value_offset(t, i):
    lane, b = i % 16 + 16 * ((t // 4) % 4), 16 * (i // 16) + 4 * (t // 16) + t % 4
    return (b // 16) * 1024 + lane * 16 + b % 16


def _offsets(G, hd, g, kind):
    """[64][hd] byte offsets in a page of head g's keys (kind 0) or values (kind 1)."""
    t, i = np.meshgrid(np.arange(PAGE), np.arange(hd), indexing="ij")
    return (kind * G + g) * PAGE * hd + (value_offset(t, i) if kind else key_offset(t, i, hd))


class Pool8:
    """An e4m3 pool: raw bytes [n_pages][page_bytes] as the library lays them out."""

    def __init__(self, raw, G, hd):
        self.raw, self.G, self.hd = np.array(raw, np.uint8).reshape(-1, page_bytes(G, hd)), G, hd
        self.at = [[_offsets(G, hd, g, kind) for g in range(G)] for kind in (0, 1)]

    def _scale_slice(self, page, g, kind):
        o = 2 * self.G * PAGE * self.hd + 8 * g + 4 * kind
        return self.raw[page, o:o + 4]

    def scale(self, page, g, kind):
        return float(self._scale_slice(page, g, kind).copy().view(np.float32)[0])

    def values(self, page, g, kind):
        """[64][hd] values that a head's keys or values in a page stand for."""
        return E4M3[self.raw[page, self.at[kind][g]]] * self.scale(page, g, kind)

    def append(self, page, g, kind, t0, new):
        """new [m][hd] at tokens t0 .. t0 + m - 1; tokens below t0 are kept.  Kept zeros on scale 1 (which zeros get)
        do not hold the new ones to it."""
        need = block_scale(new)
        at = self.at[kind][g]
        keeps = t0 and (self.scale(page, g, kind) != 1 or (self.raw[page, at[:t0]] & 127).any())
        scale = max(need, self.scale(page, g, kind)) if keeps else need
        if keeps and scale > self.scale(page, g, kind):
            kept = E4M3[self.raw[page, at[:t0]]] * self.scale(page, g, kind)
            self.raw[page, at[:t0]] = round_e4m3(kept / scale)
        self.raw[page, at[t0:t0 + len(new)]] = round_e4m3(new / scale)
        self._scale_slice(page, g, kind)[:] = np.array([scale], np.float32).view(np.uint8)


class PoolDense:
    """An fp32 or bf16 pool as values: K [pages][G][64][hd] and V transposed [pages][G][hd][64]."""

    def __init__(self, values, G, hd):
        v = np.array(values, np.float64).reshape(-1, 2 * G * PAGE * hd)
        self.k = v[:, :G * PAGE * hd].reshape(-1, G, PAGE, hd).copy()
        self.v = v[:, G * PAGE * hd:].reshape(-1, G, hd, PAGE).copy()

    def append(self, page, g, kind, t0, new):
        if kind == 0:
            self.k[page, g, t0:t0 + len(new)] = new
        else:
            self.v[page, g, :, t0:t0 + len(new)] = new.T

    def values(self, page, g, kind):
        return self.k[page, g] if kind == 0 else self.v[page, g].T


def rotate(x, pos, base):
    """Rows [R][heads][hd] turned by their positions (base 0: not at all)."""
    x = np.asarray(x, np.float64)
    if not base:
        return x.copy()
    half = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None] * base ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def append(pool, row_start, ctx, table, k, v, base=0.0, pos=None):
    """Rows k, v [R][G][hd] of every sequence into the pool, keys rotated."""
    for s, C in enumerate(ctx):
        r0, r1 = row_start[s], row_start[s + 1]
        slots = C + np.arange(r1 - r0)
        kr = rotate(k[r0:r1], slots if pos is None else pos[r0:r1], base)
        for page in sorted(set((slots // PAGE).tolist())):
            mine = np.nonzero(slots // PAGE == page)[0]
            for g in range(k.shape[1]):
                pool.append(table[s][page], g, 0, int(slots[mine[0]] % PAGE), kr[mine, g])
                pool.append(table[s][page], g, 1, int(slots[mine[0]] % PAGE), np.asarray(v, np.float64)[r0:r1][mine, g])


def gather(pool, table_row, n, G, kind):
    """[n][G][hd] keys or values of a sequence's first n slots."""
    out = []
    for p in range(-(-n // PAGE)):
        out.append(np.stack([pool.values(table_row[p], g, kind) for g in range(G)], 1))
    return np.concatenate(out)[:n] if out else np.zeros((0, G, 1))


def attention(q, k, v, C, vis):
    """Rows q [n][H][hd] of one sequence over k, v [C + n][G][hd]; vis [n][n] bool of the in-step slots."""
    n, H, hd = q.shape
    G = k.shape[1]
    seen = np.concatenate([np.ones((n, C), bool), np.asarray(vis, bool)], 1)
    out = np.zeros((n, H, hd))
    for i in range(n):
        js = np.nonzero(seen[i])[0]
        if not len(js):
            continue
        for h in range(H):
            kk, vv = k[js, h // (H // G)], v[js, h // (H // G)]
            s = kk @ q[i, h] / math.sqrt(hd)
            w = np.exp(s - s.max())
            out[i, h] = (w / w.sum()) @ vv
    return out


def token_logprobs(x, tokens, k):
    """(logprob [R], entropy [R], norm [R][2], ids [R][k], their log probabilities [R][k])."""
    x = np.asarray(x, np.float64)
    R, V = x.shape
    lp, ent, norm = np.zeros(R), np.zeros(R), np.zeros((R, 2))
    ids, top = np.full((R, k), -1, np.int32), np.full((R, k), -np.inf)
    for r in range(R):
        m = x[r].max()
        if not np.isfinite(m) or np.isnan(x[r]).any():
            lp[r] = 0.0 if tokens[r] == -1 else np.nan
            ent[r] = np.nan
            norm[r] = np.nan
            top[r] = np.nan
            continue
        ls = math.log(math.fsum(np.exp(x[r] - m)))
        logp = x[r] - m - ls
        p = np.exp(logp)
        t = tokens[r]
        lp[r] = 0.0 if t == -1 else (logp[t] if 0 <= t < V else np.nan)
        ent[r] = -math.fsum((p * np.where(p > 0, logp, 0.0)))
        norm[r] = m, ls
        order = np.lexsort((np.arange(V), -x[r]))[:k]
        order = order[x[r][order] > -np.inf]
        ids[r, :len(order)] = order
        top[r, :len(order)] = logp[order]
    return lp, ent, norm, ids, top


def token_logprobs_grad(x, tokens, g, h):
    """Gradient of sum(g * logprob + h * entropy) to the logits."""
    x = np.asarray(x, np.float64)
    out = np.zeros_like(x)
    for r in range(len(x)):
        gr = g[r] if tokens[r] >= 0 else 0.0
        if gr == 0 and h[r] == 0:
            continue
        m = x[r].max()
        logp = x[r] - m - math.log(math.fsum(np.exp(x[r] - m)))
        p = np.exp(logp)
        safe = np.where(p > 0, logp, 0.0)
        out[r] = -gr * p - h[r] * p * (safe - math.fsum(p * safe))
        if tokens[r] >= 0:
            out[r, tokens[r]] += gr
    return out
