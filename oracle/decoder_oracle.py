"""CPU oracle of what a decoder layer does around its products: norms with the residual, rotary positions, the paged cache in 8 bits and the
attention over it.  Plain numpy in 64 bits, one row, block and head at a time, from the definitions in include/moqe.h."""
from __future__ import annotations

import math

import numpy as np


def norm(x, kind, eps, gain=None, offset=None):
    x = np.asarray(x, dtype=np.float64)
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        y = y * gain
    return y + offset if offset is not None else y


def residual_norm(y, residual, gate=None, gate_rows=0, scale=1.0, post=None, pre=None):
    """Returns t and pre(t), not rounded.  post, pre: arguments of norm() after x, or None."""
    t = np.asarray(residual, dtype=np.float64).copy()
    if y is not None:
        u = np.asarray(y, dtype=np.float64)
        if post is not None:
            u = norm(u, *post)
        if gate is not None:
            g = np.asarray(gate, dtype=np.float64)
            u = u * (g[np.arange(len(u)) // gate_rows] if gate_rows > 0 else g)
        t = t + scale * u
    return t, (norm(t, *pre) if pre is not None else t)


# ------------------------------------------------------------------------------------------------ codes and their places
def e4m3_value(code):
    """What a code stands for: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    u = np.asarray(code).astype(np.int64)
    e, m = (u >> 3) & 15, u & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x = np.where((u & 127) == 127, np.nan, x)
    return np.where(u & 128, -x, x)


_VALUES = e4m3_value(np.arange(127))


def e4m3_code(x):
    """The nearest code, ties to the even one, past 448 the largest; NaN 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.where(np.isnan(x), 0.0, np.abs(x)), 448.0)
    i = np.clip(np.searchsorted(_VALUES, a), 1, 126)
    lo, hi = a - _VALUES[i - 1], _VALUES[i] - a
    c = np.where(lo < hi, i - 1, np.where(hi < lo, i, np.where((i - 1) % 2 == 0, i - 1, i)))
    c = c | np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 127, c).astype(np.uint8)


def key_at(token, dim, dh):
    lane = (dim % 32) // 8 * 16 + token % 16
    return token // 16 * (16 * dh) + dim // 64 * 1024 + lane * 16 + (dim % 64) // 32 * 8 + dim % 8


def value_at(token, dim, dh):
    u = token % 32
    lane = (u % 16) // 4 * 16 + dim % 16
    return token // 32 * (32 * dh) + dim // 32 * 1024 + lane * 16 + (dim % 32) // 16 * 8 + u // 16 * 4 + u % 4


def scale_for(amax):
    if amax == 0:
        return 2.0 ** -120
    e = math.ceil(math.log2(amax / 448.0))
    while amax > 448.0 * 2.0 ** e:                    # log2 rounds
        e += 1
    while amax <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** min(120, max(-120, e))


class Cache:
    """codes [n_blocks, n_heads, block_tokens * head_dim] uint8 and scales [n_blocks, n_heads], as in device memory."""

    def __init__(self, n_blocks, n_heads, bt, dh, fill=0):
        self.bt, self.dh, self.n_heads, self.n_blocks = bt, dh, n_heads, n_blocks
        self.k, self.v = (np.full((n_blocks, n_heads, bt * dh), fill, dtype=np.uint8) for _ in range(2))
        self.k_scale, self.v_scale = (np.ones((n_blocks, n_heads)) for _ in range(2))
        t, d = np.meshgrid(np.arange(bt), np.arange(dh), indexing="ij")
        self.at = {"k": key_at(t, d, dh), "v": value_at(t, d, dh)}       # [token, dim]

    def codes(self, which):
        return self.k if which == "k" else self.v

    def scales(self, which):
        return self.k_scale if which == "k" else self.v_scale

    def read(self, which, block, head):
        """[tokens, dims] of one block and head."""
        return e4m3_value(self.codes(which)[block, head][self.at[which]]) * self.scales(which)[block, head]

    def write(self, which, block, head, lo, x, held):
        """Tokens lo .. of the block become x [n, dims]; held: the block holds `lo` earlier tokens of the sequence."""
        codes, scales, at = self.codes(which)[block, head], self.scales(which), self.at[which]
        finite = np.abs(x[np.isfinite(x)])
        s = scale_for(finite.max() if finite.size else 0.0)
        old = scales[block, head]
        if held:
            s = max(s, old)
            if s > old:
                codes[at[:lo]] = e4m3_code(e4m3_value(codes[at[:lo]]) * (old / s))
        with np.errstate(over="ignore", invalid="ignore"):
            codes[at[lo:lo + len(x)]] = e4m3_code(x / s)
        scales[block, head] = s


def rotated(x, pos, inv_freq, rot, interleaved, mscale=1.0):
    """x [.., dims] with its first `rot` dims turned by position pos."""
    y = np.array(x, dtype=np.float64)
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, s = mscale * math.cos(pos * inv_freq[j]), mscale * math.sin(pos * inv_freq[j])
        u, v = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
        y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y


def sequences(S, T, M, kv_len, width, bt, cu=None):
    """(row0, rows, tokens) of every sequence, device values taken into their ranges."""
    out = []
    for s in range(S):
        r0, n = s * T, T
        if cu is not None:
            r0 = min(max(int(cu[s]), 0), M)
            n = max(min(max(int(cu[s + 1]), 0), M) - r0, 0)
        out.append((r0, n, min(max(int(kv_len[s]), 0), width * bt)))
    return out


def kv_append(qkv, n_heads, cache, table, seqs, T, inv_freq, rot, interleaved=False, mscale=1.0, q_gain=None, k_gain=None, eps=1e-6):
    """Writes the cache; returns the turned queries [M, n_heads, dims], not rounded (rows that are not computed: NaN)."""
    dh, H, bt = cache.dh, cache.n_heads, cache.bt
    x = np.asarray(qkv, dtype=np.float64).reshape(len(qkv), -1, dh)
    q_out = np.full((len(x), n_heads, dh), np.nan)
    for s, (r0, n, L) in enumerate(seqs):
        n_do = min(n, T)
        keys = np.zeros((n_do, H, dh))
        for i in range(n_do):
            p = L - n + i
            q, k = x[r0 + i, :n_heads], x[r0 + i, n_heads:n_heads + H]
            q = norm(q, "rms", eps, q_gain) if q_gain is not None else q
            k = norm(k, "rms", eps, k_gain) if k_gain is not None else k
            q_out[r0 + i] = rotated(q, p, inv_freq, rot, interleaved, mscale)
            keys[i] = rotated(k, p, inv_freq, rot, interleaved, mscale)
        first = L - n
        p0, end = max(first, 0), min(L, first + n_do)
        for b in range(p0 // bt, -(-end // bt) if end > p0 else 0):
            lo, hi = max(p0, b * bt), min(end, (b + 1) * bt)
            block = int(table[s, b])
            if not 0 <= block < cache.n_blocks:
                continue
            for h in range(H):
                cache.write("k", block, h, lo - b * bt, keys[lo - first:hi - first, h], lo > b * bt)
                cache.write("v", block, h, lo - b * bt, x[r0 + lo - first:r0 + hi - first, n_heads + H + h], lo > b * bt)
    return q_out


def kv_attention(q, n_heads, cache, table, seqs, T, scale, cap=0.0, window=0, slopes=None, prefix=None):
    """[M, n_heads, dims], not rounded (rows that are not computed: NaN), and the same sums over |v|, in which rounding errors are counted."""
    dh, H, bt = cache.dh, cache.n_heads, cache.bt
    q = np.asarray(q, dtype=np.float64).reshape(len(q), n_heads, dh)
    out, size = np.full(q.shape, np.nan), np.zeros(q.shape)
    G = n_heads // H
    for s, (r0, n, L) in enumerate(seqs):
        t = np.arange(L)
        blocks = [int(table[s, b]) for b in range(-(-L // bt))]
        present = np.array([0 <= b < cache.n_blocks for b in blocks], dtype=bool).repeat(bt)[:L] if L else np.zeros(0, bool)
        pre = int(prefix[s]) if prefix is not None else 0
        for h in range(H):
            K, V = (np.concatenate([cache.read(m, b, h) if 0 <= b < cache.n_blocks else np.zeros((bt, dh)) for b in blocks] or
                                   [np.zeros((0, dh))])[:L] for m in ("k", "v"))
            for i in range(min(n, T)):
                p = L - n + i
                sees = present & ((t < pre) | ((t <= p) & ((p - t < window) if window > 0 else True)))
                for g in range(h * G, (h + 1) * G):
                    if not sees.any():
                        out[r0 + i, g] = 0.0
                        continue
                    a = scale * (K[sees] @ q[r0 + i, g])
                    if cap > 0:
                        a = cap * np.tanh(a / cap)
                    if slopes is not None:
                        a = a - float(slopes[g]) * np.abs(p - t[sees])
                    w = np.exp(a - a.max())
                    out[r0 + i, g], size[r0 + i, g] = (w @ V[sees]) / w.sum(), (w @ np.abs(V[sees])) / w.sum()
    return out, size
