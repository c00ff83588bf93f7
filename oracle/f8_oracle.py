"""CPU oracle of rows and products in 8-bit floating point and of sampling: plain numpy in 64 bits from the definitions in include/moqe.h."""
from __future__ import annotations

import math

import numpy as np

from oracle.decoder_oracle import e4m3_code, e4m3_value, scale_for

BLOCK = 128


def quantize_rows(x):
    """Codes [M, 128 * blocks] and scale bytes [M, blocks] of rows x [M, d]."""
    x = np.asarray(x, dtype=np.float64)
    M, d = x.shape
    blocks = -(-d // BLOCK)
    x = np.concatenate([x, np.zeros((M, blocks * BLOCK - d))], 1).reshape(M, blocks, BLOCK)
    codes, scales = np.zeros((M, blocks, BLOCK), np.uint8), np.zeros((M, blocks), np.uint8)
    for m in range(M):
        for b in range(blocks):
            v = x[m, b]
            s = scale_for(np.abs(v[np.isfinite(v)]).max(initial=0.0))
            codes[m, b] = e4m3_code(v / s)
            scales[m, b] = 127 + int(math.log2(s))
    return codes.reshape(M, -1), scales


def rows_value(codes, scales, d):
    """What 8-bit rows stand for."""
    v = e4m3_value(codes) * np.repeat(2.0 ** (np.asarray(scales).astype(np.float64) - 127), BLOCK, axis=1)
    return v[:, :d]


def product(a, w, up=None):
    """Rows a [M, k] times matrix w [n, k], or silu(a w^T) * (a up^T)."""
    with np.errstate(over="ignore"):
        y = a @ w.T
        return y if up is None else y / (1.0 + np.exp(-y)) * (a @ up.T)


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Token of one row, its log probability, and the gap in units of the largest weight to the nearest choice that would have come out differently."""
    x = np.asarray(logits, dtype=np.float64)
    live = [i for i in range(len(x)) if x[i] > -np.inf]
    if not live:
        return -1, -np.inf, 1.0
    live.sort(key=lambda i: (-x[i], i))
    if not temperature > 0:
        return live[0], 0.0, 1.0
    m = x[live[0]]
    if m == np.inf:
        w = np.array([1.0 if x[i] == np.inf else 0.0 for i in live])
    else:
        w = np.exp((x[live] - m) / temperature)
    n, gap = len(live), 1.0
    if top_k >= 1:
        n = min(n, top_k)
    if top_p < 1:
        run, whole = np.concatenate([[0.0], np.cumsum(w[:n])]), w[:n].sum()
        want = max(top_p, 0.0) * whole
        gap = min(gap, np.abs(run[1:] - want).min()) if top_p > 0 else gap
        n = max(1, int((run[:-1] < want).sum()))
    if min_p > 0:
        least = min(min_p, 1.0)
        gap = min(gap, np.abs(w[1:n] - least).min(initial=1.0)) if least < 1 else gap
        n = int((w[:n] >= least).sum())
    at = sorted(range(n), key=lambda j: live[j])
    run = np.cumsum(w[at])
    goal = min(max(u, 0.0), 1.0) * run[-1] if u == u else 0.0
    i = int((run <= goal).sum())
    if i >= n:                                                 # u is 1: the last token with weight
        i = max(j for j in range(n) if w[at[j]] > 0)
    gap = min(gap, np.abs(run - goal).min() if goal > 0 else 1.0)
    return live[at[i]], math.log(w[at[i]] / run[-1]), gap
