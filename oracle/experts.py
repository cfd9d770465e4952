"""Float64 oracle of the operators behind the decode attention: routing to experts, the lists of pairs by expert, 8-bit
products, and sampling.  Written from the definitions in include/rk.h, token by token."""
from __future__ import annotations

from fractions import Fraction

import numpy as np


def scores(logits, score):
    """s of every expert of one token: softmax (over all experts) or sigmoid, in 64 bits."""
    x = np.asarray(logits, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-x))
        top = x.max()
        p = np.where(x == -np.inf, 0.0, np.exp(x - top))
        return p / p.sum()


def route(logits, k, bias=None, score="softmax", n_groups=1, top_groups=1, group_top=1, renorm=False, scale=1.0):
    """ids [n, k], weights [n, k] (float64)."""
    logits = np.asarray(logits, dtype=np.float64)
    n, n_e = logits.shape
    b = np.zeros(n_e) if bias is None else np.asarray(bias, dtype=np.float64)
    ids, weights = np.full((n, k), -1, dtype=np.int64), np.zeros((n, k))
    size = n_e // n_groups
    for t in range(n):
        open_ = (logits[t] != -np.inf) & (b != -np.inf)
        if np.isnan(logits[t]).any():
            weights[t] = np.nan
            continue
        s = scores(logits[t], score)
        c = s + b
        if np.isnan(c[logits[t] != -np.inf]).any():
            weights[t] = np.nan
            continue
        if n_groups > 1:
            rank = []
            for g in range(n_groups):
                mine = [c[e] for e in range(g * size, (g + 1) * size) if open_[e]]
                rank.append(sum(sorted(mine, reverse=True)[:group_top]) if mine else -np.inf)
            chosen = sorted(range(n_groups), key=lambda g: (-rank[g], g))[:top_groups]
            open_ = open_ & np.isin(np.arange(n_e) // size, chosen)
        order = sorted((e for e in range(n_e) if open_[e]), key=lambda e: (-c[e], e))[:k]
        w = np.array([s[e] for e in order])
        if renorm and len(order):
            total = w.sum()
            w = w / total if total > 0 else np.zeros_like(w)
        ids[t, :len(order)], weights[t, :len(order)] = order, w * scale
    return ids, weights


def group(ids, n_experts, keep=None):
    """row_off [n_experts + 1], rows [n * k] with -1 behind the last pair."""
    n, k = ids.shape
    lists = [[] for _ in range(n_experts)]
    for t in range(n):
        for s in range(k):
            e = int(ids[t, s])
            if 0 <= e < n_experts and (keep is None or (int(keep[t]) >> s) & 1):
                lists[e].append(t * k + s)
    off = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int64)
    rows = np.full(n * k, -1, dtype=np.int64)
    rows[:off[-1]] = [p for x in lists for p in x]
    return off, rows


def quant8(x):
    """codes (int), scales (float64 values of float32 numbers) of rows; exact quotients, ties to even."""
    x = np.asarray(x, dtype=np.float64)
    codes, scales = np.zeros(x.shape, dtype=np.int64), np.full(len(x), np.nan)
    for i, row in enumerate(x):
        if not np.isfinite(row).all():
            continue
        top = np.float32(np.abs(row).max()) if len(row) else np.float32(0)
        scales[i] = np.float64(top / np.float32(127.0))
        if scales[i] == 0.0:
            continue
        q = row / scales[i]                                    # 64 bits: off by 2^-53, decided exactly below
        low = np.floor(q)
        near = np.abs(q - low - 0.5) < 1e-9
        code = np.rint(q)
        for j in np.nonzero(near)[0]:
            exact = Fraction(float(row[j])) / Fraction(float(scales[i]))
            code[j] = float(round(exact))                      # Fraction rounds half to even
        codes[i] = np.clip(code, -127, 127).astype(np.int64)
    return codes, scales


def matmul8(w_codes, w_scales, x_codes, x_scales):
    """y [tokens, channels] in 64 bits; the integer sums are exact."""
    acc = x_codes.astype(np.float64) @ w_codes.astype(np.float64).T
    return acc * x_scales[:, None] * w_scales[None]


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The tokens that stay, ascending, and their weights p (float64).  Assumes a row without NaN and with a finite maximum."""
    x = np.asarray(logits, dtype=np.float64)
    order = sorted((i for i in range(len(x)) if x[i] > -np.inf), key=lambda i: (-x[i], i))
    top = x[order[0]]
    p = {i: float(np.exp((x[i] - top) / temperature)) for i in order}
    if 0 < top_k < len(x):
        order = order[:top_k]
    total = sum(p[i] for i in order)
    stay, front = [], 0.0
    for i in order:
        if stay and ((top_p < 1 and not front < top_p * total) or p[i] < min_p):
            break
        stay.append(i)
        front += p[i]
    stay.sort()
    return np.array(stay), np.array([p[i] for i in stay])


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob) of one row."""
    x = np.asarray(logits, dtype=np.float64)
    if np.isnan(x).any() or x.max() == -np.inf:
        return -1, np.nan
    if not temperature >= 2.0 ** -100:
        return int(np.argmax(x)), 1.0
    if x.max() == np.inf:
        x = np.where(x == np.inf, 0.0, -np.inf)
    stay, p = kept(x, temperature, top_k, top_p, min_p)
    total = np.cumsum(p)
    u = min(max(0.0, u), 1.0) if u == u else 0.0
    at = min(int(np.searchsorted(total, u * total[-1], side="right")), len(stay) - 1)
    return int(stay[at]), p[at] / total[-1]
