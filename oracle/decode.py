"""Float64 oracle of the decode operators: the 4-bit latent cache (format, append, read), attention of single
tokens over cached segments, and 4-bit weight matrices.  Written from the definitions in include/rk.h."""
from __future__ import annotations

import numpy as np

PAGE_ROWS, UNITS, PAGE_BYTES = 64, 26, 26624


def bf16_bits(x) -> np.ndarray:
    """Nearest bfloat16 (ties to even) of finite float64/float32 values, as 16-bit patterns."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def bf16_values(bits) -> np.ndarray:
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


SCALES = np.array([2.0 ** ((b >> 3) - 20) * (1 + (b & 7) / 8) for b in range(255)])


def quantise_latent(c):
    """c [n, 512] -> codes int [n, 512] in -7..7, scale bytes uint8 [n, 32] (255: a group with a non-finite value)."""
    c = np.asarray(c, dtype=np.float64)
    x = c.reshape(len(c), 32, 16)
    finite = np.isfinite(x).all(axis=2)
    x = np.where(finite[..., None], x, 0.0)
    want = np.abs(x).max(axis=2) / 7.0
    hi = np.searchsorted(SCALES, want)                     # first scale >= want
    hi = np.clip(hi, 0, 254)
    lo = np.clip(hi - 1, 0, 254)
    up, down = np.abs(SCALES[hi] - want), np.abs(want - SCALES[lo])
    byte = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    codes = np.clip(np.rint(x / SCALES[byte][..., None]), -7, 7)
    return codes.reshape(len(c), 512).astype(np.int64), np.where(finite, byte, 255).astype(np.uint8)


def latent_values(codes, byte):
    s = np.append(SCALES, np.nan)[byte]
    return (codes.reshape(len(codes), 32, 16) * s[..., None]).reshape(len(codes), 512)


def turn(x, pos, base):
    """R(pos) of interleaved pairs, x [..., 64]; pos broadcasts over the leading axes."""
    ang = np.asarray(pos, dtype=np.float64)[..., None] * base ** (-2.0 * np.arange(32) / 64)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * ang)
    return np.stack([z.real, z.imag], axis=-1).reshape(x.shape)


def pack_row(codes, byte, rope_bits) -> np.ndarray:
    """One cached row as its 26 units of 16 bytes, uint8 [26, 16]."""
    out = np.zeros((UNITS, 16), dtype=np.uint8)
    for d in range(512):
        u, w, r = d // 32, (d % 32) // 8, d % 8
        bit = 32 * w + 16 * (r % 2) + 4 * (r // 2)
        out[u, bit // 8] |= np.uint8((int(codes[d]) + 8) << (bit % 8))
    for g in range(32):
        out[16 + (g // 4) % 2, 4 * (g // 8) + g % 4] = byte[g]
    out[18:] = np.asarray(rope_bits, dtype=np.uint16).view(np.uint8).reshape(8, 16)
    return out


def unpack_row(units):
    """Inverse of pack_row: (codes [512], scale bytes [32], rope values [64])."""
    codes, byte = np.zeros(512, dtype=np.int64), np.zeros(32, dtype=np.uint8)
    for d in range(512):
        u, w, r = d // 32, (d % 32) // 8, d % 8
        bit = 32 * w + 16 * (r % 2) + 4 * (r // 2)
        codes[d] = ((int(units[u, bit // 8]) >> (bit % 8)) & 15) - 8
    for g in range(32):
        byte[g] = units[16 + (g // 4) % 2, 4 * (g // 8) + g % 4]
    return codes, byte, bf16_values(np.ascontiguousarray(units[18:]).view(np.uint16).reshape(64))


class Cache:
    """Host model of the page pool: uint8 [n_pages, 26, 64, 16]."""

    def __init__(self, n_pages, fill=0):
        self.pages = np.full((n_pages, UNITS, PAGE_ROWS, 16), fill, dtype=np.uint8)

    def write_row(self, page, slot, units):
        self.pages[page, :, slot] = units

    def rows(self, page_list, n):
        """(values [n, 576]) of the first n rows of a segment, vectorised."""
        if n == 0:
            return np.zeros((0, 576))
        p = self.pages[np.asarray(page_list)[:(n + 63) // 64]]              # [P, 26, 64, 16]
        p = np.ascontiguousarray(p.transpose(0, 2, 1, 3)).reshape(-1, UNITS, 16)[:n]
        w = np.ascontiguousarray(p[:, :16]).view(np.uint32)                 # [n, 16, 4]
        sh = np.array([16 * (r % 2) + 4 * (r // 2) for r in range(8)], dtype=np.uint32)
        codes = ((w[..., None] >> sh) & 15).astype(np.int64).reshape(n, 512) - 8
        byte = np.stack([p[:, 16 + (g // 4) % 2, 4 * (g // 8) + g % 4] for g in range(32)], axis=1)
        rope = bf16_values(np.ascontiguousarray(p[:, 18:]).reshape(n, 128).view(np.uint16))
        return np.concatenate([latent_values(codes, byte), rope], axis=1)


def attention(q, pos, items, sm_scale, base):
    """q [R, 576] at request positions, pos [R]; items: list of (rows [n, 576], delta).  Returns O [R, 512],
    lse [R] (natural log; -inf and O = 0 for a row that sees nothing), and what enters error bounds: mass [R, 512] =
    sum p |c|, and per row the largest sum |q_rope| |k_rope| and sum |q| |k| over the visible keys."""
    q, pos = np.asarray(q, dtype=np.float64), np.asarray(pos)
    logits, vals, big, size = [], [], np.zeros(len(q)), np.zeros(len(q))
    for rows, delta in items:
        qr = turn(q[:, 512:], np.full(len(q), -float(delta)), base)
        s = (q[:, :512] @ rows[:, :512].T + qr @ rows[:, 512:].T) * sm_scale
        seen = (delta + np.arange(len(rows)))[None, :] <= pos[:, None]
        logits.append(np.where(seen, s, -np.inf))
        vals.append(rows[:, :512])
        if len(rows):
            turned = np.abs(qr) @ np.abs(rows[:, 512:]).T
            big = np.maximum(big, np.where(seen, turned, 0.0).max(axis=1))
            size = np.maximum(size, np.where(seen, turned + np.abs(q[:, :512]) @ np.abs(rows[:, :512]).T, 0.0).max(axis=1))
    if not logits or sum(x.shape[1] for x in logits) == 0:
        return np.zeros((len(q), 512)), np.full(len(q), -np.inf), np.zeros((len(q), 512)), big, size
    s, v = np.concatenate(logits, axis=1), np.concatenate(vals)
    mx = s.max(axis=1)
    safe = np.where(np.isneginf(mx), 0.0, mx)
    p = np.exp(s - safe[:, None])
    tot = p.sum(axis=1)
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.where(tot[:, None] > 0, p / tot[:, None], 0.0)
        lse = np.where(tot > 0, safe + np.log(tot), -np.inf)
    return p @ v, lse, p @ np.abs(v), big, size


def quantise_weights(w, group):
    """w [..., k] -> the values their codes stand for (float64)."""
    w = np.asarray(w, dtype=np.float64)
    x = w.reshape(w.shape[:-1] + (w.shape[-1] // group, group))
    s = bf16_values(bf16_bits(np.abs(x).max(axis=-1) / 7.0))[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        n = np.where(s > 0, np.clip(np.rint(x / s), -7, 7), 0.0)
    return (n * s).reshape(w.shape)
