"""CPU float64 definitions of attention over packed prompts and of the 4-bit key format.  numpy only; shares no code with
the GPU path."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
# scale bytes 0 .. 0xe2: a float16 without its sign and its lower seven bits
SCALES = np.array([m / 8 * 2.0 ** -14 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 15) for e in range(1, 32) for m in range(8)])[:0xe3]


def fp4_quantise(x):
    """Rows [n, d] -> (codes [n, d] 0..15, scale bytes [n, ceil(d / 32)])."""
    n, d = x.shape
    g = (d + 31) // 32
    codes, scales = np.zeros((n, d), dtype=np.uint8), np.zeros((n, g), dtype=np.uint8)
    for r in range(n):
        for i in range(g):
            k = x[r, 32 * i:32 * i + 32].astype(np.float64)
            if not np.isfinite(k).all():
                scales[r, i] = 0xff
                continue
            fits = np.nonzero(6 * SCALES >= np.abs(k).max())[0]
            scales[r, i] = fits[0] if len(fits) else 0xe2
            s = SCALES[scales[r, i]]
            for j, v in enumerate(k):
                gap = np.abs(min(abs(v), 6 * s) - MAGNITUDES * s)       # (beyond the largest value the nearest is that one)
                near = np.nonzero(gap == gap.min())[0]
                c = int(near[0]) if len(near) == 1 or s == 0 else int([m for m in near if m % 2 == 0][0])
                codes[r, 32 * i + j] = c + (8 if v < 0 and c else 0)
    return codes, scales


def fp4_values(codes, scales):
    """What the codes and scale bytes stand for, [n, d]."""
    s = np.where(scales == 0xff, np.nan, SCALES[np.minimum(scales, 0xe2)])
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def fp4_storage(codes, scales):
    """The storage of consecutive rows: code bytes padded to 16, then scale bytes padded to 16."""
    n, d = codes.shape
    pc, ps = (d // 2 + 15) // 16 * 16, (scales.shape[1] + 15) // 16 * 16
    a, b = np.zeros((n, pc), dtype=np.uint8), np.zeros((n, ps), dtype=np.uint8)
    a[:, :d // 2] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    b[:, :scales.shape[1]] = scales
    return np.concatenate([a.reshape(-1), b.reshape(-1)])


def turned(x, pos, theta):
    """x [T, heads, d_k] rotated to positions pos [T] (pair (j, j + d_k/2) by -pos theta^(-2j/d_k))."""
    x = x.astype(np.float64)
    if not theta:
        return x
    half = x.shape[-1] // 2
    a = np.asarray(pos, dtype=np.float64)[:, None, None] * theta ** (-np.arange(half) / half)
    x1, x2 = x[..., :half], x[..., half:]
    return np.concatenate([x1 * np.cos(a) + x2 * np.sin(a), x2 * np.cos(a) - x1 * np.sin(a)], -1)


def attention(q, k, v, theta, causal):
    """One sequence: q [nq, H, d_k], k, v [nk, KV, d_k].  Returns (o [nq, H, d_k], sum_j p |v|, largest sum |q||k| / sqrt(d_k) of a row)."""
    nq, H, dk = q.shape
    nk, kv = k.shape[:2]
    o, pv, qk = np.zeros((nq, H, dk)), np.zeros((nq, H, dk)), np.zeros((nq, H))
    if nq == 0 or nk == 0:
        return o, pv, qk
    with np.errstate(invalid="ignore", over="ignore"):
        qr, kr = turned(q, np.arange(nq) + nk - nq, theta), turned(k, np.arange(nk), theta)
        for h in range(H):
            g = h * kv // H
            s = qr[:, h] @ kr[:, g].T / np.sqrt(dk)
            mag = np.abs(qr[:, h]) @ np.abs(kr[:, g]).T / np.sqrt(dk)
            for i in range(nq):
                n = max(0, min(nk, i + 1 + nk - nq)) if causal else nk
                if n == 0:
                    continue
                p = np.exp(s[i, :n] - s[i, :n].max())
                p /= p.sum()
                o[i, h], pv[i, h], qk[i, h] = p @ v[:n, g].astype(np.float64), p @ np.abs(v[:n, g].astype(np.float64)), mag[i, :n].max()
    return o, pv, qk
