"""fp64 CPU oracle for the operators of a training step: norms of queries and keys with the position rotation, the balance
loss of the gates, dropout.

TEST INFRASTRUCTURE ONLY (same rules as switchhead_oracle.py: nothing in the product imports it).  Written from the formulas
in include/switchhead.h, one row at a time where that is the definition; the Philox generator from Salmon, Moraes, Dror and
Shaw, "Parallel random numbers: as easy as 1, 2, 3" (2011), on Python integers.
"""
from __future__ import annotations

import numpy as np


def rotate(v, positions, base, rotated, halves, back=False):
    """v [B, T, H, D], positions [B, T]: pairs of the first `rotated` columns turned by position * base^(-2i/rotated)."""
    out = np.array(v, dtype=np.float64)
    for i in range(rotated // 2):
        a, b = (i, i + rotated // 2) if halves else (2 * i, 2 * i + 1)
        ang = np.asarray(positions, dtype=np.float64) * float(base) ** (-2.0 * i / rotated)
        c, s = np.cos(ang)[..., None], np.sin(ang)[..., None] * (-1.0 if back else 1.0)
        out[..., a], out[..., b] = v[..., a] * c - v[..., b] * s, v[..., a] * s + v[..., b] * c
    return out


def qk_norm(x, gain, positions, eps, base=10000.0, rotated=0, halves=False, scale=1.0):
    x = np.asarray(x, dtype=np.float64)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        n = n * np.asarray(gain, dtype=np.float64)
    return scale * rotate(n, positions, base, rotated, halves)


def qk_norm_backward(x, dy, gain, positions, eps, base=10000.0, rotated=0, halves=False, scale=1.0):
    """Gradients with respect to x and the gain of sum(qk_norm(x) * dy)."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    D = x.shape[-1]
    g = np.ones(D) if gain is None else np.asarray(gain, dtype=np.float64)
    size = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = scale * rotate(dy, positions, base, rotated, halves, back=True)
    dgain = (u * x / size).reshape(-1, D).sum(0)
    dx = g * u / size - x * (g * u * x).sum(-1, keepdims=True) / (D * size ** 3)
    return dx, dgain


def balance(logits, idx, kind, coef, mask=None, gloss=1.0):
    """logits [N, S, H, E], idx [S, N, H, k], mask [N].  Returns loss, counts, prob, dlogits."""
    z = np.asarray(logits, dtype=np.float64)
    N, S, H, E = z.shape
    keep = np.ones(N, dtype=bool) if mask is None else np.asarray(mask).astype(bool)
    p = np.zeros_like(z)
    counts = np.zeros((S, H, E), dtype=np.int64)
    for t in np.nonzero(keep)[0]:
        for s in range(S):
            for h in range(H):
                row = z[t, s, h]
                if np.isnan(row).any() or not (row == -np.inf).all():
                    with np.errstate(invalid="ignore"):
                        e = np.exp(row - row.max())
                        p[t, s, h] = e / e.sum()
                for j in idx[s, t, h]:
                    if 0 <= j < E:
                        counts[s, h, j] += 1
    n = int(keep.sum())
    loss, slope = 0.0, np.zeros((S, H, E))
    P = p.sum(0) / max(n, 1)
    if n:
        for s in range(S):
            for h in range(H):
                if kind == "counts":
                    f = counts[s, h] / max(counts[s, h].sum(), 1)
                    loss += coef * E * (f * P[s, h]).sum()
                    slope[s, h] = coef * E * f
                else:
                    used = P[s, h] != 0
                    loss += coef * (P[s, h][used] * np.log(P[s, h][used])).sum()
                    slope[s, h][used] = coef * (np.log(P[s, h][used]) + 1.0)
    dz = gloss * p * (slope - (p * slope).sum(-1, keepdims=True)) / max(n, 1)
    dz[~keep] = 0.0
    return loss, counts, P, dz


def philox4x32_10(counter, key):
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_kept(rows, cols, seed, offset, p, first_row=0):
    """The mask [rows, cols] of rows first_row .. first_row + rows - 1, and the factor of what is kept."""
    limit = int(round(p * 65536))
    seed, offset = int(seed) & (2 ** 64 - 1), int(offset) & (2 ** 64 - 1)
    kept = np.zeros((rows, cols), dtype=bool)
    for r in range(rows):
        for b in range((cols + 7) // 8):
            words = philox4x32_10((b, first_row + r, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
            bits = [(w >> (16 * half)) & 0xFFFF for w in words for half in (0, 1)]
            n = min(8, cols - 8 * b)
            kept[r, 8 * b:8 * b + n] = np.array(bits[:n]) >= limit
    return kept, 65536.0 / (65536 - limit) if limit < 65536 else 0.0
