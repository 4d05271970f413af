"""Low-rank adapters beside a projection and dropout from a counter-based
generator, in float64.

TEST INFRASTRUCTURE (oracle); see ``oracle/__init__``.

Dropout of a [rows, k] matrix: element (i, j) has a 16-bit draw, half j % 2
(low first) of word (j % 8) // 2 of Philox4x32-10 under the key (seed mod
2^32, seed >> 32) and the counter (g mod 2^32, g >> 32, offset mod 2^32,
offset >> 32) with g = i ceil(k / 8) + j // 8.  It is kept when the draw is at
least T = p 65536 rounded to nearest; kept elements are multiplied by
65536 / (65536 - T).

Adapters: row i has adapter l = index[i], none outside [0, adapters).  With
A_l, B_l cut to the first ranks[l] of the rank, s_l and the dropped, scaled
x~ = dropout(x):
  t_i = x~_i A_l^T, out_i = c_i + s_l t_i B_l^T;
  u_i = s_l dy_i B_l, dx_i = dx_in_i + dropout'(u_i A_l),
  dA_l = sum_i u_i^T x~_i, dB_l = s_l sum_i dy_i^T t_i.
"""
from __future__ import annotations

import numpy as np

from . import philox


def threshold(p: float) -> int:
    return int(np.rint(p * 65536.0))


def draws(rows: int, k: int, seed: int, offset: int, row_index=None) -> np.ndarray:
    """uint32 [rows, k] draws in [0, 65536); ``row_index`` picks rows of a
    larger matrix."""
    groups = -(-k // 8)
    r = np.arange(rows, dtype=np.uint64) if row_index is None else np.asarray(row_index, np.uint64)
    g = (r[:, None] * np.uint64(groups) + np.arange(groups, dtype=np.uint64)[None, :]).reshape(-1)
    low = np.uint64(0xFFFFFFFF)
    counter = np.stack([g & low, g >> np.uint64(32),
                        np.full_like(g, offset & 0xFFFFFFFF),
                        np.full_like(g, (offset >> 32) & 0xFFFFFFFF)], axis=-1)
    key = np.array([seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF], dtype=np.uint64)
    words = philox.philox4x32(counter, key).reshape(-1, 4)
    halves = np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], axis=-1)
    return halves.reshape(len(r), groups * 8)[:, :k]


def factors(rows: int, k: int, p: float, seed: int, offset: int, row_index=None) -> np.ndarray:
    """float64 [rows, k]: 0 where dropped, 1 / (1 - p) where kept."""
    t = threshold(p)
    kept = draws(rows, k, seed, offset, row_index) >= t
    return np.where(kept, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)


def dropout(x, p, seed=0, offset=0, residual=None):
    x = np.asarray(x, np.float64)
    f = factors(*x.shape, p, seed, offset)
    y = np.where(f != 0, x, 0.0) * f
    return y if residual is None else y + np.asarray(residual, np.float64)


def _cut(a, b, ranks, l):
    r = a.shape[1] if ranks is None else min(max(int(ranks[l]), 0), a.shape[1])
    return np.asarray(a[l, :r], np.float64), np.asarray(b[l, :, :r], np.float64), r


def forward(x, a, b, index, c=None, scaling=None, ranks=None, p=0.0, seed=0, offset=0):
    """(out [m, n], t [m, rank])."""
    m, n, rank = x.shape[0], b.shape[1], a.shape[1]
    xd = dropout(x, p, seed, offset)
    out = np.zeros((m, n)) if c is None else np.array(c, np.float64)
    t = np.zeros((m, rank))
    for l in range(a.shape[0]):
        rows = np.flatnonzero(np.asarray(index) == l)
        al, bl, r = _cut(a, b, ranks, l)
        t[rows, :r] = xd[rows] @ al.T
        out[rows] += (1.0 if scaling is None else float(scaling[l])) * (t[rows, :r] @ bl.T)
    return out, t


def backward(dy, x, t, a, b, index, dx=None, scaling=None, ranks=None, p=0.0, seed=0, offset=0):
    """(dx [m, k], dA, dB); ``t`` as the forward pass kept it."""
    m, k = x.shape
    xd = dropout(x, p, seed, offset)
    f = factors(m, k, p, seed, offset)
    dy = np.asarray(dy, np.float64)
    t = np.asarray(t, np.float64)
    dx = np.zeros((m, k)) if dx is None else np.array(dx, np.float64)
    da, db = np.zeros(a.shape), np.zeros(b.shape)
    for l in range(a.shape[0]):
        rows = np.flatnonzero(np.asarray(index) == l)
        al, bl, r = _cut(a, b, ranks, l)
        s = 1.0 if scaling is None else float(scaling[l])
        u = s * (dy[rows] @ bl)
        dx[rows] += np.where(f[rows] != 0, u @ al, 0.0) * f[rows]
        da[l, :r] = u.T @ xd[rows]
        db[l, :, :r] = s * (dy[rows].T @ t[rows, :r])
    return dx, da, db
