"""Plain 64-bit statements (numpy) of the operators around the key/value cache: which tokens a query sees, what they receive, which
of them stay, and rotary positions."""
from __future__ import annotations

import numpy as np


def attention(q, k, v, seen, scale):
    """q [n_q, Hq, D], k, v [n, H, D], seen [n_q, n]: out, lse, the largest sum of |q k| scale of a row, sum p |v|, p [n_q, Hq, n]."""
    G = q.shape[1] // k.shape[1]
    n = k.shape[0]
    kk, vv = np.repeat(k, G, 1), np.repeat(v, G, 1)
    s = np.einsum("ihd,thd->iht", q, kk) * scale
    mag = (np.einsum("ihd,thd->iht", np.abs(q), np.abs(kk)) * abs(scale)).max(-1) if n else np.zeros(q.shape[:2])
    s = np.where(seen[:, None, :], s, -np.inf)
    top = s.max(-1, initial=-np.inf)
    ref = np.where(np.isfinite(top), top, 0)
    p = np.exp(s - ref[..., None])
    total = p.sum(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.where(total[..., None] > 0, p / np.where(total > 0, total, 1)[..., None], 0)
        lse = np.where(total > 0, ref + np.log(total), -np.inf)
    return np.einsum("iht,thd->ihd", p, vv), lse, mag, np.einsum("iht,thd->ihd", p, np.abs(vv)), p


def causal(n, n_q):
    return np.arange(n)[None, :] <= (n - n_q + np.arange(n_q))[:, None]


def in_window(n, n_q, window, sinks):
    at, t = (n - n_q + np.arange(n_q))[:, None], np.arange(n)[None, :]
    return (t <= at) & ((t > at - window) | (t < sinks))


def evict(mass, lens, src, keep, first, recent, max_len, room):
    """Lists of the tokens that stay, ascending."""
    rows, ldm = mass.shape
    got = []
    for a, k in zip(src, keep):
        n = max(0, min(lens[a], max_len, ldm)) if 0 <= a < rows else 0
        k = max(0, min(k, room, n))
        order = list(range(n - 1, max(n - recent, 0) - 1, -1)) + [t for t in range(min(first, n)) if t < n - recent]
        free = np.ones(n, bool)
        free[order] = False
        rest = np.flatnonzero(free)
        m = mass[a, rest].astype(np.float64) if n else np.zeros(0)
        rest = rest[np.lexsort((rest, np.where(np.isnan(m), 0, -m), np.isnan(m)))]
        got.append(sorted((order + rest.tolist())[:k]))
    return got


def rotary(x, positions, axis_of, freq, neighbours):
    """x [rows, heads, D] in 64 bits -> turned; pairs 0 .. len(freq) - 1."""
    half = len(freq)
    i = np.arange(half)
    lo, hi = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
    angle = positions.astype(np.float64)[axis_of].T * freq.astype(np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y = x.copy()
    y[..., lo], y[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
    return y
