"""Block summaries, scores and selection in 64 bits (test-only).

A block's summary holds, for every dim, the largest and smallest key of its
tokens in whole steps of 2^e, outwards; e is the smallest exponent >= -126 with
max|k| <= 127 * 2^e.  A query head is rounded to whole steps by the same rule.
A block's score for a KV head is the largest over the head's queries of
step_q * step_k * sum_d max(q8 hi, q8 lo); +inf if a key is not finite, a query
that is not finite counting as 0.  The first and last blocks are taken always,
then by score, of equal ones the lower index.
"""
from __future__ import annotations

import numpy as np


def exponent(top: np.ndarray) -> np.ndarray:
    e = np.full(top.shape, -126)
    for c in range(-126, 123):
        e = np.where(top > 127 * 2.0 ** e, c + 1, e)
    return e


def summary(keys: np.ndarray):
    """keys [L, H, D] of one request (fp64, what the cache stands for) ->
    hi, lo [n, H, D] and e [n, H]; e = 127 where a key is not finite."""
    L, H, D = keys.shape
    n = -(-L // 16)
    hi, lo, top = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H))
    fine = np.zeros((n, H), bool)
    for j in range(n):
        b = keys[16 * j:16 * j + 16]
        fine[j] = np.isfinite(b).all((0, 2))
        x = np.where(fine[j][None, :, None], b, 0.0)
        top[j], hi[j], lo[j] = np.abs(x).max((0, 2)), x.max(0), x.min(0)
    e = exponent(top)
    step = np.ldexp(1.0, e)[..., None]
    hi, lo, e = np.ceil(hi / step), np.floor(lo / step), np.where(fine, e, 127)
    return hi, lo, e


def scores(q: np.ndarray, keys: np.ndarray) -> np.ndarray:
    """q [Hq, D], keys [L, H, D] -> [H, n] (exact; fp32 holds every value)."""
    hi, lo, e = summary(keys)
    n, H, D = hi.shape
    G = q.shape[0] // H
    out = np.full((H, n), -np.inf)
    for h in range(q.shape[0]):
        g = h // G
        if np.isfinite(q[h]).all():
            eq = exponent(np.abs(q[h]).max())
            q8 = np.clip(np.rint(q[h] / 2.0 ** eq), -127, 127)
        else:
            eq, q8 = 0, np.zeros(D)
        s = np.maximum(q8 * hi[:, g], q8 * lo[:, g]).sum(1)
        s = np.where(e[:, g] == 127, np.inf, s * np.ldexp(1.0, np.where(e[:, g] == 127, 0, e[:, g]) + eq))
        out[g] = np.maximum(out[g], s)
    return out


def select(score: np.ndarray, top_k: int, n_first: int, n_last: int) -> np.ndarray:
    """score [H, n] -> [H, top_k], ascending, -1 behind."""
    H, n = score.shape
    sel = np.full((H, top_k), -1, np.int32)
    for g in range(H):
        keep = [i for i in range(n) if i < n_first or i >= n - n_last]
        rest = sorted((i for i in range(n) if i not in set(keep)), key=lambda i: (-score[g, i], i))
        keep = sorted((keep + rest)[:max(0, min(n, top_k))]) if n > top_k else list(range(n))
        sel[g, :len(keep)] = keep
    return sel
