"""fp64 restatement of what decides an eviction from the 8-bit cache, and of the eviction itself."""
from __future__ import annotations

import numpy as np


def weights(q, k, lse, scale: float, rows: int):
    """Weight that each of n tokens receives: q [rows, hq, hd] of the last rows, k [n, hk, hd], lse [rows, hq];
    returns (sum [hk, n], its bound's part: the terms times their relative error [hk, n])."""
    n, hk, hd = k.shape
    hq = q.shape[1]
    out, off = np.zeros((hk, n)), np.zeros((hk, n))
    for i in range(rows):
        seen = n - rows + i + 1
        if seen <= 0:
            continue
        for h in range(hq):
            if np.isinf(lse[i, h]):                  # no weight
                continue
            g = h // (hq // hk)
            s = k[:seen, g] @ q[i, h] * scale
            p = np.exp(s - lse[i, h])
            top = np.abs(q[i, h]).max()
            small = np.where(np.abs(q[i, h]) < top * 2.0 ** -9, 1.0, 0.0)
            err = abs(scale) * (2.0 ** -17 * top * (np.abs(k[:seen, g]) @ small) +
                                2.0 ** -16 * (np.abs(k[:seen, g]) @ np.abs(q[i, h])))
            err += 3 * 2.0 ** -24 * (np.abs(s) + abs(lse[i, h])) + 2.0 ** -22
            out[g, :seen] += p
            off[g, :seen] += p * err
    return out, off


def stay(n_tokens: int, keep: int, first: int, recent: int, room: int):
    n = min(max(keep, 0), n_tokens, room)
    recent = min(recent, n)
    return n, min(first, n - recent), recent


def kept(scores, n_tokens: int, keep: int, first: int, recent: int, room: int):
    """Places [n] of the tokens that stay, by their scores [>= n_tokens]."""
    n, first, recent = stay(n_tokens, keep, first, recent, room)
    lo, hi = first, n_tokens - recent
    middle = np.asarray(scores[lo:hi], np.float64)
    order = np.argsort(-np.where(np.isnan(middle), -np.inf, middle), kind="stable")
    isnan = np.isnan(middle)[order]
    order = np.concatenate((order[~isnan], order[isnan]))[:n - first - recent] + lo
    return np.sort(np.concatenate((np.arange(first), order, np.arange(n_tokens - recent, n_tokens)))).astype(np.int64)
