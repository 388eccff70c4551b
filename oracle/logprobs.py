"""fp64 restatement of the token log probabilities: one row at a time in numpy."""
from __future__ import annotations

import numpy as np


def row(x, tokens, n_top: int, temperature: float):
    """(logprobs [n], entropy, top_ids [n_top], top_logprobs [n_top]) of logits x [vocab]."""
    x = np.asarray(x, np.float64)
    inside = [0 <= t < len(x) for t in tokens]
    if np.isnan(x).any() or np.isposinf(x).any():
        return np.full(len(tokens), np.nan), np.nan, np.full(n_top, -1), np.full(n_top, np.nan)
    order = np.argsort(-x, kind="stable")[:n_top]
    if np.isneginf(x).all():
        lp, entropy = x, 0.0
    else:
        z = (x - x.max()) / temperature
        lp = z - np.log(np.exp(z).sum())
        if np.exp(z).sum() < 1.5:                    # next to 1: from what is beside the largest
            at = int(np.argmax(x))
            lp = z - np.log1p(np.exp(np.delete(z, at)).sum())
        p = np.exp(lp)
        entropy = -(p[p > 0] * lp[p > 0]).sum()
    return np.array([lp[t] if ok else np.nan for t, ok in zip(tokens, inside)]), entropy, order, lp[order]
