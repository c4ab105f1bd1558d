"""Plain form of tq_sample in numpy, in 64 bits."""
import math

import numpy as np


def sample(logits, noise, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, slack=0.0):
    """One row: (token, logprob).  `slack` moves the borders of top-p and min-p by that part."""
    x = np.asarray(logits, np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x[x == np.inf] = np.finfo(np.float32).max
    if not (x > -np.inf).any():
        return 0, -math.inf
    order = np.lexsort((np.arange(len(x)), -x))
    top = x[order[0]]
    lse = math.log(np.exp(x - top).sum())
    held = order[: top_k] if 0 < top_k < len(x) else order
    if not temperature > 0:
        held = held[:1]
    else:
        with np.errstate(over="ignore", divide="ignore"):
            w = np.where(x[held] > -np.inf, np.exp((x[held] - top) / temperature), 0)
        before = np.cumsum(w) - w
        first = np.arange(len(held)) == 0
        kept = first | (np.full(len(held), top_p >= 1) | (before < top_p * (1 + slack) * w.sum()))
        kept &= first | (w >= min_p * (1 + slack))
        held, w = held[kept & (w > 0)], w[kept & (w > 0)]
    if len(held) == 1:
        return int(held[0]), x[held[0]] - top - lse
    with np.errstate(divide="ignore"):
        quotient = w / np.asarray(noise, np.float64)[held]
    token = int(held[quotient == quotient.max()].min())
    return token, x[token] - top - lse
