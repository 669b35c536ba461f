"""The next token by temperature, top-k, top-p and min-p, in plain 64-bit arithmetic, one row at a time."""
import numpy as np


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    x = np.asarray(logits, np.float64)
    real = np.flatnonzero(x > -np.inf)                                   # neither -inf nor NaN
    if not len(real):
        return 0
    order = real[np.lexsort((real, -x[real]))]                           # by logit, the lower index first of equals
    if not temperature > 0:
        return int(order[0])
    if top_k > 0:
        order = order[:top_k]
    with np.errstate(invalid="ignore"):
        w = np.where(x[order] == x[order[0]], 1.0, np.exp((x[order] - x[order[0]]) / temperature))
    if top_p < 1:
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        keep = before < max(top_p, 0.0) * w.sum()
        keep[0] = True
        order, w = order[keep], w[keep]
    if min_p > 0:
        keep = w >= min_p
        keep[0] = True
        order, w = order[keep], w[keep]
    by_index = np.argsort(order)
    sums = np.cumsum(w[by_index])
    u = min(max(u, 0.0), 1 - 2.0 ** -53) if u == u else 0.0
    return int(order[by_index][np.searchsorted(sums, u * sums[-1], side="right")])
