"""Log-prob of an action, entropy and likeliest words of a row at a temperature, and their gradient, in fp64 numpy.

The words are the logits above -1e8; the likeliest come first, the lowest index first among equals.
"""
import numpy as np

LIVE = -1e8


def row(z, act, n, tau=1.0):
    """(log-prob of act, entropy, ids [n], their log-probs [n], every word's log-prob [V], -inf where masked)."""
    z = np.asarray(z, np.float64)
    live = np.flatnonzero(z > LIVE)
    lp = np.full(z.size, -np.inf)
    ids, top = np.full(n, -1, np.int64), np.full(n, -np.inf)
    entropy = 0.0
    if live.size:
        x = (z[live] - z[live].max()) / tau
        lp[live] = x - np.log(np.exp(x).sum())
        entropy = -(np.exp(lp[live]) * lp[live]).sum()
        order = live[np.argsort(-z[live], kind="stable")][:n]
        ids[:order.size], top[:order.size] = order, lp[order]
    return (lp[act] if 0 <= act < z.size else 0.0), entropy, ids, top, lp


def gradient(lp, entropy, act, ids, dlogp, dentropy, dtop, tau=1.0):
    """d(dlogp log p(act) + dentropy H + sum_j dtop_j log p(ids_j)) / dz, from row()'s results."""
    c = np.zeros(lp.size)
    live = lp > -np.inf
    if 0 <= act < lp.size and live[act]:
        c[act] += dlogp
    for i, e in zip(ids, dtop):
        if i >= 0:
            c[i] += e
    d = np.zeros(lp.size)
    d[live] = (c[live] - np.exp(lp[live]) * (c.sum() + dentropy * (lp[live] + entropy))) / tau
    return d
