"""The rollout's sampling distribution of a row, a draw from it and a log-prob's gradient, in fp64 numpy.

The words above -1e8, ordered by logit from the largest down and by index among equals; the first top_k; of these the
shortest prefix with the share top_p of their weights exp((z - max) / tau); of these the words of weight >= min_p.
Temperature 0 keeps the first word alone.
"""
import numpy as np

LIVE = -1e8


def kept(z, tau=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(indices of the kept words, ascending; their weights; the row's maximum).  No index for a row without one."""
    z = np.asarray(z, np.float64)
    live = np.flatnonzero(z > LIVE)
    if live.size == 0:
        return live, np.zeros(0), -np.inf
    order = live[np.argsort(-z[live], kind="stable")]
    top = z[order[0]]
    if tau == 0:
        return order[:1], np.ones(1), top
    if top_k > 0:
        order = order[:top_k]
    w = np.exp((z[order] - top) / tau)
    n = order.size
    if top_p < 1:
        cum = np.cumsum(w)
        n = min(n, int(np.argmax(cum >= top_p * cum[-1])) + 1)
    n = min(n, int((w >= min_p).sum()))
    order, w = order[:n], w[:n]
    by_index = np.argsort(order)
    return order[by_index], w[by_index], top


def draw(z, u, **settings):
    """(action, its log-prob, the number of kept words)."""
    at, w, _ = kept(z, **settings)
    if at.size == 0:
        return -1, -np.inf, 0
    cum = np.cumsum(w)
    over = np.flatnonzero(cum > u * cum[-1])
    i = over[0] if over.size else np.flatnonzero(w > 0)[-1]
    return int(at[i]), float(np.log(w[i] / cum[-1])), int(at.size)


def logp(z, action, **settings):
    """(log-prob of the action, the number of kept words, d logp / dz)."""
    z = np.asarray(z, np.float64)
    at, w, top = kept(z, **settings)
    d = np.zeros(z.size)
    i = np.searchsorted(at, action)
    if i >= at.size or at[i] != action:
        return -np.inf, int(at.size), d
    tau = settings.get("tau", 1.0)
    S = w.sum()
    if tau > 0:
        d[at] = -w / S / tau
        d[action] += 1.0 / tau
        return float((z[action] - top) / tau - np.log(S)), int(at.size), d
    return 0.0, 1, d
