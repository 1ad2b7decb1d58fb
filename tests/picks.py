"""What draws and largest logits are, a row at a time in 64 bits, from the definition (plain loops over the order of a row)."""
import math

import numpy as np


def order_of(z):
    """Ids of a row's tokens: larger logit first, of equal ones the lower id; -inf and NaN are none."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    ids = np.flatnonzero(z > -np.inf)
    return ids[np.lexsort((ids, -z[ids]))]


def logs_of(z, order, t):
    """Logarithms of the weights."""
    z = np.asarray(z, dtype=np.float64)[order]
    if z[0] == np.inf:
        return np.where(z == np.inf, 0.0, -np.inf)
    with np.errstate(over="ignore"):
        return (z - z[0]) / min(float(t), 3.4028234663852886e38)


def kept_of(z, t, k, p, m):
    """The kept ids in the row's order, with their weights. Settings are taken as the floats they are."""
    order = order_of(z)
    if not len(order):
        return order, np.zeros(0)
    if not t > 0:
        return order[:1], np.ones(1)
    x = logs_of(z, order, t)
    w, n = np.exp(x), len(order)
    if k > 0:
        n = min(n, k)
    if p < 1:
        upto = np.cumsum(w[:n])
        n = min(n, int(np.searchsorted(upto, max(p, 0.0) * upto[-1], side="left")) + 1)
    if m > 0:
        n = min(n, max(1, int((x >= math.log(m)).sum())))      # (weights next to 1 are 1 in 64 bits, their logarithms are not 0)
    return order[:n], w[:n]


def check_draw(z, u, t, k, p, m, token, logprob):
    """Whether a draw is what the definition gives. Weights are whole numbers of units of 2^-(62 - ceil(log2 V)), each off by half a unit: a sum of V of them is off by V / 2 units, less
    than 2^-(61 - 2 log2 V) of the largest weight, which is no more than the sum itself; 64-bit products and sums here by V 2^-53."""
    kept, w = kept_of(z, t, k, p, m)
    if not len(kept):
        return token == -1 and logprob == 0.0
    if not t > 0:
        return token == kept[0] and logprob == 0.0
    v = len(z)
    eps = 2.0 ** (2 * math.ceil(math.log2(max(2, v))) - 61) + v * 2.0 ** -52
    by_id = np.argsort(kept)
    ids, w = kept[by_id], w[by_id]
    total = w.sum()
    at = np.flatnonzero(ids == token)
    if not len(at) or w[at[0]] <= 0:
        return False
    i = at[0]
    u = 0.0 if not u > 0 else min(float(u), 1.0)
    before, upto = w[:i].sum() / total, w[:i + 1].sum() / total
    want = math.log(w[i] / total)
    return before - eps <= u and (u <= upto + eps) and abs(logprob - want) <= 2.0 ** -24 * abs(want) + 2 * eps


def near_draw(z, u, t, k, p, m, token, slack):
    """Whether a token is the draw from logits that make shares differ by a part `slack` of themselves: one that is kept, or next to the last that is, whose stretch is at most `slack` from u
    (sums up to it differ by that part; what is or is not kept at the border makes as much)."""
    kept, w = kept_of(z, t, k, p, m)
    order = order_of(z)
    more = order[:len(kept) + 2]                     # the border may lie a token further on
    weights = np.exp(logs_of(z, more, t))
    for last in {max(1, len(kept) - 1), len(kept), min(len(kept) + 1, len(order))}:
        by_id = np.argsort(more[:last])
        ids, share = more[:last][by_id], weights[:last][by_id] / weights[:last].sum()
        upto = np.cumsum(share)
        at = np.flatnonzero(ids == token)
        if len(at) and upto[at[0]] - share[at[0]] - slack <= u <= upto[at[0]] + slack:
            return True
    return False
