"""Draws and lists of the most likely tokens from their definitions, in 64 bits, one row at a time."""
import numpy as np

NO_TOKEN = -1
BORDER = 2.0 ** -40              # a number this near the border between two tokens may give either


def ordered(z, allow):
    """Ids of the allowed tokens by logit, the largest first, and by id; and their logits (NaN: -inf)."""
    ids = np.flatnonzero(allow)
    x = np.asarray(z, dtype=np.float64)[ids]
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    order = np.lexsort((ids, -x))
    return ids[order], x[order]


def weights(x, temperature):
    if temperature == 0:
        return (np.arange(len(x)) == 0).astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        w = np.exp((x - x[0]) / temperature)
    return np.where(x == x[0], 1.0, np.where(x == -np.inf, 0.0, w))


def kept(x, w, top_k, top_p, min_p):
    """How many tokens of the order stay."""
    n = len(x)
    if top_k and top_k < n:
        n = int(np.count_nonzero(x >= x[top_k - 1]))
    if top_p < 1:
        first = np.concatenate([[True], x[1:n] != x[:n - 1]])       # of its logit
        above = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])[first]
        stays = above < top_p * np.sum(w[:n])
        stays[0] = True
        n = int(np.count_nonzero(x[:n] >= x[:n][first][stays][-1]))
    return max(1, min(n, int(np.count_nonzero(w >= min_p))))


def draw(z, allow, u, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """{token: its log-probability} of the tokens that may be drawn: one but where u is at a border."""
    temperature, top_p, min_p, u = (float(np.float32(v)) for v in (temperature, top_p, min_p, u))
    ids, x = ordered(z, allow)
    if len(ids) == 0:
        return {NO_TOKEN: 0.0}
    if x[0] == -np.inf:
        return {int(ids[0]): -np.inf}
    if temperature == 0:
        return {int(ids[0]): 0.0}
    w = weights(x, temperature)
    n = kept(x, w, top_k, top_p, min_p)
    w = w[:n]
    upto = np.cumsum(w)
    total = upto[-1]
    target = min(max(u, 0.0), 1.0) * total
    last = int(np.flatnonzero(w)[-1])
    near = BORDER * total if u > 0 else 0.0              # at 1: any token from which on they weigh next to nothing
    lo, hi = (min(int(np.searchsorted(upto, t, side="right")), last) for t in (target - near, target + near))
    with np.errstate(divide="ignore"):
        return {int(ids[i]): float(np.log(w[i] / total)) for i in range(lo, hi + 1)}


def top(z, allow, k, temperature):
    """(ids, log-probabilities), k of each."""
    ids, x = ordered(z, allow)
    out, lp = np.full(k, NO_TOKEN, dtype=np.int64), np.full(k, -np.inf)
    if len(ids) == 0 or x[0] == -np.inf:
        return out, lp
    w = weights(x, temperature)
    n = min(k, int(np.count_nonzero(x > -np.inf)))
    out[:n] = ids[:n]
    with np.errstate(invalid="ignore"):
        lp[:n] = (x[:n] - x[0]) / temperature - np.log(np.sum(w)) if x[0] < np.inf else np.nan
    return out, lp
