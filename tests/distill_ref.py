"""The distillation loss and its gradient from their definition, in 64 bits, one row at a time."""
import numpy as np

F32_MAX = float(np.finfo(np.float32).max)


def row(z, allow, ids, values, temperature, tail):
    """(loss, gradient of one row by its logits), without its weight."""
    v = len(z)
    c = 1.0 / float(np.float32(temperature))
    z = np.asarray(z, dtype=np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    on = np.asarray(allow, dtype=bool) & (z > -np.inf)
    grad = np.zeros(v)
    inside = (ids >= 0) & (ids < v)
    at = np.where(inside, ids, 0)
    live = inside & np.isfinite(values) & (on[at] if v else False)
    if not live.any():
        return 0.0, grad
    if np.isinf(z[on]).any():
        return np.nan, np.full(v, np.nan)
    top = z[on].max()
    x = np.full(v, -np.inf)
    with np.errstate(over="ignore", under="ignore"):
        x[on] = (z[on] - top) * c
        lp = x - np.log(np.sum(np.exp(x[on])))
        named = np.zeros(v, dtype=bool)
        named[at[live]] = True
        counts = live & (np.where(live, lp[at], -np.inf) >= -F32_MAX)
        a = np.where(counts, values.astype(np.float64), -np.inf)
        if tail:
            q = np.exp(np.minimum(a, 0.0))
        elif counts.any():
            q = np.exp(a - a.max())
            q /= q.sum()
        else:
            q = np.zeros(len(ids))
        others = on & ~named
        rest = max(0.0, 1.0 - q.sum()) if tail and others.any() else 0.0
        teacher = np.zeros(v)
        np.add.at(teacher, at[counts], q[counts])
        loss = sum(t * (np.log(t) - lp[i]) for t, i, k in zip(q, at, counts) if k and t > 0)
        if rest > 0:
            most = x[others].max()
            share = np.exp(x[others] - most)
            ln_tail = most + np.log(share.sum()) - np.log(np.sum(np.exp(x[on])))
            loss += rest * (np.log(rest) - ln_tail)
            teacher[others] += rest * share / share.sum()
        p = np.where(on, np.exp(lp), 0.0)
    grad[on] = c * (p[on] * (q.sum() + rest) - teacher[on])
    return loss, grad


def loss(z, allow, ids, values, weights, temperature, tail):
    """(loss, losses, gradient, size of what the gradient is the difference of)."""
    losses, grads, size = [], [], []
    for i in range(len(z)):
        l, g = row(z[i], allow[i], ids[i], values[i], temperature, tail) if weights[i] != 0 else (0.0, np.zeros(z.shape[1]))
        losses.append(l)
        grads.append(weights[i] * g if weights[i] != 0 else g)
    losses = np.array(losses, dtype=np.float64)
    return float(np.sum(weights * losses)) if len(losses) else 0.0, losses, np.array(grads).reshape(z.shape)
