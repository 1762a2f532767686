"""Plain 64-bit forms of the log-probability, policy loss and preference loss (tests only), and how far
binary32 arithmetic may be from them."""
from __future__ import annotations

import numpy as np

NO_TOKEN = -1


def log_softmax(z, allow, temperature):
    """z: float64 [n, v] (NaN counts as -inf); allow: bool [n, v].  -inf where the probability is zero."""
    z = np.where(allow & ~np.isnan(z), z, -np.inf)
    m = z.max(axis=1, keepdims=True, initial=-np.inf)
    with np.errstate(invalid="ignore", divide="ignore"):
        x = np.where(np.isinf(z), -np.inf, (z - np.where(np.isinf(m), 0.0, m)) / temperature)
        return x - np.log(np.exp(x).sum(axis=1, keepdims=True))


def token_logprobs(z, allow, tokens, temperature, weights=None):
    """(lp, takes part, log p of all tokens)."""
    n, v = z.shape
    logp = log_softmax(z, allow, temperature)
    if v == 0:
        lp = np.full(n, -np.inf)
    else:
        at = np.clip(tokens, 0, v - 1)
        lp = np.where((tokens >= 0) & (tokens < v), logp[np.arange(n), at], -np.inf)
    lp = np.where(np.isnan(lp) | (lp < np.finfo(np.float32).min), -np.inf, lp)       # what binary32 cannot hold is probability zero
    live = np.isfinite(lp)
    none = tokens == NO_TOKEN
    if weights is not None:
        none = none | (weights == 0)
    return np.where(none, 0.0, lp), live & ~none, logp


def gradient(logp, tokens, live, down, temperature):
    """down * d lp / d z, zero in rows that take no part."""
    with np.errstate(invalid="ignore"):
        g = -np.exp(np.where(np.isnan(logp), -np.inf, logp))
    n = len(tokens)
    g[np.arange(n)[live], tokens[live]] += 1.0
    return np.where(live[:, None], g * (np.where(live, down, 0.0) / temperature)[:, None], 0.0)


def policy(lp, live, old, ref, adv, weights, low, high, kl):
    """(loss, d loss / d lp, |w| times what an error of lp may do to a row's term or slope)."""
    x = np.where(live, lp, 0.0)
    r = np.exp(x - old)
    free, bound = r * adv, np.clip(r, 1.0 - low, 1.0 + high) * adv
    each = -np.minimum(free, bound)
    down = np.where(free <= bound, -free, 0.0)
    size = r * np.abs(adv)
    if kl:
        e = np.exp(ref - x)
        each = each + kl * (e - (ref - x) - 1.0)
        down = down + kl * (1.0 - e)
        size = size + abs(kl) * (e + 1.0 + np.abs(ref - x))
    w = np.where(live, weights, 0.0)
    each, down, size = (np.where(live, a, 0.0) for a in (each, down, size))       # (exp of the others may overflow)
    return float((w * each).sum()), w * down, np.abs(w) * size


def preference(lp, live, ref, begin, beta, smoothing):
    """(loss, rewards, d loss / d lp)."""
    n, pairs = len(lp), (len(begin) - 1) // 2
    over = np.where(live, np.where(live, lp, 0.0) - ref, 0.0)
    rewards = beta * np.array([over[a:b].sum() for a, b in zip(begin[:-1], begin[1:])])
    gap = rewards[0::2] - rewards[1::2]
    loss = float(np.mean((1.0 - smoothing) * np.logaddexp(0.0, -gap) + smoothing * np.logaddexp(0.0, gap))) if pairs else 0.0
    slope = -(1.0 - smoothing) / (1.0 + np.exp(gap)) + smoothing / (1.0 + np.exp(-gap))
    down = np.zeros(n)
    for k in range(2 * pairs):
        down[begin[k]:begin[k + 1]] = (slope[k // 2] if k % 2 == 0 else -slope[k // 2]) * beta / pairs
    return loss, rewards, down


# --------------------------------------------------------------------------- tolerances
# u = 2^-24.  A sum of exponentials is made of chains of at most 520 additions (a row of 131,072 tokens over 256 lanes)
# and a few joins, each off by u of the sum, and of exponentials whose argument x = (z - m) / T is off by 3 u |x| and whose
# value by 2 u: 520 u + (3 * 16 + 2) u = 3.4e-5 at the very most, where terms of |x| > 16 are below 2^-23 of the largest.
# The logarithm turns that into an absolute error; the token's own x adds 3 u |x|.
REL_SUM = 3.6e-5
U = 2.0 ** -24


def tol_lp(lp):
    return REL_SUM + 4 * U * np.abs(np.where(np.isfinite(lp), lp, 0.0))


def tol_gradient(g, logp, tokens, live, down, tol_down, temperature, bf16):
    """g = (down / T) (one - p): p is off by p (REL_SUM + 6 u |log p|) with the statistics' error in it, the difference and the
    product by u each, down by tol_down; then half a unit of the last place of the result's type."""
    with np.errstate(invalid="ignore"):
        p = np.exp(np.where(np.isnan(logp), -np.inf, logp))
        off = p * (2 * REL_SUM + 6 * U * np.where(p > 0, np.abs(logp), 0.0))
    one = np.zeros_like(p)
    one[np.arange(len(tokens))[live], tokens[live]] = 1.0
    scale = np.where(live, np.abs(down), 0.0)[:, None] / temperature
    tol = scale * (off + 4 * U * (one + p)) + (np.where(live, tol_down, 0.0)[:, None] / temperature) * np.abs(one - p)
    tol = tol + (2.0 ** -8 if bf16 else 2 * U) * (np.abs(g) + tol) + 1e-37 * scale + 1e-38
    return np.where(live[:, None], tol, 0.0)
