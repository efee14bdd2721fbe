"""Plain implementations, in 64 bits, of switchsd_logprobs and switchsd_resample as include/switchsd_target.h defines them
(numpy, no shared code)."""
import math

import numpy as np

M64 = (1 << 64) - 1


def logprobs(x, temperature):
    """x [V] float64 logits of one position: (log probabilities [V], entropy, lse, tokens by rank)."""
    live = x > -np.inf  # (NaN is not)
    order = [int(v) for v in np.argsort(-np.where(live, x, -np.inf), kind="stable") if live[v]]
    if not order:
        return np.full(len(x), -np.inf), 0.0, -np.inf, order
    top = x[order[0]]
    if temperature == 0:
        lp = np.full(len(x), -np.inf)
        lp[order[0]] = 0
        return lp, 0.0, top, order
    z = np.where(live, x, -np.inf) / temperature
    lse = z.max() + math.log(np.exp(z - z.max()).sum())
    lp = z - lse
    p = np.exp(lp)
    return lp, -float((p[live] * lp[live]).sum()), lse, order


def _mix(z):
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def noise(seed, place, V):
    """ln E_v of the tokens of the appended position `place` = ctx_len + a."""
    key = _mix((int(seed) + (int(place) + 1) * 0x9E3779B97F4A7C15) & M64)
    r = []
    for n in range((V + 1) // 2):
        z = _mix((key + (n + 1) * 0x9E3779B97F4A7C15) & M64)
        r += [z & 0xFFFFFFFF, z >> 32]
    x = (np.array(r[:V], np.float64) + 0.5) / 2.0**32
    return np.log(-np.log1p(-x))


def accepted(p, q, u, n):
    for i in range(n):
        if not np.float32(np.float32(u[i]) * np.float32(q[i])) < np.float32(p[i]):
            return i
    return n


def weights(l, temperature, *, lse=0.0, skip=-1, lq=None, q_lse=0.0):
    """ln w of every token (temperature > 0)."""
    live = l > -np.inf
    y = np.where(live, l, -np.inf) / temperature - lse
    w = y.copy()
    if lq is not None:
        yq = np.where(lq > -np.inf, lq, -np.inf) / temperature - q_lse
        with np.errstate(divide="ignore"):
            w = np.log(np.maximum(np.exp(y) - np.exp(yq), 0))
    if skip >= 0:
        w[skip] = -np.inf
    return y if w.max() == -np.inf else w


def token(l, temperature, seed, place, **kw):
    if not (l > -np.inf).any():
        return -1
    if temperature == 0:
        return int(np.argmax(np.where(l > -np.inf, l, -np.inf)))
    return int(np.argmax(weights(l, temperature, **kw) - noise(seed, place, len(l))))
