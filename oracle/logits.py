"""Oracle of the rules on logits and of the choice of a token under them.

The definition fixes the float32 steps up to z and y, which are reproduced
step by step; probabilities are float64. Written per sequence, token by token
where a rule names it.
"""

import numpy as np

f32 = np.float32


def rules(x, params=(1, 1, 0, 0), history=(), biases=(), allowed=None):
    """x [V] float32, biases a list of (token, value), allowed [V] bool.
    Returns z and y [V] float32: the logits before and after the temperature,
    -inf where they are not allowed."""
    t, r, p, f = (f32(v) for v in params)
    z = x.astype(f32).copy()
    counts = {}
    for v in history:
        counts[int(v)] = counts.get(int(v), 0) + 1
    with np.errstate(all="ignore"):
        for v, c in counts.items():
            scaled = f32(z[v] / r) if z[v] > 0 else f32(z[v] * r)
            z[v] = f32(scaled - f32(f32(f * f32(c)) + p))
        for v, value in {int(v): value for v, value in biases}.items():      # the last entry of a token counts
            z[v] = f32(z[v] + f32(value))
        y = (z * f32(f32(1) / t)).astype(f32)
    if allowed is not None:
        z[~allowed], y[~allowed] = -np.inf, -np.inf
    return z, y


def pick(z, t, kind):
    """(token, confidence, ln sum e^(z / t), the largest |z - max| / t that
    weighs anything) of one row in float64."""
    z = z.astype(np.float64)
    if np.isnan(z).any():
        return int(np.flatnonzero(np.isnan(z))[0]), np.nan, np.nan, 0.0
    m = z.max()
    if m == -np.inf:
        return -1, 0.0, -np.inf, 0.0
    token = int(np.flatnonzero(z == m)[0])
    if m == np.inf:
        return token, np.nan, np.inf, 0.0
    w = np.float64(f32(1) / f32(t))
    seen = z > -np.inf
    d = (z[seen] - m) * w
    e = np.exp(d)
    total = e.sum()
    if kind == "probability":
        c = 1 / total
    elif kind == "margin":
        rest = np.delete(z, token)
        second = rest.max(initial=-np.inf)
        c = (1 - (np.exp((second - m) * w) if second > -np.inf else 0.0)) / total
    else:
        c = (e * d).sum() / total - np.log(total)
    return token, c, m * w + np.log(total), -d[d > -100].min(initial=0.0)
