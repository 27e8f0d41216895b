"""Oracle of the cached-decoding operators: rotary tables and their
application, the paged 8-bit key/value cache, attention over it, and linears
with group-scaled 4-bit weights.

Values are float64 except where the definition fixes float32 steps (the
cache's scales and codes), which are reproduced step by step. Written per
sequence and per block, in plain loops.
"""

import numpy as np

SCALE_FLOOR = np.float32(2.0 ** -100)


def rope_frequencies(rot, theta, scaling="none", factor=1.0, original=0.0, beta_fast=32.0, beta_slow=1.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        # turns of pair i within the original length
        def pair(turns):
            return rot * np.log(original / (2 * np.pi * turns)) / (2 * np.log(theta))
        low, high = max(np.floor(pair(beta_fast)), 0), min(np.ceil(pair(beta_slow)), rot - 1)
        if high <= low:
            high = low + 1e-3
        mix = np.clip((i - low) / (high - low), 0, 1)
        f = f / factor * mix + f * (1 - mix)
    return f


def rope_table(positions, rot, theta, mscale=1.0, **scaling):
    a = np.arange(positions, dtype=np.float64)[:, None] * rope_frequencies(rot, theta, **scaling)
    return np.stack([np.cos(a), np.sin(a)], axis=-1) * mscale


def rope(x, pos, table, interleaved, inverse=False, dtype=np.float64):
    """x [T][heads][D]; table [positions][rot / 2][2]. With dtype float32 the
    products and the sum are rounded one by one."""
    rot = 2 * table.shape[1]
    x = x.astype(dtype)
    y = x.copy()
    c, s = (table[pos][:, None, :, k].astype(dtype) for k in (0, 1))
    if inverse:
        s = -s
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    a, b = x[..., first], x[..., second]
    y[..., first] = a * c - b * s
    y[..., second] = b * c + a * s
    return y


def append_block(codes, scale, kept, rows):
    """One block: codes [page][D] (integers in [-127, 127]) and its float32
    scale, `kept` rows stay, `rows` [m][D] float32 follow. Returns the new
    codes of rows 0 .. kept + m - 1 and the scale."""
    f = np.float32
    bad = not np.all(np.isfinite(rows)) or (kept > 0 and np.isnan(scale))
    if bad:
        return np.zeros((kept + len(rows), rows.shape[1]), np.int64), f(np.nan)
    top = f(np.abs(rows).max())
    s = max(f(scale) if kept else f(0), f(top / f(127)), SCALE_FLOOR)
    r = f(f(1) / s)
    new = np.clip(np.rint((rows.astype(f) * r).astype(f)), -127, 127).astype(np.int64)
    old = codes[:kept].astype(np.int64)
    if kept and s > scale:
        old = np.clip(np.rint((old.astype(f) * f(f(scale) / s)).astype(f)), -127, 127).astype(np.int64)
    return np.concatenate([old, new]), s


def append(codes, scales, page_table, past, rows, page):
    """In place for one sequence: codes [pages][Hkv][page][D] integers,
    scales [pages][Hkv] float32, rows [n][Hkv][D] float32."""
    n = len(rows)
    if n == 0:
        return
    for blk in range(past // page, (past + n + page - 1) // page):
        p = page_table[blk]
        lo, hi = max(past, blk * page), min(past + n, (blk + 1) * page)
        kept = lo - blk * page
        for h in range(codes.shape[1]):
            c, s = append_block(codes[p, h], scales[p, h], kept, rows[lo - past:hi - past, h])
            codes[p, h, :len(c)] = c
            scales[p, h] = s


def read(codes, scales, page_table, first, n, page):
    """Rows [n][Hkv][D] as float64 (the exact products)."""
    out = np.zeros((n, codes.shape[1], codes.shape[3]))
    for i in range(n):
        p, s = page_table[(first + i) // page], (first + i) % page
        out[i] = codes[p, :, s].astype(np.float64) * scales[p].astype(np.float64)[:, None]
    return out


def attention(q, k, v, scale, causal=False, key_mask=None):
    """One sequence: q [n][H][D], k, v [L][Hkv][D]. Returns out [n][H][D],
    lse [n][H], and for error bounds the mean magnitude sum_j p |v| / sum p
    [n][H][D] and the largest sum_d |q_d k_d| scale over the seen keys
    [n][H]."""
    n, H, D = q.shape
    L, Hkv = k.shape[:2]
    out, mag = np.zeros((n, H, D)), np.zeros((n, H, D))
    lse, size = np.full((n, H), -np.inf), np.zeros((n, H))
    for i in range(n):
        see = np.ones(L, bool) if key_mask is None else key_mask[:L] != 0
        if causal:
            see = see & (np.arange(L) <= L - n + i)
        if not see.any():
            continue
        for h in range(H):
            kk, vv = k[see, h // (H // Hkv)], v[see, h // (H // Hkv)]
            s = kk @ q[i, h] * scale
            m = s.max()
            p = np.exp(s - m)
            out[i, h] = p @ vv / p.sum()
            mag[i, h] = p @ np.abs(vv) / p.sum()
            lse[i, h] = m + np.log(p.sum())
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, lse, mag, size


def w4g_linear(x, codes, scales, bias=None):
    """x [L][K], codes [N][K] integers, scales [N][K / group]: the result and
    sum_k |x w|."""
    w = codes.astype(np.float64) * np.repeat(scales.astype(np.float64), codes.shape[1] // scales.shape[1], axis=1)
    x = x.astype(np.float64)
    y = x @ w.T
    size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, size = y + bias.astype(np.float64), size + np.abs(bias.astype(np.float64))
    return y, size


def window_sees(n, L, window, sinks, causal, key_mask=None):
    """[n][L]: which slots the n new tokens (the last of L) see through a
    window and the first `sinks` slots."""
    see = np.zeros((n, L), bool)
    for i in range(n):
        own = L - n + i
        for j in range(L):
            see[i, j] = (j > own - window or j < sinks) and (j <= own or not causal) and (key_mask is None or key_mask[j] != 0)
    return see


def attention_of(q, k, v, scale, see):
    """attention() for any see [n][L]; the same four results."""
    n, H, D = q.shape
    out, mag = np.zeros((n, H, D)), np.zeros((n, H, D))
    lse, size = np.full((n, H), -np.inf), np.zeros((n, H))
    G = H // k.shape[1]
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        for i in range(n):
            at = np.flatnonzero(see[i])
            if len(at) == 0:
                continue
            s = kk[at] @ q[i, h] * scale
            p = np.exp(s - s.max())
            out[i, h], mag[i, h] = p @ vv[at] / p.sum(), p @ np.abs(vv[at]) / p.sum()
            lse[i, h] = s.max() + np.log(p.sum())
            size[i, h] = (np.abs(kk[at]) @ np.abs(q[i, h])).max() * scale
    return out, lse, mag, size
