"""The cached-decoding operators against oracle/decode.py.

Tolerances (u = the output type's unit roundoff: 2^-24, 2^-11, 2^-8):
- Rotary tables: float64 with one rounding: 2^-24 m, plus 1e-9 for the
  float64 angles of different pow implementations.
- Rotation: two float32 products and a sum, 3 2^-24 (|a c| + |b s|), and one
  rounding u |y|.
- Cache codes and scales: the definition fixes every float32 step, so they
  are bit-exact; reading in float32 is one product, bit-exact.
- Attention against float64 on the same codes: a score's float32 sum of D
  products is off by at most d = D 2^-24 S, S the largest sum of magnitudes
  (times the softmax scale), and its products with the scales by 4 2^-24 of
  it, so a weight is off by e^d - 1 <= 2 d + 2^-20 relative (exponential
  2^-22), and by 2^-11 where it is rounded to fp16. A weighted mean of
  magnitude A is then off by at most A (2 (2 d + 2^-20) + 2^-11 + L 2^-24 +
  2^-20), L keys summed in float32, plus one rounding of the output; the
  log-sum-exp by 2 d + L 2^-24 + 2^-19 (1 + |lse|). Where weights lie many
  orders of magnitude apart a channel may owe its value to the smallest
  alone, and fp16's smallest step counts: a row's largest weight times scale
  is held as at least 2^7, so each of L is off by up to 2^-25 of 2^7 of the
  largest, 2^-32 L 127 max_j p_j s_v(j) in all.
- 4-bit linears: (K / 8 + 16) 2^-24 sum |x w| for the float32 sums (an MMA
  adds 16 products, a block's sums are added once more), and one rounding.
"""

import numpy as np
import pytest
import torch

from oracle import decode as od
from oracle import sgat as osg

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -149}
i32 = lambda v: torch.tensor(np.asarray(v, dtype=np.int32).reshape(-1), device="cuda")
num = lambda t: t.detach().double().cpu().numpy()


def randn(rng, shape, dtype):
    """A tensor of the type and its exact values in float64."""
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda()
    return t, num(t)


# --------------------------------------------------------------------------
# Rotary positions
# --------------------------------------------------------------------------
@pytest.mark.parametrize("rot,theta,kw", [
    (128, 1e4, dict()), (64, 1e6, dict(scaling="linear", factor=4.0)), (2, 1e4, dict()),
    (96, 1e4, dict(scaling="ntk", factor=8.0)), (128, 1e4, dict(scaling="parts", factor=16.0, original=4096.0)),
    (64, 5e5, dict(scaling="parts", factor=2.5, original=1000.0, beta_fast=16.0, beta_slow=2.0))])
def test_rope_table(abi, rot, theta, kw):
    P = 9001
    t = torch.empty(P, rot // 2, 2, device="cuda")
    abi.rope_table(t, theta, **kw)
    m = 0.1 * np.log(kw["factor"]) + 1 if kw.get("scaling") == "parts" else 1.0
    ref = od.rope_table(P, rot, theta, m, **kw)
    assert np.all(np.abs(num(t) - ref) <= 2.0 ** -24 * m + 1e-9)
    abi.rope_table(t, theta, mscale=1.5, **kw)
    assert np.all(np.abs(num(t) - ref * (1.5 / m)) <= 2.0 ** -24 * 1.5 + 1e-9)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L,heads,D,rot,pad,inter", [
    (37, 5, 128, 128, 0, False), (37, 6, 128, 128, 8, True), (1, 1, 64, 64, 0, False), (19, 9, 64, 32, 16, True),
    (64, 3, 80, 48, 0, False), (11, 4, 40, 18, 0, True), (7, 2, 96, 96, 3, False), (5, 2, 10, 0, 0, False)])
@pytest.mark.parametrize("inverse,in_place", [(False, False), (True, False), (False, True)])
def test_rope_apply(abi, dtype, L, heads, D, rot, pad, inter, inverse, in_place):
    rng = np.random.default_rng(L * 100 + D + rot)
    table = torch.from_numpy(od.rope_table(300, max(rot, 2), 1e4, 1.25).astype(np.float32)).cuda()[:, : rot // 2] \
        .contiguous()
    x, xn = randn(rng, (L, heads * D + pad), dtype)
    y = x if in_place else torch.full((L, heads * D + 2 * pad), 7.0, dtype=dtype, device="cuda")
    pos = rng.integers(0, 300, L)
    abi.rope_apply(x, heads, i32(pos), table, y, D=D, interleaved=inter, inverse=inverse)
    abi.check_status()
    xh = xn[:, : heads * D].reshape(L, heads, D)
    t64 = num(table)
    ref = od.rope(xh, pos, t64, inter, inverse)
    size = od.rope(np.abs(xh), pos, np.abs(t64) * [1, -1], inter)       # |a c| + |b s| in the first of a pair
    size = np.maximum(size, od.rope(np.abs(xh), pos, np.abs(t64), inter))
    got = num(y)[:, : heads * D].reshape(L, heads, D)
    assert np.all(np.abs(got - ref) <= 3 * 2.0 ** -24 * np.abs(size) + U[dtype] * np.abs(ref) + TINY[dtype])
    assert np.array_equal(got[..., rot:], xh[..., rot:])                # the other channels are copied
    assert np.array_equal(num(y)[:, heads * D:], xn[:, heads * D:] if in_place else np.full((L, 2 * pad), 7.0))


def test_rope_gradient(abi):
    """The transposed map is the gradient: against the formula (float64
    autograd) and against differences of the forward pass in float32."""
    rng = np.random.default_rng(3)
    L, heads, D, rot = 5, 3, 64, 32
    table = torch.from_numpy(od.rope_table(50, rot, 1e4, 1.2).astype(np.float32)).cuda()
    pos = i32(rng.integers(0, 50, L))
    x, _ = randn(rng, (L, heads * D), torch.float32)
    w, wn = randn(rng, (L, heads * D), torch.float32)
    for inter in (False, True):
        g = torch.empty_like(x)
        abi.rope_apply(w, heads, pos, table, g, interleaved=inter, inverse=True)
        ref = od.rope(wn.reshape(L, heads, D), pos.cpu().numpy(), num(table), inter, inverse=True)
        assert np.all(np.abs(num(g).reshape(ref.shape) - ref) <= 2.0 ** -21 * (1 + np.abs(ref)))
        f = lambda z: float((num(z) * wn).sum())
        y0, y1 = torch.empty_like(x), torch.empty_like(x)
        for at in [(0, 0), (1, 17), (2, 31), (3, 40), (4, 64 + 5), (0, 128 + 30)]:
            lo, hi = x.clone(), x.clone()
            lo[at] -= 0.5
            hi[at] += 0.5
            abi.rope_apply(lo, heads, pos, table, y0, interleaved=inter)
            abi.rope_apply(hi, heads, pos, table, y1, interleaved=inter)
            # the map is linear: a difference of 1 (up to the rounding of lo and hi) gives the derivative
            step = float(hi[at].double() - lo[at].double())
            assert abs((f(y1) - f(y0)) / step - float(g[at])) <= 1e-5 * np.abs(wn).sum() ** 0.5


def test_rope_position_outside_the_table(abi):
    x = torch.ones(4, 64, dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    table = torch.zeros(10, 32, 2, device="cuda")
    for bad in (10, -1):
        abi.rope_apply(x, 1, i32([0, 1, bad, 9]), table, y)
        with pytest.raises(abi.StarqError) as e:
            abi.check_status()
        assert e.value.code == abi.ERR_RANGE
    abi.check_status()


# --------------------------------------------------------------------------
# The cache
# --------------------------------------------------------------------------
class Paged:
    """A cache with scattered pages on both sides (GPU, oracle)."""

    def __init__(self, abi, rng, B, most, Hkv, page, D, stale=True):
        self.page, self.Hkv, self.D = page, Hkv, D
        width = max(1, (most + page - 1) // page)
        self.pages = B * width + 2
        self.table = rng.permutation(self.pages)[: B * width].reshape(B, width)
        self.cache = abi.KVCache.empty(self.pages, Hkv, page, D)
        if stale:                                     # what an earlier user of the pages left
            shape = (self.pages, Hkv, page, D)
            self.cache.K.copy_(torch.from_numpy(rng.integers(1, 256, shape).astype(np.uint8)))
            self.cache.V.copy_(torch.from_numpy(rng.integers(1, 256, shape).astype(np.uint8)))
            self.cache.k_scale.fill_(float("nan"))
            self.cache.v_scale.fill_(float("inf"))
        self.k, self.v = (t.cpu().numpy().astype(np.int64) - 128 for t in (self.cache.K, self.cache.V))
        self.ks, self.vs = self.cache.k_scale.cpu().numpy(), self.cache.v_scale.cpu().numpy()
        self.dev_table = torch.tensor(self.table, dtype=torch.int32, device="cuda")

    def check(self, past, new):
        """The rows that the sequences hold are the oracle's, bit for bit."""
        for codes, ref, scale, rs in ((self.cache.K, self.k, self.cache.k_scale, self.ks),
                                      (self.cache.V, self.v, self.cache.v_scale, self.vs)):
            codes, scale = codes.cpu().numpy().astype(np.int64) - 128, scale.cpu().numpy()
            assert np.array_equal(scale, rs, equal_nan=True)
            for b in range(len(past)):
                for s in range(past[b] + new[b]):
                    p = self.table[b, s // self.page]
                    assert np.array_equal(codes[p, :, s % self.page], ref[p, :, s % self.page]), (b, s)


def append_both(abi, rng, pg, past, new, H, dtype, rot, inter, pos=None, loud=1.0):
    """One append on both sides; returns the rows that went in."""
    T, w, D = sum(new), pg.Hkv * pg.D, pg.D
    start = np.concatenate([[0], np.cumsum(new)])
    x, xn = randn(rng, (T, H * D + 2 * w + 8), dtype)
    x *= loud
    xn = num(x)
    q, k, v = x[:, : H * D], x[:, H * D: H * D + w], x[:, H * D + w: H * D + 2 * w]
    if pos is None:
        pos = np.concatenate([np.arange(p, p + n) for p, n in zip(past, new)]).astype(np.int64)
    table = torch.from_numpy(od.rope_table(int(max(pos, default=0)) + 1, max(rot, 2), 1e4).astype(np.float32)).cuda()
    tn = table.cpu().numpy()
    qo = torch.full((T, H * D + 16), 7.0, dtype=dtype, device="cuda")
    abi.kv_cache_append(pg.cache, k, v, i32(start), i32(past), pg.dev_table, i32(pos),
                        table if rot else None, max_new=max(new) + 1, Q=q, Q_out=qo[:, : H * D], interleaved=inter)
    abi.check_status()
    f = np.float32
    turn = (lambda r: od.rope(r.astype(f), pos, tn, inter, dtype=f)) if rot else (lambda r: r.astype(f))
    kn = turn(xn[:, H * D: H * D + w].reshape(T, pg.Hkv, D))
    vn = xn[:, H * D + w: H * D + 2 * w].reshape(T, pg.Hkv, D).astype(f)
    for b in range(len(past)):
        r = slice(start[b], start[b + 1])
        od.append(pg.k, pg.ks, pg.table[b], past[b], kn[r], pg.page)
        od.append(pg.v, pg.vs, pg.table[b], past[b], vn[r], pg.page)
    ref = torch.from_numpy(turn(xn[:, : H * D].reshape(T, H, D)).reshape(T, H * D)).to(dtype)
    assert torch.equal(qo[:, : H * D].cpu(), ref)                 # one rounding of exact float32 steps
    assert torch.all(qo[:, H * D:] == 7.0)
    return xn


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("page,D,H,Hkv,rot,inter", [
    (16, 64, 4, 2, 64, False), (32, 128, 7, 1, 128, False), (64, 128, 3, 3, 64, True), (128, 128, 5, 5, 128, True),
    (128, 64, 2, 1, 32, False), (64, 64, 1, 1, 0, False), (16, 128, 6, 2, 16, True)])
def test_append(abi, dtype, page, D, H, Hkv, rot, inter):
    """Ragged appends behind each other: prompts (a sequence without rows,
    one row, page boundaries), then tokens one by one, then a longer run
    whose larger values make the scales grow."""
    rng = np.random.default_rng(page + D + H)
    new = [0, 1, page, page + 1, 2 * page - 1, 5]
    past = [0, 3, 0, page - 1, 1, page]
    pg = Paged(abi, rng, len(new), 8 * page, Hkv, page, D)
    # something to keep: fill the pasts first
    append_both(abi, rng, pg, [0] * 6, past, H, dtype, rot, inter)
    pg.check([0] * 6, past)
    append_both(abi, rng, pg, past, new, H, dtype, rot, inter)
    pg.check(past, new)
    past = [p + n for p, n in zip(past, new)]
    for step in range(3):
        append_both(abi, rng, pg, past, [1] * 6, H, dtype, rot, inter, loud=1.0 + step)
        past = [p + 1 for p in past]
    pg.check(past, [0] * 6)
    append_both(abi, rng, pg, past, [3, page, 0, 2, 1, 7], H, dtype, rot, inter, loud=8.0)
    pg.check(past, [3, page, 0, 2, 1, 7])


def test_append_again_and_read(abi):
    """A block under denoising: the same slots written again and again behind
    a kept prefix; the same rows twice give the same cache; reading gives
    scale times code."""
    rng = np.random.default_rng(5)
    pg = Paged(abi, rng, 2, 200, 2, 32, 64)
    append_both(abi, rng, pg, [0, 0], [45, 7], 2, torch.bfloat16, 64, False)
    for _ in range(3):
        append_both(abi, rng, pg, [45, 7], [32, 9], 2, torch.bfloat16, 64, False)
        pg.check([45, 7], [32, 9])
    before = [t.clone() for t in (pg.cache.K, pg.cache.V, pg.cache.k_scale, pg.cache.v_scale)]
    append_both(abi, np.random.default_rng(9), pg, [45, 7], [32, 9], 2, torch.bfloat16, 64, False)
    mid = [t.clone() for t in (pg.cache.K, pg.cache.V, pg.cache.k_scale, pg.cache.v_scale)]
    append_both(abi, np.random.default_rng(9), pg, [45, 7], [32, 9], 2, torch.bfloat16, 64, False)
    after = [pg.cache.K, pg.cache.V, pg.cache.k_scale, pg.cache.v_scale]
    assert not torch.equal(before[0], mid[0])
    for x, y in zip(mid, after):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    first, n = [3, 0], [70, 16]
    start = [0, 70, 86]
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        K = torch.full((90, 130), 7.0, dtype=dtype, device="cuda")[:, :128] if dtype != torch.float32 else \
            torch.empty(90, 128, device="cuda")
        K = torch.full((90, 128), 7.0, dtype=dtype, device="cuda")
        V = torch.full((90, 128), 7.0, dtype=dtype, device="cuda")
        abi.kv_cache_read(pg.cache, pg.dev_table, i32(first), i32(start), K, V, max_rows=70)
        abi.check_status()
        for got, codes, scales in ((K, pg.k, pg.ks), (V, pg.v, pg.vs)):
            ref = np.concatenate([od.read(codes, scales, pg.table[b], first[b], n[b], 32) for b in range(2)])
            ref = torch.from_numpy(ref.reshape(86, 128).astype(np.float32)).to(dtype)
            assert torch.equal(got[:86].cpu(), ref)
            assert torch.all(got[86:] == 7.0)
    only = torch.empty(86, 128, device="cuda")
    abi.kv_cache_read(pg.cache, pg.dev_table, i32(first), i32(start), None, only, max_rows=70)
    assert np.array_equal(num(only), np.concatenate(
        [od.read(pg.v, pg.vs, pg.table[b], first[b], n[b], 32) for b in range(2)]).reshape(86, 128).astype(np.float32))


def test_append_extremes(abi):
    """All-zero rows, the smallest and largest numbers of bf16, and rows that
    are not finite (the block reads as NaN until it is begun anew)."""
    page, D = 16, 64
    for rows, keep in (([0.0] * 4, True), ([1e-38] * 4, True), ([3.3e38, -3.3e38, 1.0, 0.0], True),
                       ([float("inf"), 1.0, 1.0, 1.0], False), ([1.0, float("nan"), 1.0, 1.0], False)):
        pg = Paged(abi, np.random.default_rng(1), 1, 3 * page, 1, page, D)
        x = torch.zeros(4, D, dtype=torch.bfloat16, device="cuda")
        x[:, 5] = torch.tensor(rows).to(torch.bfloat16)
        w = torch.ones(4, D, dtype=torch.bfloat16, device="cuda")
        go = lambda k, past, n: abi.kv_cache_append(pg.cache, k[:n], w[:n], i32([0, n]), i32([past]), pg.dev_table,
                                                    None, None, max_new=n)
        xn = num(x).reshape(4, 1, D).astype(np.float32)
        one = np.ones((4, 1, D), np.float32)
        go(x, 0, 4)
        go(w, 4, 3)                                     # behind them, in the same block
        for codes, scales, a in ((pg.k, pg.ks, xn), (pg.v, pg.vs, one)):
            od.append(codes, scales, pg.table[0], 0, a, page)
            od.append(codes, scales, pg.table[0], 4, one[:3], page)
        abi.check_status()
        pg.check([7], [0])
        p = pg.table[0, 0]
        assert np.isfinite(pg.ks[p, 0]) == keep and pg.vs[p, 0] == np.float32(1) / np.float32(127)
        go(w, 0, 4)                                     # begun anew
        assert pg.cache.k_scale[p, 0].item() == pg.cache.v_scale[p, 0].item()


def test_append_outside_its_bounds(abi):
    """Numbers that do not fit are reported and write nothing."""
    pg = Paged(abi, np.random.default_rng(1), 1, 64, 1, 16, 64, stale=False)
    x = torch.ones(8, 64, dtype=torch.float16, device="cuda")
    far = torch.tensor([[pg.pages, -1]], dtype=torch.int32, device="cuda")
    for start, past, table in (([0, 9], 0, pg.dev_table), ([0, 8], -1, pg.dev_table), ([0, 8], 60, pg.dev_table),
                               ([0, 8], 0, far), ([0, 8], 16, far), ([8, 0], 0, pg.dev_table),
                               ([0, 7], 2 ** 31 - 1, pg.dev_table)):
        if past == 60:
            table = table[:, :1].contiguous()
        abi.kv_cache_append(pg.cache, x, x, i32(start), i32([past]), table, None, None, max_new=8)
        with pytest.raises(abi.StarqError) as e:
            abi.check_status()
        assert e.value.code == abi.ERR_RANGE
    assert torch.all(pg.cache.K == 128) and torch.all(pg.cache.k_scale == 0)
    out = torch.full((8, 64), 7.0, dtype=torch.float16, device="cuda")
    abi.kv_cache_read(pg.cache, far, i32([0]), i32([0, 8]), out, None, max_rows=8)
    with pytest.raises(abi.StarqError):
        abi.check_status()
    assert torch.all(out == 7.0)


# --------------------------------------------------------------------------
# Attention
# --------------------------------------------------------------------------
def fill(pg, rng, lens, spread=0.3):
    """Codes and scales straight into the pages of the sequences' lengths;
    other blocks keep what an earlier user left (scales NaN and infinite)."""
    for codes, scales, name in ((pg.k, pg.ks, "K"), (pg.v, pg.vs, "V")):
        for b, L in enumerate(lens):
            for blk in range((L + pg.page - 1) // pg.page):
                p = pg.table[b, blk]
                codes[p] = np.clip(np.rint(rng.standard_normal(codes[p].shape) * 40), -127, 127)
                scales[p] = (np.exp(rng.standard_normal(pg.Hkv) * spread) / 40).astype(np.float32)
        getattr(pg.cache, name).copy_(torch.from_numpy((codes + 128).astype(np.uint8)))
    pg.cache.k_scale.copy_(torch.from_numpy(pg.ks))
    pg.cache.v_scale.copy_(torch.from_numpy(pg.vs))


def check_attention(pg, q, out, lse, new, lens, H, dtype, scale, causal, mask, apart=False):
    start = np.concatenate([[0], np.cumsum(new)])
    D = pg.D
    q, out, lse = num(q).reshape(-1, H, D), num(out).reshape(-1, H, D), num(lse)
    for b, L in enumerate(lens):
        r = slice(start[b], start[b + 1])
        k, v = (od.read(c, s, pg.table[b], 0, L, pg.page) for c, s in ((pg.k, pg.ks), (pg.v, pg.vs)))
        ref, rl, mag, size = od.attention(q[r], k, v, scale, causal, None if mask is None else mask[b])
        d = ((D + 4) * 2.0 ** -24 * size)[..., None]
        rel = 2 * (2 * d + 2.0 ** -20) + 2.0 ** -11 + L * 2.0 ** -24 + 2.0 ** -20
        err = np.abs(out[r] - ref)
        if apart:
            mag = mag + 2.0 ** -32 * L * 127 * largest_weight(pg, q[r], b, L, scale, rl) / rel
        assert np.all(err <= mag * rel + U[dtype] * np.abs(ref) * (1 + rel) + TINY[dtype]), (b, L, err.max())
        empty = np.isneginf(rl)
        assert np.array_equal(empty, np.isneginf(lse[r])) and np.all(out[r][empty] == 0)
        tol = 2 * d[..., 0] + L * 2.0 ** -24 + 2.0 ** -19 * (1 + np.abs(np.where(empty, 0, rl)))
        assert np.all(np.abs(np.where(empty, 0, lse[r]) - np.where(empty, 0, rl)) <= tol), (b, L)


def largest_weight(pg, q, b, L, scale, lse):
    """max_j p_j s_v(j) of every row and head, p normalised: [n][H][1]."""
    k = od.read(pg.k, pg.ks, pg.table[b], 0, L, pg.page)
    sv = np.repeat(pg.vs[pg.table[b]], pg.page, axis=0)[:L].astype(np.float64)
    G = q.shape[1] // pg.Hkv
    s = np.einsum("nhd,lhd->nhl", q, np.repeat(k, G, axis=1)) * scale
    return (np.exp(s - lse[..., None]) * np.repeat(sv, G, axis=1).T[None]).max(-1, keepdims=True)


def attend(abi, rng, pg, new, lens, H, dtype, causal=False, mask=None, scale=None, q=None, pad=0,
           apart=False):
    T, D = sum(new), pg.D
    if q is None:
        q, _ = randn(rng, (T, H * D + pad), dtype)
        q = q[:, : H * D]
    out = torch.full((T, H * D + pad), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda")
    start = np.concatenate([[0], np.cumsum(new)])
    dm = None if mask is None else torch.from_numpy(mask).cuda()
    abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32(lens), i32(start), out[:, : H * D], max_new=max(new),
                           max_len=max(lens), causal=causal, key_mask=dm, scale=scale, lse=lse)
    abi.check_status()
    assert torch.all(out[:, H * D:] == 7.0)
    check_attention(pg, q, out[:, : H * D], lse, new, lens, H, dtype, D ** -0.5 if scale is None else scale, causal,
                    mask, apart)
    return out[:, : H * D], lse


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("page,D,H,Hkv", [(16, 64, 2, 1), (32, 128, 7, 1), (64, 128, 4, 4), (128, 64, 6, 2),
                                          (16, 128, 3, 1), (64, 64, 5, 5), (128, 128, 16, 2)])
@pytest.mark.parametrize("causal,masked", [(False, False), (True, False), (False, True), (True, True)])
def test_attention(abi, dtype, page, D, H, Hkv, causal, masked):
    """Lengths from none to several tiles, new tokens from none to more than
    the sequence holds, masks that leave rows empty."""
    rng = np.random.default_rng(page * 7 + D + H)
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 129, 300]
    new = [2, 1, 3, 16, 0, 5, 1, 33, 9, 4]
    pg = Paged(abi, rng, len(lens), max(lens), Hkv, page, D)
    fill(pg, rng, lens)
    mask = None
    if masked:
        mask = (rng.random((len(lens), max(lens) + 5)) < 0.6).astype(np.uint8) * 3
        mask[6] = 0
        mask[8, :128] = 0
        mask[9, 64:192] = 0
    attend(abi, rng, pg, new, lens, H, dtype, causal, mask, pad=8)


@pytest.mark.parametrize("new,H,Hkv,D", [(1, 28, 4, 128), (32, 4, 4, 128), (32, 7, 1, 128), (61, 3, 1, 64),
                                         (128, 2, 1, 128), (1, 2, 1, 64)])
def test_attention_long(abi, new, H, Hkv, D):
    """Many tiles a unit (runs joined over CTAs), a short sequence beside a
    long one."""
    rng = np.random.default_rng(new + H)
    lens = [5000, 130, 2049]
    pg = Paged(abi, rng, 3, 5000, Hkv, 64, D)
    fill(pg, rng, lens)
    a, la = attend(abi, rng, pg, [new, 1, new], lens, H, torch.bfloat16)
    b, lb = attend(abi, np.random.default_rng(new + H), pg, [new, 1, new], lens, H, torch.bfloat16, causal=True)
    q, _ = randn(rng, (2 * new + 1, H * D), torch.bfloat16)
    first = attend(abi, rng, pg, [new, 1, new], lens, H, torch.bfloat16, q=q)
    again = attend(abi, rng, pg, [new, 1, new], lens, H, torch.bfloat16, q=q)
    for x, y in zip(first, again):                     # the same bits whatever the timing
        assert torch.equal(x, y)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,H,Hkv", [(7, 7, 1), (19, 2, 2), (3, 14, 2), (61, 1, 1), (37, 7, 1)])
def test_attention_odd_rows(abi, new, H, Hkv, D):
    """An odd number of rows of a key/value head: partial runs of theirs lie
    side by side in the workspace."""
    rng = np.random.default_rng(new + D)
    pg = Paged(abi, rng, 3, 2300, Hkv, 32, D)
    lens = [2300, 700, 1999]
    fill(pg, rng, lens)
    attend(abi, rng, pg, [new, new - 1, new], lens, H, torch.bfloat16, causal=new == 61)


@pytest.mark.parametrize("bound", [0, 1 << 19])
@pytest.mark.parametrize("dtype,page,D,H,Hkv,new", [
    (torch.float16, 16, 64, 16, 2, 5), (torch.bfloat16, 64, 128, 7, 1, 3), (torch.bfloat16, 32, 128, 14, 2, 9),
    (torch.float16, 128, 64, 3, 1, 17), (torch.bfloat16, 16, 128, 4, 4, 64), (torch.float16, 64, 64, 8, 1, 8)])
@pytest.mark.parametrize("causal,masked", [(False, False), (True, False), (True, True)])
def test_attention_bound(abi, bound, dtype, page, D, H, Hkv, new, causal, masked):
    """17 to 64 rows of a key/value head under a tight and a generous bound
    of the lengths (they lead to different kernels)."""
    rng = np.random.default_rng(new + page)
    lens = [new, 333, 1201, 64]
    count = [new, new - 1, new, 0]
    pg = Paged(abi, rng, 4, 1201, Hkv, page, D)
    fill(pg, rng, lens)
    most = max(lens) + bound
    mask = None
    if masked:
        mask = (rng.random((4, most)) < 0.6).astype(np.uint8)
        mask[1, 64:] = 0                              # most of a sequence is not seen
        mask[2, :130] = 0
    q, _ = randn(rng, (sum(count), H * D), dtype)
    out, lse = torch.empty_like(q), torch.empty(sum(count), H, device="cuda")
    abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32(lens), i32(np.concatenate([[0], np.cumsum(count)])), out,
                           max_new=new, max_len=most, causal=causal, lse=lse,
                           key_mask=None if mask is None else torch.from_numpy(mask).cuda())
    abi.check_status()
    check_attention(pg, q, out, lse, count, lens, H, dtype, D ** -0.5, causal, mask)


@pytest.mark.parametrize("new", [1, 20])
def test_attention_many_sequences(abi, new):
    """More sequences than threads of a CTA."""
    rng = np.random.default_rng(new)
    lens = [int(x) for x in rng.integers(0, 70, 300)]
    pg = Paged(abi, rng, 300, 70, 1, 16, 64)
    fill(pg, rng, lens)
    attend(abi, rng, pg, [new if b % 7 else 0 for b in range(300)], lens, 2, torch.float16)


@pytest.mark.parametrize("new", [1, 40])
def test_attention_extremes(abi, new):
    """Scores in the hundreds and far apart, block scales eight orders of
    magnitude apart, values all zero, large and tiny queries."""
    rng = np.random.default_rng(2)
    lens = [200]
    pg = Paged(abi, rng, 1, 200, 1, 16, 128)
    fill(pg, rng, lens, spread=1.5)
    for blk, f in ((0, 1e-6), (3, 1e3), (7, 3e-4)):
        pg.vs[pg.table[0, blk]] *= np.float32(f)
    p = pg.table[0, 5]
    pg.v[p], pg.vs[p] = 0, od.SCALE_FLOOR
    p = pg.table[0, 6]
    pg.v[p], pg.vs[p] = 0, 0.0                          # a block that was never written
    pg.cache.V.copy_(torch.from_numpy((pg.v + 128).astype(np.uint8)))
    pg.cache.v_scale.copy_(torch.from_numpy(pg.vs))
    for size in (1.0, 30.0, 1e-3, 1e-30):
        for dtype in (torch.float16, torch.bfloat16):
            x, _ = randn(rng, (new, 3 * 128), dtype)
            attend(abi, rng, pg, [new], lens, 3, dtype, q=x * size, apart=True)
    x, _ = randn(rng, (new, 3 * 128), torch.bfloat16)
    attend(abi, rng, pg, [new], lens, 3, torch.bfloat16, q=x * 1e20, scale=1e-20, apart=True)


def test_attention_not_finite(abi):
    """A poisoned block that a row sees makes the row NaN; one that only
    masked slots touch does not; a NaN query makes its own row NaN."""
    for new in (2, 24):
        rng = np.random.default_rng(4)
        pg = Paged(abi, rng, 1, 96, 1, 32, 64)
        fill(pg, rng, [96])
        for which in ("k_scale", "v_scale"):
            keep = getattr(pg.cache, which).clone()
            getattr(pg.cache, which)[pg.table[0, 1]] = float("nan")
            q, _ = randn(rng, (new, 2 * 64), torch.float16)
            out = torch.empty_like(q)
            lse = torch.empty(new, 2, device="cuda")
            go = lambda mask: abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32([96]), i32([0, new]), out,
                                                     max_new=new, max_len=96, key_mask=mask, lse=lse)
            go(None)
            assert torch.isnan(out).all()
            mask = np.ones((1, 96), np.uint8)
            mask[0, 32:64] = 0
            go(torch.from_numpy(mask).cuda())
            check_attention(pg, q, out, lse, [new], [96], 2, torch.float16, 0.125, False, mask)
            getattr(pg.cache, which).copy_(keep)
        q[0, 3] = float("nan")
        go(None)
        assert torch.isnan(out[0, :64]).all() and torch.isfinite(out[0, 64:]).all() and torch.isfinite(out[1:]).all()
        abi.check_status()


def test_attention_outside_its_bounds(abi):
    for new in (1, 30):
        rng = np.random.default_rng(4)
        pg = Paged(abi, rng, 2, 64, 1, 16, 64)
        fill(pg, rng, [64, 64])
        q, _ = randn(rng, (2 * new, 64), torch.float16)
        out = torch.empty_like(q)
        wrong = pg.dev_table.clone()
        wrong[0, 2] = pg.pages
        for table, lens, start, most in ((wrong, [64, 64], [0, new, 2 * new], 64), (pg.dev_table, [65, 64], [0, new, 2 * new], 64),
                                         (pg.dev_table, [64, 64], [0, new, 2 * new + 1], 64),
                                         (pg.dev_table, [80, 64], [0, new, 2 * new], 80)):
            abi.kv_cache_attention(q, pg.cache, table, i32(lens), i32(start), out, max_new=new, max_len=most)
            with pytest.raises(abi.StarqError) as e:
                abi.check_status()
            assert e.value.code == abi.ERR_RANGE
        abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32([64, 64]), i32([0, new, 2 * new]), out, max_new=new,
                               max_len=64)
        abi.check_status()


@pytest.mark.parametrize("new", [1, 40])
def test_attention_far_pages(abi, new):
    """Pages whose byte offsets pass 32 bits."""
    page, D, Hkv = 128, 128, 2
    pages = (1 << 32) // (page * D * Hkv) + 9
    K, V = (torch.empty(pages, Hkv, page, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((pages, Hkv), float("nan"), device="cuda") for _ in range(2))
    cache = abi.KVCache(K, V, ks, vs)
    rng = np.random.default_rng(8)
    L = 300
    table = torch.tensor([[pages - 1, 3, pages - 5]], dtype=torch.int32, device="cuda")
    x, xn = randn(rng, (L, 2 * Hkv * D), torch.float16)
    w = Hkv * D
    abi.kv_cache_append(cache, x[:, :w], x[:, w:], i32([0, L]), i32([0]), table, None, None, max_new=L)
    back = torch.empty(L, w, device="cuda")
    vback = torch.empty(L, w, device="cuda")
    abi.kv_cache_read(cache, table, i32([0]), i32([0, L]), back, vback, max_rows=L)
    k, v = num(back).reshape(L, Hkv, D), num(vback).reshape(L, Hkv, D)
    # a code is off by at most half a step, a step at most max / 127
    assert np.all(np.abs(k - xn[:, :w].reshape(k.shape)) <= np.abs(xn).max() / 127 * 0.501)
    q, qn = randn(rng, (new, w), torch.float16)
    out, lse = torch.empty_like(q), torch.empty(new, Hkv, device="cuda")
    abi.kv_cache_attention(q, cache, table, i32([L]), i32([0, new]), out, max_new=new, max_len=L, lse=lse)
    abi.check_status()
    ref, rl, mag, _ = od.attention(qn.reshape(new, Hkv, D), k, v, D ** -0.5)
    assert np.all(np.abs(num(out).reshape(ref.shape) - ref) <= mag * 2.0 ** -10 + 2.0 ** -11 * np.abs(ref))
    assert np.all(np.abs(num(lse) - rl) <= 1e-4)


def test_cache_on_another_stream(abi):
    """Append, read and attention enqueued on a side stream."""
    rng = np.random.default_rng(6)
    pg = Paged(abi, rng, 1, 100, 1, 32, 64)
    x, _ = randn(rng, (70, 3 * 64), torch.float16)
    q, k, v = x[:, :64], x[:, 64:128], x[:, 128:]
    side = torch.cuda.Stream()
    outs = []
    for s in (torch.cuda.current_stream(), side):
        s.wait_stream(torch.cuda.current_stream())
        out = torch.empty(70, 64, dtype=torch.float16, device="cuda")
        ws = torch.empty(abi.kv_cache_attention_workspace_size(1, 70, 1, 1, 64), dtype=torch.uint8, device="cuda")
        args = (i32([0, 70]), i32([0]), i32([70]))
        torch.cuda.synchronize()
        abi.kv_cache_append(pg.cache, k, v, args[0], args[1], pg.dev_table, None, None, max_new=70, stream=s)
        abi.kv_cache_attention(q, pg.cache, pg.dev_table, args[2], args[0], out, max_new=70, max_len=70, causal=True,
                               workspace=ws, stream=s)
        s.synchronize()
        outs.append(out)
    assert torch.equal(outs[0], outs[1])


# --------------------------------------------------------------------------
# Linears with group-scaled 4-bit weights
# --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("L,N,K,group,bias", [
    (1, 64, 128, 128, False), (1, 33, 32, 32, True), (2, 100, 64, 64, False), (8, 16, 4096, 128, True),
    (9, 257, 1056, 32, False), (17, 48, 960, 64, True), (25, 31, 1408, 128, False), (32, 15, 2080, 32, True),
    (5, 1, 3584, 64, False), (1, 5000, 192, 64, True), (16, 40, 9728, 128, False)])
def test_w4g_linear(abi, dtype, L, N, K, group, bias):
    rng = np.random.default_rng(L + N + K)
    x, xn = randn(rng, (L, K + 8), dtype)
    x, xn = x[:, :K], xn[:, :K]
    codes = rng.integers(-8, 8, (N, K))
    packed = torch.from_numpy(((codes[:, 0::2] & 15) | ((codes[:, 1::2] & 15) << 4)).astype(np.uint8)).cuda()
    scales = (np.exp(rng.standard_normal((N, K // group))) / 50).astype(np.float32)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    ref, size = od.w4g_linear(xn, codes, scales, b)
    for ydt in (dtype, torch.float32):
        Y = torch.full((L, N + 3), 7.0, dtype=ydt, device="cuda")
        abi.w4g_linear(x, packed, torch.from_numpy(scales).cuda(), Y[:, :N],
                       bias=None if b is None else torch.from_numpy(b).cuda())
        abi.check_status()
        tol = (K / 8 + 16) * 2.0 ** -24 * size + U[ydt] * np.abs(ref) * 1.01 + TINY[ydt]
        assert np.all(np.abs(num(Y)[:, :N] - ref) <= tol)
        assert torch.all(Y[:, N:] == 7.0)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4g_weights_from_prepare(abi, group):
    """The library's own weight quantiser on rows of one group gives the
    codes and scales of this linear."""
    rng = np.random.default_rng(group)
    N, K = 48, 512
    W, Wn = randn(rng, (N, K), torch.float16)
    Wq = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(N, K // group, device="cuda")
    abi.sgat_prepare_weight(W.view(-1, group), None, 1, Wq.view(-1, group // 2), scales.view(-1))
    codes = osg.unpack_int4(Wq.cpu().numpy())
    x, xn = randn(rng, (3, K), torch.float16)
    Y = torch.empty(3, N, device="cuda")
    abi.w4g_linear(x, Wq, scales, Y)
    ref, size = od.w4g_linear(xn, codes, scales.cpu().numpy())
    assert np.all(np.abs(num(Y) - ref) <= (K / 8 + 16) * 2.0 ** -24 * size)
    back = codes * np.repeat(num(scales), group, axis=1)
    assert np.all(np.abs(back - Wn) <= np.repeat(num(scales), group, axis=1) * 0.5 * (1 + 1e-6))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("L,group", [(1, 32), (5, 64), (11, 128), (32, 64)])
def test_w4g_values(abi, dtype, L, group):
    """Codes of zero give exact zeros (and the bias); an infinite or NaN
    activation shows in its own row alone, as the formula has it; a block of
    tiny and one of huge activations keep their places."""
    rng = np.random.default_rng(group + L)
    N, K = 130, 512
    codes = rng.integers(1, 8, (N, K)) * rng.choice([-1, 1], (N, K))
    codes[:40] = 0
    x, _ = randn(rng, (L, K), dtype)
    small, large = (2.0 ** -14, 2.0 ** 10) if dtype is torch.float16 else (2.0 ** -100, 2.0 ** 100)
    x[:, :128] *= small
    x[:, 128:256] *= large
    xn = num(x)
    packed = torch.from_numpy(((codes[:, 0::2] & 15) | ((codes[:, 1::2] & 15) << 4)).astype(np.uint8)).cuda()
    scales = (np.exp(rng.standard_normal((N, K // group))) / 50).astype(np.float32)
    bias = rng.standard_normal(N).astype(np.float32)
    run = lambda t, w: abi.w4g_linear(t, w, torch.from_numpy(scales).cuda(), Y, bias=torch.from_numpy(bias).cuda())
    Y = torch.empty(L, N, device="cuda")
    run(x, packed)
    ref, size = od.w4g_linear(xn, codes, scales, bias)
    tol = (K / 8 + 16) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(ref) * 1.01
    assert np.all(np.abs(num(Y) - ref) <= tol)
    assert torch.equal(Y[:, :40], torch.from_numpy(bias[:40]).cuda().expand(L, 40))
    only = codes.copy()                               # each block on its own
    for blk in range(4):
        only[:] = 0
        only[:, blk * 128:(blk + 1) * 128] = codes[:, blk * 128:(blk + 1) * 128]
        run(x, torch.from_numpy(((only[:, 0::2] & 15) | ((only[:, 1::2] & 15) << 4)).astype(np.uint8)).cuda())
        ref, size = od.w4g_linear(xn, only, scales, bias)
        assert np.all(np.abs(num(Y) - ref) <= (K / 8 + 16) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(ref) * 1.01)
    run(x, packed)
    before = Y.clone()
    bad = L // 2
    y = x.clone()
    y[bad, 300] = float("inf")
    run(y, packed)
    assert torch.isnan(Y[bad, :40]).all()             # 0 times infinity
    assert torch.equal(Y[bad, 40:], torch.from_numpy(np.sign(codes[40:, 300]) * np.inf).float().cuda())
    rest = [i for i in range(L) if i != bad]
    assert torch.equal(Y[rest], before[rest])
    y[bad, 300] = float("nan")
    run(y, packed)
    assert torch.isnan(Y[bad]).all() and torch.equal(Y[rest], before[rest])


@pytest.mark.parametrize("dtype,page,D,H,Hkv,B,new", [
    (torch.bfloat16, 16, 128, 7, 1, 40, 1), (torch.float16, 64, 64, 8, 4, 200, 2), (torch.bfloat16, 32, 128, 28, 4, 9, 32),
    (torch.float16, 128, 64, 6, 2, 90, 100), (torch.bfloat16, 64, 64, 2, 2, 1, 300)])
@pytest.mark.parametrize("most", [1, 100, 256, 1000])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_short(abi, dtype, page, D, H, Hkv, B, new, most, causal):
    """Many short sequences, some without tokens in the cache, some without
    rows: units that are not cut have nothing to join, and rows without keys
    are written by their unit."""
    rng = np.random.default_rng(B + most)
    lens = [int(v) for v in rng.integers(0, most + 1, B)]
    lens[0] = most
    count = [int(v) for v in rng.integers(0, new + 1, B)]
    count[0] = new
    pg = Paged(abi, rng, B, most, Hkv, page, D)
    fill(pg, rng, lens)
    q, _ = randn(rng, (sum(count), H * D), dtype)
    out, lse = torch.full_like(q, 7.0), torch.full((sum(count), H), 7.0, device="cuda")
    start = np.concatenate([[0], np.cumsum(count)])
    abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32(lens), i32(start), out, max_new=new, max_len=most,
                           causal=causal, lse=lse)
    abi.check_status()
    for b in [0] + [int(v) for v in rng.choice(B, min(B, 12), replace=False)]:
        r = slice(start[b], start[b + 1])
        one = Paged.__new__(Paged)
        one.__dict__.update(pg.__dict__)
        one.table = pg.table[b:b + 1]
        check_attention(one, q[r], out[r], lse[r], [count[b]], [lens[b]], H, dtype, D ** -0.5, causal, None)
    empty = np.repeat(np.asarray(lens) == 0, count)
    assert torch.isfinite(out).all() and not (out == 7.0).all(dim=1).any()
    assert torch.isneginf(lse[torch.from_numpy(empty).cuda()]).all()
