"""Cache attention and group-scaled linears where their kernels can go wrong
apart from ordinary inputs: numbers at the ends of their ranges, and the forms
that only some sizes reach. Tolerances are those derived in
test_gpu_decode.py.
"""

import numpy as np
import pytest
import torch

from oracle import decode as od
from tests.test_gpu_decode import TINY, U, Paged, attend, check_attention, fill, i32, num, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page,D,H,Hkv,new", [(16, 128, 2, 1, 40), (64, 64, 6, 2, 61), (32, 128, 7, 1, 64),
                                              (64, 128, 8, 2, 2), (16, 64, 6, 3, 7), (32, 128, 2, 1, 19)])
@pytest.mark.parametrize("scale", [None, 1e-20])
@pytest.mark.parametrize("masked", [False, True])
def test_causal_zero_rows(abi, dtype, page, D, H, Hkv, new, scale, masked):
    """Each kernel, causal: query rows that are zero or tiny, key blocks that
    are zero (at the smallest scale and at none), as padding leaves them. The
    factor of a score may then be too small for a float, and the scores of
    keys that a row does not see are -inf."""
    rng = np.random.default_rng(new + D)
    lens = [23, new, new + 13, 203, 1201]
    count = [new, new, new - 1, new, new]
    pg = Paged(abi, rng, len(lens), max(lens), Hkv, page, D)
    fill(pg, rng, lens)
    for b, L in enumerate(lens):
        for blk in range((L + page - 1) // page):
            if blk % 3 != 1:                          # the last blocks among them
                p = pg.table[b, blk]
                pg.k[p], pg.ks[p] = 0, od.SCALE_FLOOR if blk % 3 == 0 else 0.0
    pg.cache.K.copy_(torch.from_numpy((pg.k + 128).astype(np.uint8)))
    pg.cache.k_scale.copy_(torch.from_numpy(pg.ks))
    q, _ = randn(rng, (sum(count), H * D), dtype)
    q[0::5] = 0
    q[1::5] *= 1e-30 if dtype is torch.bfloat16 else 2.0 ** -22
    q[2::5, :D] = 0                                   # one head of a row
    mask = (rng.random((len(lens), max(lens))) < 0.6).astype(np.uint8) if masked else None
    attend(abi, rng, pg, count, lens, H, dtype, causal=True, mask=mask, scale=scale, q=q)


@pytest.mark.parametrize("new", [1, 70])
def test_attention_on_another_stream(abi, monkeypatch, new):
    """Without a workspace of the caller's: it comes from the pool of the
    call's stream, and tensors that the current stream makes and fills right
    behind the call do not touch it."""
    rng = np.random.default_rng(new)
    lens, H = [4000, 2001], 2
    pg = Paged(abi, rng, 2, 4000, 1, 32, 64)
    fill(pg, rng, lens)
    q, _ = randn(rng, (2 * new, H * 64), torch.float16)
    out, lse = torch.empty_like(q), torch.empty(2 * new, H, device="cuda")
    lens32, start = i32(lens), i32([0, new, 2 * new])
    where, real = [], abi.lib

    class Library:
        def __getattr__(self, name):
            if name == "kv_cache_attention":
                return lambda *args: where.append(args[-3]) or real.kv_cache_attention(*args)
            return getattr(real, name)

    monkeypatch.setattr(abi, "lib", Library())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    size = abi.kv_cache_attention_workspace_size(2, new, H, 1, 64)
    for _ in range(20):
        abi.kv_cache_attention(q, pg.cache, pg.dev_table, lens32, start, out, max_new=new, max_len=4000, lse=lse,
                               stream=side)
        torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)
    side.synchronize()
    abi.check_status()
    check_attention(pg, q, out, lse, [new, new], lens, H, torch.float16, 0.125, False, None)
    pools = [(s["address"], s["address"] + s["total_size"], s["stream"]) for s in torch.cuda.memory_snapshot()]
    assert len(where) == 20
    for p in where:
        assert [s for a, b, s in pools if a <= p < b] == [side.cuda_stream]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("L,N,K,group,bias", [
    (12, 29201, 256, 32, True),          # CTAs of 16 warps (more than 8 rows, channels that fill the SMs)
    (17, 29187, 1408, 128, False),
    (32, 29230, 2560, 64, True),         # and more blocks than their shared memory has room for
    (24, 37888, 3584, 64, False),
    (32, 48, 18944, 64, False),          # CTAs of 8 warps, a slice in several chunks
    (27, 130, 12288, 32, True)])
def test_w4g_wide_and_deep(abi, dtype, L, N, K, group, bias):
    """The forms of the linear that many channels or a long K lead to."""
    rng = np.random.default_rng(L + N + K)
    x, xn = randn(rng, (L, K + 8), dtype)
    x, xn = x[:, :K], xn[:, :K]
    codes = rng.integers(-8, 8, (N, K), dtype=np.int8)
    packed = torch.from_numpy(((codes[:, 0::2] & 15) | ((codes[:, 1::2] & 15) << 4)).astype(np.uint8)).cuda()
    scales = (np.exp(rng.standard_normal((N, K // group))) / 50).astype(np.float32)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    parts = [od.w4g_linear(xn, codes[n:n + 2048], scales[n:n + 2048], None if b is None else b[n:n + 2048])
             for n in range(0, N, 2048)]
    ref, size = (np.concatenate(p, axis=1) for p in zip(*parts))
    for ydt in (dtype, torch.float32):
        Y = torch.full((L, N + 3), 7.0, dtype=ydt, device="cuda")
        abi.w4g_linear(x, packed, torch.from_numpy(scales).cuda(), Y[:, :N],
                       bias=None if b is None else torch.from_numpy(b).cuda())
        abi.check_status()
        tol = (K / 8 + 16) * 2.0 ** -24 * size + U[ydt] * np.abs(ref) * 1.01 + TINY[ydt]
        assert np.all(np.abs(num(Y)[:, :N] - ref) <= tol)
        assert torch.all(Y[:, N:] == 7.0)


# --------------------------------------------------------------------------
# More than 64 rows of a key/value head: the tcgen05 kernel, whatever the
# lengths are
# --------------------------------------------------------------------------
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("new", [40, 70])
def test_tcgen05_not_finite(abi, which, new):
    """A poisoned block makes the rows that see it NaN, and no others; a NaN
    query its own row alone."""
    rng = np.random.default_rng(new)
    L, H = 96, 2
    pg = Paged(abi, rng, 1, L, 1, 32, 64)
    fill(pg, rng, [L])
    q, _ = randn(rng, (new, H * 64), torch.float16)
    out, lse = torch.empty_like(q), torch.empty(new, H, device="cuda")

    def go(causal=False, mask=None):
        abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32([L]), i32([0, new]), out, max_new=new, max_len=L,
                               causal=causal, key_mask=mask, lse=lse)
        abi.check_status()

    scale = getattr(pg.cache, which)
    keep = scale.clone()
    scale[pg.table[0, 1]] = float("nan")
    go()
    assert torch.isnan(out).all()
    mask = np.ones((1, L), np.uint8)
    mask[0, 32:64] = 0
    for causal in (False, True):
        go(causal, torch.from_numpy(mask).cuda())
        check_attention(pg, q, out, lse, [new], [L], H, torch.float16, 0.125, causal, mask)
    scale.copy_(keep)
    scale[pg.table[0, 2]] = float("nan")              # slots 64 .. 95, which row i sees from 64 <= L - new + i on
    go(True)
    few = 64 - (L - new)
    assert torch.isnan(out[few:]).all()
    check_attention(pg, q[:few], out[:few], lse[:few], [few], [64], H, torch.float16, 0.125, True, None)
    scale.copy_(keep)
    q[0, 3] = float("nan")
    go()
    assert torch.isnan(out[0, :64]).all() and torch.isfinite(out[0, 64:]).all() and torch.isfinite(out[1:]).all()


def test_tcgen05_outside_its_bounds(abi):
    rng = np.random.default_rng(4)
    new = 70
    pg = Paged(abi, rng, 2, 64, 1, 16, 64)
    fill(pg, rng, [64, 64])
    q, _ = randn(rng, (2 * new, 64), torch.float16)
    out, lse = torch.empty_like(q), torch.empty(2 * new, 1, device="cuda")
    wrong = pg.dev_table.clone()
    wrong[0, 2] = pg.pages
    none = pg.dev_table.clone()
    none[1, 0] = -1
    fits = [0, new, 2 * new]
    for table, lens, start, most in ((wrong, [64, 64], fits, 64), (none, [64, 64], fits, 64),
                                     (pg.dev_table, [65, 64], fits, 64), (pg.dev_table, [64, -1], fits, 64),
                                     (pg.dev_table, [64, 64], [0, new, 2 * new + 1], 64),
                                     (pg.dev_table, [64, 64], [0, new, new - 1], 64),
                                     (pg.dev_table, [80, 64], fits, 80), (pg.dev_table, [80, 64], fits, 1 << 19)):
        abi.kv_cache_attention(q, pg.cache, table, i32(lens), i32(start), out, max_new=new, max_len=most)
        with pytest.raises(abi.StarqError) as e:
            abi.check_status()
        assert e.value.code == abi.ERR_RANGE
    abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32([64, 64]), i32(fits), out, max_new=new, max_len=64, lse=lse)
    abi.check_status()
    check_attention(pg, q, out, lse, [new, new], [64, 64], 1, torch.float16, 0.125, False, None)


def test_tcgen05_far_pages(abi):
    """Pages whose byte offsets pass 32 bits."""
    page, D, Hkv, L, new = 128, 128, 2, 300, 80
    pages = (1 << 32) // (page * D * Hkv) + 9
    K, V = (torch.empty(pages, Hkv, page, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((pages, Hkv), float("nan"), device="cuda") for _ in range(2))
    cache = abi.KVCache(K, V, ks, vs)
    rng = np.random.default_rng(8)
    near = Paged(abi, rng, 1, L, Hkv, page, D)        # the same rows in a small cache, for the oracle
    fill(near, rng, [L])
    far = [pages - 1, 3, pages - 5]
    for big, small in ((K, near.cache.K), (V, near.cache.V), (ks, near.cache.k_scale), (vs, near.cache.v_scale)):
        big[far] = small[near.table[0].tolist()]
    q, _ = randn(rng, (new, Hkv * D), torch.float16)
    out, lse = torch.empty_like(q), torch.empty(new, Hkv, device="cuda")
    for causal in (False, True):
        abi.kv_cache_attention(q, cache, i32(far)[None], i32([L]), i32([0, new]), out, max_new=new, max_len=L,
                               causal=causal, lse=lse)
        abi.check_status()
        check_attention(near, q, out, lse, [new], [L], Hkv, torch.float16, D ** -0.5, causal, None)


@pytest.mark.parametrize("bound", [0, 1 << 19])
@pytest.mark.parametrize("causal", [False, True])
def test_tcgen05_many_sequences(abi, bound, causal):
    """More sequences than threads of a CTA, dealt out whole and cut."""
    B, new = 1100, 70
    rng = np.random.default_rng(B)
    lens = [int(v) for v in rng.integers(0, 70, B)]
    count = [0 if b % 7 == 3 else new if b % 5 == 0 else int(rng.integers(0, 9)) for b in range(B)]
    count[-1] = new
    pg = Paged(abi, rng, B, 70, 1, 16, 64)
    fill(pg, rng, lens)
    q, _ = randn(rng, (sum(count), 64), torch.float16)
    out, lse = torch.full_like(q, 7.0), torch.full((sum(count), 1), 7.0, device="cuda")
    abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32(lens), i32(np.concatenate([[0], np.cumsum(count)])), out,
                           max_new=new, max_len=70 + bound, causal=causal, lse=lse)
    abi.check_status()
    check_attention(pg, q, out, lse, count, lens, 1, torch.float16, 0.125, causal, None)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("new", [2, 70])
def test_infinite_value_scale(abi, causal, new):
    """A block whose value scale is infinite shows in every row that sees it,
    and in no other."""
    rng = np.random.default_rng(new)
    L = 96
    pg = Paged(abi, rng, 1, L, 1, 32, 64)
    fill(pg, rng, [L])
    pg.cache.v_scale[pg.table[0, 2]] = float("inf")   # slots 64 .. 95
    q, _ = randn(rng, (new, 64), torch.float16)
    out, lse = torch.empty_like(q), torch.empty(new, 1, device="cuda")
    abi.kv_cache_attention(q, pg.cache, pg.dev_table, i32([L]), i32([0, new]), out, max_new=new, max_len=L,
                           causal=causal, lse=lse)
    abi.check_status()
    few = max(0, 64 - (L - new)) if causal else 0     # rows before slot 64
    assert not torch.isfinite(out[few:]).any()
    if few:
        check_attention(pg, q[:few], out[:few], lse[:few], [few], [64], 1, torch.float16, 0.125, True, None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,H,Hkv,new", [(128, 7, 1, 1), (64, 8, 4, 2), (128, 4, 2, 7), (64, 6, 2, 5), (128, 2, 1, 19),
                                         (64, 8, 1, 9)])
@pytest.mark.parametrize("loud", [1, 4])
def test_attention_loud_channels(abi, dtype, D, H, Hkv, new, loud):
    """A few channels set the scale of a block of keys and the others have
    codes of a few units, and the queries have a mean: the bits of a score are
    those of sum q c, not of the largest codes."""
    rng = np.random.default_rng(new + D + loud)
    lens = [300, 77]
    pg = Paged(abi, rng, 2, 300, Hkv, 32, D)
    fill(pg, rng, lens)
    pg.k[:] = np.clip(np.rint(rng.standard_normal(pg.k.shape) * 2), -127, 127)
    at = rng.permutation(D)[:loud]
    pg.k[..., at] = rng.choice([-127, 127], pg.k[..., at].shape)
    pg.ks[:] = 0.5
    pg.cache.K.copy_(torch.from_numpy((pg.k + 128).astype(np.uint8)))
    pg.cache.k_scale.copy_(torch.from_numpy(pg.ks))
    x = rng.standard_normal((2 * new, H, D)) + 2
    x[..., at] = rng.standard_normal(x[..., at].shape) / 32
    q = torch.from_numpy(x.reshape(2 * new, H * D)).to(dtype).cuda()
    attend(abi, rng, pg, [new, new], lens, H, dtype, q=q, causal=new > 5)
