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
