"""Cached decoding without a GPU: the oracle against closed forms, and the
argument checks of the C ABI (nothing is launched by a refused call)."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import decode as od


@pytest.fixture(scope="module")
def lib():
    from paper_2606_04945_gb300 import build
    build.build()
    from paper_2606_04945_gb300 import abi
    return abi


# ---- the oracle ------------------------------------------------------------
def test_rope_is_a_rotation():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((6, 3, 16))
    pos = np.array([0, 1, 5, 9, 9, 2])
    t = od.rope_table(10, 8, 100.0)
    for inter in (False, True):
        y = od.rope(x, pos, t, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.allclose(y[0], x[0])
        assert np.allclose(od.rope(y, pos, t, inter, inverse=True), x)
        # scores depend on the distance alone
        z = np.broadcast_to(x[:1], x.shape)
        a, b = od.rope(z, pos, t, inter), od.rope(z, pos + 0, t, inter)
        assert np.isclose(a[1, 0] @ b[2, 0], od.rope(z, pos * 0 + 4, t, inter)[0, 0] @ od.rope(z, pos * 0, t, inter)[0, 0])


def test_rope_scalings():
    f = od.rope_frequencies(64, 1e4)
    assert np.allclose(od.rope_frequencies(64, 1e4, "linear", 4.0), f / 4)
    n = od.rope_frequencies(64, 1e4, "ntk", 4.0)
    assert np.isclose(n[0], f[0]) and np.isclose(n[-1], f[-1] / 4)
    p = od.rope_frequencies(64, 1e4, "parts", 4.0, original=2048.0)
    assert np.isclose(p[0], f[0]) and np.isclose(p[-1], f[-1] / 4) and np.all(p <= f + 1e-15) and np.all(p >= f / 4 - 1e-15)


def test_append_error_bound():
    """A stored value is off by half a step of its block's scale for every
    time that the scale grew, and by half a step when it was stored."""
    rng = np.random.default_rng(1)
    page, D = 16, 8
    codes, scales = np.zeros((3, 1, page, D), np.int64), np.zeros((3, 1), np.float32)
    rows = rng.standard_normal((40, 1, D)).astype(np.float32) * np.linspace(1, 3, 40, dtype=np.float32)[:, None, None]
    table = np.array([2, 0, 1])
    for i in range(40):
        od.append(codes, scales, table, i, rows[i:i + 1], page)
    back = od.read(codes, scales, table, 0, 40, page)
    for blk in range(3):
        part = slice(blk * page, min(40, (blk + 1) * page))
        top = np.abs(rows[part]).max()
        assert np.isclose(scales[table[blk], 0], top / 127, rtol=1e-6)
        growths = sum(np.abs(rows[j]).max() > np.abs(rows[part][:j - blk * page]).max(initial=0)
                      for j in range(part.start, part.stop))
        assert np.abs(back[part] - rows[part]).max() <= (growths + 1) * 0.5 * top / 127 * 1.001


def test_attention_against_softmax():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    out, lse, mag, _ = od.attention(q, k, v, 0.3, causal=True)
    kk, vv = np.repeat(k, 2, axis=1), np.repeat(v, 2, axis=1)
    s = torch.from_numpy(np.einsum("nhd,lhd->nhl", q, kk) * 0.3)
    s[0, :, 5:] = -np.inf
    s[1, :, 6:] = -np.inf
    assert np.allclose(out, torch.einsum("nhl,lhd->nhd", s.softmax(-1), torch.from_numpy(vv)).numpy())
    assert np.allclose(lse, s.logsumexp(-1).numpy()) and np.all(mag >= np.abs(out))
    out, lse, _, _ = od.attention(q, k, v, 0.3, key_mask=np.zeros(7, np.uint8))
    assert np.all(out == 0) and np.all(np.isneginf(lse))


def test_w4g_against_dequantised():
    rng = np.random.default_rng(3)
    x, c, s = rng.standard_normal((2, 8)), rng.integers(-8, 8, (3, 8)), rng.random((3, 2)).astype(np.float32)
    y, _ = od.w4g_linear(x, c, s)
    for i in range(2):
        for n in range(3):
            assert np.isclose(y[i, n], sum(x[i, k] * c[n, k] * float(s[n, k // 4]) for k in range(8)))


# ---- refusals --------------------------------------------------------------
P = ctypes.c_void_p(4096)          # a non-null, aligned stand-in; never dereferenced
ODD = ctypes.c_void_p(4100)


def cache(lib, **kw):
    f = dict(K=4096, V=4096, k_scale=4096, v_scale=4096, pages=4, page=16, Hkv=2, D=64)
    f.update(kw)
    return ctypes.byref(lib.StarqKvCache(*[f[n] for n, _ in lib.StarqKvCache._fields_]))


BAD_CACHE = [(dict(D=96), -2), (dict(page=24), -2), (dict(page=256), -2), (dict(Hkv=0), -2), (dict(pages=-1), -2),
             (dict(K=0), -1), (dict(v_scale=0), -1), (dict(V=4104), -3)]


def refuse(lib, fn, names, base, changes, code):
    args = dict(base)
    args.update(changes)
    assert set(changes) <= set(names)
    assert getattr(lib.lib, fn)(*[args[n] for n in names]) == code, changes
    assert lib.lib.starq_last_error()


TABLE = "table positions rot theta scaling factor original beta_fast beta_slow mscale stream".split()


@pytest.mark.parametrize("changes,code", [
    (dict(rot=3), -2), (dict(rot=0), -2), (dict(positions=-1), -2), (dict(theta=1.0), -1), (dict(theta=float("nan")), -1),
    (dict(scaling=4), -1), (dict(scaling=1, factor=0.5), -1), (dict(scaling=3, original=0.0), -1),
    (dict(scaling=3, beta_fast=1.0), -1), (dict(mscale=-1.0), -1), (dict(table=None), -1), (dict(table=ODD), -3)])
def test_rope_table_refusals(lib, changes, code):
    base = dict(table=P, positions=4, rot=64, theta=1e4, scaling=0, factor=2.0, original=100.0, beta_fast=32.0,
                beta_slow=1.0, mscale=0.0, stream=None)
    refuse(lib, "glue_rope_table", TABLE, base, changes, code)


def test_nothing_to_do(lib):
    """Empty calls succeed without a launch."""
    assert lib.lib.glue_rope_table(None, 0, 64, 1e4, 0, 1.0, 0.0, 32.0, 1.0, 0.0, None) == 0
    assert lib.lib.glue_rope_apply(None, 128, 0, 0, 2, 64, 64, 0, 0, None, None, 0, None, 128, None) == 0
    c = cache(lib)
    assert lib.lib.kv_cache_append(c, None, 0, None, 0, None, 0, None, 0, 0, 0, 0, None, None, 0, 0, None, 0, None,
                                   None, 0, 0, 0, None) == 0
    assert lib.lib.kv_cache_read(c, None, 0, None, None, 0, 0, 0, None, None, 0, 0, None) == 0
    assert lib.lib.kv_cache_attention(None, 0, 0, 0, None, 0, 0, 2, c, None, 0, None, 0, 0, None, 0, 1.0, None, 0, None,
                                      None, 0, None) == 0
    assert lib.lib.w4g_linear(None, 64, 0, 0, 64, None, None, 64, 8, None, None, 8, 0, None) == 0


APPLY = "X ldx dtype L heads D rot interleaved inverse pos table positions Y ldy stream".split()


@pytest.mark.parametrize("changes,code", [
    (dict(dtype=3), -1), (dict(L=-1), -2), (dict(heads=0), -2), (dict(D=0), -2), (dict(rot=65), -2), (dict(rot=66), -2),
    (dict(ldx=100), -2), (dict(ldy=127), -2), (dict(positions=-1), -2), (dict(Y=P, ldy=256), -1), (dict(X=None), -1),
    (dict(pos=None), -1), (dict(table=None), -1), (dict(X=ctypes.c_void_p(4097)), -3)])
def test_rope_apply_refusals(lib, changes, code):
    base = dict(X=P, ldx=128, dtype=0, L=3, heads=2, D=64, rot=64, interleaved=0, inverse=0, pos=P, table=P,
                positions=10, Y=ctypes.c_void_p(1 << 20), ldy=128, stream=None)
    if "Y" in changes:
        changes["X"] = changes["Y"]
    refuse(lib, "glue_rope_apply", APPLY, base, changes, code)


APPEND = ("cache K ldk V ldv Q ldq Qo ldqo H dtype T seq_start past B max_new page_table table_ld pos table positions rot "
          "interleaved stream").split()


@pytest.mark.parametrize("changes,code", [(dict(cache=c), r) for c, r in BAD_CACHE] + [
    (dict(dtype=2), -1), (dict(T=-1), -2), (dict(B=70000), -2), (dict(max_new=-1), -2), (dict(rot=8), -2),
    (dict(rot=80), -2), (dict(Q=None), -1), (dict(H=0), -2), (dict(ldk=120), -2), (dict(ldk=132), -3), (dict(K=ODD), -3),
    (dict(V=None), -1), (dict(seq_start=None), -1), (dict(page_table=None), -1), (dict(pos=None), -1),
    (dict(table=ctypes.c_void_p(4104)), -3), (dict(past=ctypes.c_void_p(4098)), -3)])
def test_append_refusals(lib, changes, code):
    base = dict(cache=cache(lib), K=P, ldk=128, V=P, ldv=128, Q=P, ldq=256, Qo=P, ldqo=256, H=4, dtype=0, T=3,
                seq_start=P, past=P, B=1, max_new=3, page_table=P, table_ld=4, pos=P, table=P, positions=9, rot=64,
                interleaved=0, stream=None)
    if "cache" in changes:
        changes = dict(cache=cache(lib, **changes["cache"]))
    refuse(lib, "kv_cache_append", APPEND, base, changes, code)


READ = "cache page_table table_ld first out_start B max_rows T K V ld dtype stream".split()


@pytest.mark.parametrize("changes,code", [(dict(cache=c), r) for c, r in BAD_CACHE] + [
    (dict(dtype=3), -1), (dict(T=-1), -2), (dict(B=-1), -2), (dict(ld=64), -2), (dict(V=ODD), -3), (dict(first=None), -1)])
def test_read_refusals(lib, changes, code):
    base = dict(cache=cache(lib), page_table=P, table_ld=4, first=P, out_start=P, B=1, max_rows=3, T=3, K=P, V=P, ld=128,
                dtype=0, stream=None)
    if "cache" in changes:
        changes = dict(cache=cache(lib, **changes["cache"]))
    refuse(lib, "kv_cache_read", READ, base, changes, code)


ATTEND = ("Q ldq dtype T seq_start B max_new H cache page_table table_ld kv_len max_len causal key_mask mask_ld scale Out "
          "ldo lse workspace workspace_bytes stream").split()


@pytest.mark.parametrize("changes,code", [(dict(cache=c), r) for c, r in BAD_CACHE] + [
    (dict(dtype=2), -1), (dict(T=-1), -2), (dict(H=3), -2), (dict(H=0), -2), (dict(max_new=1 << 27), -2),
    (dict(max_len=-1), -2), (dict(key_mask=P, mask_ld=63), -2), (dict(scale=0.0), -1), (dict(scale=float("inf")), -1),
    (dict(scale=float("nan")), -1), (dict(Q=None), -1), (dict(ldq=255), -2), (dict(ldo=260), -3), (dict(Out=ODD), -3),
    (dict(kv_len=None), -1), (dict(workspace=None), -1), (dict(workspace=ctypes.c_void_p(4096 + 128)), -3)])
def test_attention_refusals(lib, changes, code):
    base = dict(Q=P, ldq=256, dtype=0, T=3, seq_start=P, B=1, max_new=3, H=4, cache=cache(lib), page_table=P, table_ld=4,
                kv_len=P, max_len=64, causal=0, key_mask=None, mask_ld=0, scale=0.125, Out=P, ldo=256, lse=None,
                workspace=P, workspace_bytes=1 << 40, stream=None)
    if "cache" in changes:
        changes = dict(cache=cache(lib, **changes["cache"]))
    refuse(lib, "kv_cache_attention", ATTEND, base, changes, code)


def test_attention_workspace(lib):
    size = lib.lib.kv_cache_attention_workspace_size
    assert size(1, 1, 28, 4, 128) > 0 and size(1, 1, 27, 4, 128) == 0 and size(1, 1, 4, 4, 96) == 0
    assert size(-1, 1, 4, 4, 64) == 0
    base = dict(Q=P, ldq=256, dtype=0, T=3, seq_start=P, B=1, max_new=3, H=4, cache=cache(lib), page_table=P, table_ld=4,
                kv_len=P, max_len=64, causal=0, key_mask=None, mask_ld=0, scale=0.125, Out=P, ldo=256, lse=None,
                workspace=P, workspace_bytes=size(1, 3, 4, 2, 64) - 1, stream=None)
    refuse(lib, "kv_cache_attention", ATTEND, base, {}, -1)


LINEAR = "X ldx dtype L K Wq scales group N bias Y ldy y_dtype stream".split()


@pytest.mark.parametrize("changes,code", [
    (dict(dtype=2), -1), (dict(y_dtype=3), -1), (dict(L=33), -2), (dict(L=-1), -2), (dict(group=16), -2),
    (dict(K=96), -2), (dict(K=0), -2), (dict(N=0), -2), (dict(ldx=120), -2), (dict(ldy=7), -2), (dict(ldx=129), -3),
    (dict(X=ODD), -3), (dict(Wq=ctypes.c_void_p(4104)), -3), (dict(Wq=None), -1), (dict(scales=None), -1),
    (dict(Y=None), -1)])
def test_w4g_linear_refusals(lib, changes, code):
    base = dict(X=P, ldx=128, dtype=0, L=3, K=128, Wq=P, scales=P, group=64, N=8, bias=None, Y=P, ldy=8, y_dtype=0,
                stream=None)
    refuse(lib, "w4g_linear", LINEAR, base, changes, code)


def test_binding_refusals(lib):
    """The binding's own checks of shapes, types and strides (host tensors:
    nothing reaches the library)."""
    t = torch.zeros
    with pytest.raises(ValueError):
        lib.KVCache(t(2, 1, 16, 64, dtype=torch.int8), t(2, 1, 16, 64, dtype=torch.int8), t(2, 1), t(2, 1))
    with pytest.raises(ValueError):
        lib.KVCache(t(2, 1, 16, 64, dtype=torch.uint8), t(2, 1, 16, 64, dtype=torch.uint8), t(2, 2), t(2, 1))
    c = lib.KVCache(t(2, 1, 16, 64, dtype=torch.uint8), t(2, 1, 16, 64, dtype=torch.uint8), t(2, 1), t(2, 1))
    i = lambda *v: torch.tensor(v, dtype=torch.int32)
    x = t(3, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        lib.kv_cache_append(c, x[:, :32], x, i(0, 3), i(0), i(0, 1)[None], None, None, max_new=3)
    with pytest.raises(ValueError):
        lib.kv_cache_append(c, x, x, torch.tensor([0, 3]), i(0), i(0, 1)[None], None, None, max_new=3)
    with pytest.raises(ValueError):
        lib.kv_cache_append(c, x, x, i(0, 3), i(0), i(0, 1)[None], None, None, max_new=3, Q=x)
    with pytest.raises(ValueError):
        lib.kv_cache_attention(x, c, i(0, 1)[None], i(3), i(0, 3), t(3, 64), max_new=3, max_len=3)
    with pytest.raises(ValueError):
        lib.kv_cache_attention(x, c, i(0, 1)[None], i(3), i(0, 3), x, max_new=3, max_len=3,
                               key_mask=t(1, 2, dtype=torch.uint8))
    with pytest.raises(ValueError):
        lib.rope_apply(x, 2, i(0, 1, 2), t(4, 32, 2), D=64)
    with pytest.raises(ValueError):
        lib.w4g_linear(x, t(8, 16, dtype=torch.uint8), t(8, 1), t(3, 8))
