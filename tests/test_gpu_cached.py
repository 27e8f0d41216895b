"""Block-wise denoising behind a cached prefix (cached.py): every operator of
every pass against oracle/decode.py on the GPU's own inputs (the tolerances
are those of test_gpu_decode.py), and what a step must not change.
"""

import numpy as np
import pytest
import torch

from oracle import decode as od
from oracle import sgat as osg

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -149}
num = lambda t: t.detach().double().cpu().numpy()

SHAPES = [
    # 16 rows a key/value head; steps that do not divide the block; a page ends inside the blocks
    dict(hidden=256, ffn=512, heads=4, kv_heads=2, dim=64, layers=2, vocab=500, batch=2, block=8, unmask_per_step=3,
         capacity=96, page=16, group=32, dtype=torch.float16),
    # 96 rows a key/value head; positions past the trained length
    dict(hidden=512, ffn=384, heads=6, kv_heads=2, dim=128, layers=2, vocab=333, batch=1, block=32, unmask_per_step=16,
         capacity=160, page=32, group=64, scaling="parts", factor=4.0, original=64.0),
]


class Mirror:
    """The caches of the stack on the oracle's side, and the checks."""

    def __init__(self, stack):
        self.stack, self.c = stack, stack.cfg
        self.table = stack.page_table.cpu().numpy()
        self.rope = stack.rope.cpu().numpy()
        side = lambda t: t.cpu().numpy().astype(np.int64) - 128
        self.k, self.v = ([side(getattr(x, n)) for x in stack.caches] for n in "KV")
        self.ks, self.vs = ([getattr(x, n).cpu().numpy() for x in stack.caches] for n in ("k_scale", "v_scale"))
        self.seen = []

    def __call__(self, layer, name, values):
        self.seen.append(name)
        if name == "append":
            self.append(layer, *values)
        elif name == "attention":
            self.attention(layer, *values)
        else:
            self.linear(*values)

    def linear(self, m, X, Y):
        codes, scales = osg.unpack_int4(m.Wq.cpu().numpy()), m.scales.cpu().numpy()
        ref, size = od.w4g_linear(num(X), codes, scales, None if m.bias is None else m.bias.cpu().numpy())
        tol = (m.K / 8 + 16) * 2.0 ** -24 * size + U[Y.dtype] * np.abs(ref) * 1.01 + TINY[Y.dtype]
        assert np.all(np.abs(num(Y) - ref) <= tol)

    def append(self, i, cache, qkv, q_out, pos):
        c, f = self.c, np.float32
        past, n, x, pos = self.stack.past.cpu().numpy(), len(qkv) // c.batch, num(qkv).astype(f), pos.cpu().numpy()
        heads = x.reshape(len(x), -1, c.dim)
        turned = od.rope(heads[:, : c.heads + c.kv_heads], pos, self.rope, False, dtype=f)
        ref = torch.from_numpy(turned[:, : c.heads].reshape(len(x), -1)).to(c.dtype)
        assert torch.equal(q_out.cpu(), ref)
        for b in range(c.batch):
            r = slice(b * n, (b + 1) * n)
            od.append(self.k[i], self.ks[i], self.table[b], past[b], turned[r, c.heads:], c.page)
            od.append(self.v[i], self.vs[i], self.table[b], past[b], heads[r, c.heads + c.kv_heads:], c.page)
        for got, ref, scale, rs in ((cache.K, self.k, cache.k_scale, self.ks), (cache.V, self.v, cache.v_scale, self.vs)):
            assert np.array_equal(scale.cpu().numpy(), rs[i])
            got = got.cpu().numpy().astype(np.int64) - 128
            for b in range(c.batch):
                for s in range(past[b] + n):
                    p = self.table[b, s // c.page]
                    assert np.array_equal(got[p, :, s % c.page], ref[i][p, :, s % c.page]), (b, s)

    def attention(self, i, cache, q, held, out):
        c = self.c
        q, out, held = num(q).reshape(-1, c.heads, c.dim), num(out).reshape(-1, c.heads, c.dim), held.cpu().numpy()
        n = len(q) // c.batch
        for b, L in enumerate(held):
            r = slice(b * n, (b + 1) * n)
            k, v = (od.read(x[i], s[i], self.table[b], 0, L, c.page) for x, s in ((self.k, self.ks), (self.v, self.vs)))
            ref, _, mag, size = od.attention(q[r], k, v, c.dim ** -0.5)
            d = ((c.dim + 4) * 2.0 ** -24 * size)[..., None]
            rel = 2 * (2 * d + 2.0 ** -20) + 2.0 ** -11 + L * 2.0 ** -24 + 2.0 ** -20
            assert np.all(np.abs(out[r] - ref) <= mag * rel + U[c.dtype] * np.abs(ref) * (1 + rel) + TINY[c.dtype])


def made(shape):
    from paper_2606_04945_gb300.cached import CachedConfig, CachedStack
    stack = CachedStack(CachedConfig(**shape))
    rng = np.random.default_rng(shape["vocab"])
    prompt = torch.from_numpy(rng.integers(1, shape["vocab"], (shape["batch"], 37))).cuda()
    return stack, prompt, rng


@pytest.mark.parametrize("shape", SHAPES)
def test_operators_of_every_pass(abi, shape):
    """A prompt, two steps of a block, its final pass, and a pass of the next
    block."""
    stack, prompt, rng = made(shape)
    c = stack.cfg
    mirror = Mirror(stack)
    stack.past.zero_()
    stack.forward(prompt, mirror)
    stack.keep(prompt.shape[1])
    for last in (False, False, True, False):
        tok = torch.from_numpy(rng.integers(0, c.vocab, (c.batch, c.block))).cuda()
        logits = stack.forward(tok, mirror)
        assert torch.isfinite(logits).all()
        if last:
            stack.keep(c.block)
    abi.check_status()
    assert mirror.seen == (["qkv", "append", "attention", "o", "gu", "down"] * c.layers + ["head"]) * 5


@pytest.mark.parametrize("shape", SHAPES)
def test_generate(abi, shape):
    """Replayed passes give the eager ones' tokens; every position is
    unmasked; a further pass over the last block's final tokens behind its
    prefix leaves the caches as they are, bit for bit. (Scales that other
    tokens' rows have grown stay grown, so a fresh stack that never saw the
    masked steps may hold other codes.)"""
    stack, prompt, _ = made(shape)
    c = stack.cfg
    tokens = stack.generate(prompt, 2)
    assert tokens.shape == (c.batch, 2 * c.block) and bool((tokens != stack.mask_id).all())
    assert stack.held == 37 + 2 * c.block == int(stack.past[0])
    rows = lambda: [(x.K.clone(), x.V.clone(), x.k_scale.clone(), x.v_scale.clone()) for x in stack.caches]
    after = rows()
    stack.keep(-c.block)
    stack.forward(tokens[:, -c.block:])
    assert all(torch.equal(p, q) for x, y in zip(after, rows()) for p, q in zip(x, y))
    stack.prefill(prompt)
    assert torch.equal(stack.generate(prompt, 2, stack.capture()), tokens)
    abi.check_status()


def test_refusals():
    stack, prompt, _ = made(SHAPES[0])
    with pytest.raises(ValueError):
        stack.generate(prompt, 8)
    with pytest.raises(ValueError):
        stack.prefill(torch.ones(2, 97, dtype=torch.long, device="cuda"))
