"""Cases of the cached-decoding operators: rotary positions from a table, appending to a paged 8-bit key/value
cache, attention over that cache, and products of a few rows with 4-bit weights that carry group scales.

Each case has a plain form (elementary torch operations in 32 bits, rounded once at the end), the call of the
library's operator, and a 64-bit value from the operator's definition.
"""

import math

import torch

own = False

DT = {"float16": torch.float16, "bfloat16": torch.bfloat16}
SCALE_FLOOR = 2.0 ** -100        # the smallest scale of a cache block


def listed():
    return [
        # the query and key heads of four 2048-token prompts of the Dream-7B block (28 + 4 heads of 128)
        dict(name="rope_prompt", op="rope", dtype="bfloat16", tokens=8192, heads=32, dim=128, rot=128,
             interleaved=False, inverse=False, span=32768, stretch=4.0),
        # the gradient of a partly rotated, interleaved layout on an odd number of small heads
        dict(name="rope_grad_partial", op="rope", dtype="float16", tokens=333, heads=13, dim=64, rot=32,
             interleaved=True, inverse=True, span=4096, stretch=1.0),
        # one new token for each of 64 running sequences: latency
        dict(name="append_token", op="append", dtype="bfloat16", batch=64, new=1, past=700, heads=28, kv_heads=4,
             dim=128, page=64, rot=128, interleaved=False),
        # a block of 32 positions under denoising, rewritten behind a ragged prefix; 32 heads with keys of their own
        dict(name="append_block", op="append", dtype="float16", batch=8, new=32, past=1000, heads=32, kv_heads=32,
             dim=128, page=32, rot=64, interleaved=True),
        # ragged prompts of up to 2048 tokens entering the cache behind a short shared part
        dict(name="append_prompt", op="append", dtype="bfloat16", batch=4, new=2048, past=37, heads=28, kv_heads=4,
             dim=128, page=64, rot=128, interleaved=False),
        # one query token of one sequence on a short cache: latency
        dict(name="attend_one", op="attend", dtype="bfloat16", batch=1, new=1, len=777, heads=28, kv_heads=4,
             dim=128, page=64, causal=False, masked=False),
        # five drafted tokens per sequence, causal among themselves, heads of 64 on pages of 16
        dict(name="attend_draft", op="attend", dtype="float16", batch=16, new=5, len=4001, heads=16, kv_heads=2,
             dim=64, page=16, causal=True, masked=False),
        # one token for each of four sequences with long caches: the cache's bytes
        dict(name="attend_long", op="attend", dtype="bfloat16", batch=4, new=1, len=131072, heads=28, kv_heads=4,
             dim=128, page=64, causal=False, masked=False),
        # a denoising step of 32-position blocks, bidirectional, on cached prefixes with dropped positions
        dict(name="attend_block", op="attend", dtype="bfloat16", batch=8, new=32, len=16384, heads=28, kv_heads=4,
             dim=128, page=32, causal=False, masked=True),
        # the attention output projection of one token
        dict(name="matvec_square", op="matvec", dtype="float16", rows=1, n=4096, k=4096, group=128, bias=False),
        # the gate and up projections of one token (18944 channels each)
        dict(name="matvec_gate_up", op="matvec", dtype="bfloat16", rows=1, n=37888, k=3584, group=64, bias=False),
        # the down projection of a few tokens, small groups, with a bias
        dict(name="matvec_few_rows", op="matvec", dtype="float16", rows=9, n=4096, k=12288, group=32, bias=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = ((28, 4), (32, 32), (32, 8), (16, 2), (12, 3), (8, 8), (5, 5), (24, 1))


def draw(rng):
    op = rng.choice(("rope", "append", "append", "attend", "attend", "attend", "matvec", "matvec"))
    dtype = rng.choice(("float16", "bfloat16"))
    dim = rng.choice((64, 128, 128))
    if op == "rope":
        return dict(op=op, dtype=dtype, tokens=_log(rng, 1, 8192), heads=rng.randint(1, 32), dim=dim,
                    rot=rng.choice((32, 64, dim)), interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5,
                    span=32768, stretch=rng.choice((1.0, 2.5, 8.0)))
    if op == "matvec":
        group = rng.choice((32, 64, 128))
        return dict(op=op, dtype=dtype, rows=rng.choice((1, 1, 2, 3, 5, 8, 13, 16, 27, 32)), n=_log(rng, 33, 37888),
                    k=max(group, _log(rng, 128, 3584 if rng.random() < 0.5 else 12288) // group * group),
                    group=group, bias=rng.random() < 0.5)
    heads, kv_heads = rng.choice(HEADS)
    page = rng.choice((16, 32, 64, 128))
    new = rng.choice((1, 1, 2, 5, 7, 16, 32, 61))
    if op == "append":
        if rng.random() < 0.3:
            new = _log(rng, 100, 2048)
        batch = _log(rng, 1, max(1, min(64, 8192 // new)))
        return dict(op=op, dtype=dtype, batch=batch, new=new, past=_log(rng, 1, 2000) - 1, heads=heads,
                    kv_heads=kv_heads, dim=dim, page=page, rot=rng.choice((32, 64, dim)),
                    interleaved=rng.random() < 0.5)
    batch = _log(rng, 1, 64)
    length = _log(rng, 1, 131072)
    # no more cache bytes, and no more products, than the largest listed cases have
    length = min(length, (3 * 131072 * 4 * 128) // (batch * kv_heads * dim) // (2 if batch < 3 else 1))
    length = min(length, (8 * 32 * 28 * 128 * 9000) // (batch * new * heads * dim))
    return dict(op=op, dtype=dtype, batch=batch, new=new, len=max(1, length), heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, causal=rng.random() < 0.4, masked=rng.random() < 0.4)


# ---------------------------------------------------------------------------
# Lengths: functions of the case alone, ragged over the batch.
# ---------------------------------------------------------------------------
def _ragged(top, b, lowest):
    """top for the first sequence, then spread over [top / 4, top]."""
    return top if b == 0 else max(lowest, int(top * (0.25 + 0.75 * ((b * 0.6180339887) % 1.0))))


def _lengths(case):
    """(new tokens, cached tokens before, cached tokens after) of every sequence."""
    B, n = case["batch"], case["new"]
    if case["op"] == "append":
        new = [n if n <= 64 else _ragged(n, b, 1) for b in range(B)]
        past = [_ragged(case["past"], b, 0) for b in range(B)]
        return new, past, [a + p for a, p in zip(new, past)]
    return [n] * B, None, [_ragged(case["len"], b, 1) for b in range(B)]


def work(case):
    size = 2
    if case["op"] == "rope":
        values = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * size * values + case["tokens"] * (4 + 4 * case["rot"]),
                "flops": 3 * case["tokens"] * case["heads"] * case["rot"]}
    if case["op"] == "matvec":
        m, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": n * k // 2 + 4 * n * (k // case["group"]) + size * m * (k + n) + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    new, past, total = _lengths(case)
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    T = sum(new)
    if case["op"] == "append":
        held = sum(t - p // page * page for t, p in zip(total, past))      # the touched blocks, read back
        blocks = sum((t + page - 1) // page - p // page for t, p in zip(total, past))
        rows = T * D * (2 * H + 2 * Hkv) * size + T * 2 * Hkv * D          # rows in, queries out, codes out
        back = held * 2 * Hkv * D * (1 + size)                             # codes in, values out
        return {"bytes": rows + back + blocks * 2 * Hkv * 4 + T * (4 + 4 * case["rot"]),
                "flops": 3 * T * (H + Hkv) * case["rot"] + 4 * T * Hkv * D}
    L = sum(total)
    blocks = sum((t + page - 1) // page for t in total)
    pairs = sum(n * t for n, t in zip(new, total))
    if case["causal"]:
        pairs = sum(sum(max(0, t - n + i + 1) for i in range(n)) for n, t in zip(new, total))
    return {"bytes": L * 2 * Hkv * D + blocks * (2 * Hkv * 4 + 4) + 2 * T * H * D * size + T * H * 4
            + (L if case["masked"] else 0),
            "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _table(span, rot, stretch, device="cuda"):
    """cos and sin of position / stretch * 10000^(-2 i / rot), from 64 bits: [span][rot / 2][2]."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(span, dtype=torch.float64, device=device)[:, None] / stretch * f
    return torch.stack([a.cos(), a.sin()], dim=-1).float().contiguous()


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _cache(case, g, tokens):
    """A paged cache whose sequences hold `tokens` each: codes (byte = code + 128), scales and page table. Pages lie in a
    random order; pages that no sequence uses hold stale codes and no valid scale."""
    Hkv, D, page = case["kv_heads"], case["dim"], case["page"]
    need = [(t + page - 1) // page for t in tokens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda")
    width = max(1, max(need))
    first = torch.tensor(_starts(need)[:-1], device="cuda")[:, None]
    col = torch.arange(width, device="cuda")[None, :]
    used = col < torch.tensor(need, device="cuda")[:, None]
    table = torch.where(used, order[(first + col).clamp(max=pages - 1)], -1).to(torch.int32).contiguous()
    codes, scales = [], []
    for _ in range(2):
        c = torch.empty(pages, Hkv, page, D, device="cuda", dtype=torch.float16).normal_(0.0, 36.0, generator=g)
        codes.append(c.round_().clamp_(-127, 127).add_(128).to(torch.uint8))
        s = (torch.rand(pages, Hkv, generator=g, device="cuda") + 0.5) / 36.0
        s[order[sum(need):]] = float("nan")
        scales.append(s)
    return dict(K=codes[0], V=codes[1], k_scale=scales[0], v_scale=scales[1], table=table)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dt = DT[case["dtype"]]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)
    st = dict(case=case)
    if case["op"] == "rope":
        T, H, D = case["tokens"], case["heads"], case["dim"]
        st["x"] = randn(T, H * D)
        start = int(torch.randint(0, case["span"] - T + 1, (1,), generator=g, device="cuda")) if case["span"] > T else 0
        st["pos"] = torch.arange(start, start + T, dtype=torch.int32, device="cuda")
        st["table"] = _table(case["span"], case["rot"], case["stretch"])
        st["y"] = torch.empty_like(st["x"])
        return st
    if case["op"] == "matvec":
        m, n, k, gs = case["rows"], case["n"], case["k"], case["group"]
        st["x"] = randn(m, k)
        codes = torch.randint(-7, 8, (n, k), generator=g, device="cuda", dtype=torch.int16)
        st["w"] = ((codes[:, 0::2] & 15) | ((codes[:, 1::2] & 15) << 4)).to(torch.uint8).contiguous()
        st["scales"] = (torch.rand(n, k // gs, generator=g, device="cuda") + 0.5) * (0.3 / math.sqrt(k))
        st["bias"] = torch.randn(n, generator=g, device="cuda") if case["bias"] else None
        st["y"] = torch.empty(m, n, dtype=dt, device="cuda")
        return st
    new, past, total = _lengths(case)
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    st["cache"] = _cache(case, g, total)
    st["start"] = _i32(_starts(new))
    st["max_new"] = max(new)
    T = sum(new)
    if case["op"] == "append":
        # queries, keys and values side by side, as a fused projection leaves them; keys with a few large channels
        st["qkv"] = randn(T, (H + 2 * Hkv) * D)
        loud = torch.randint(0, Hkv * D, (max(1, Hkv * D // 32),), generator=g, device="cuda")
        st["qkv"][:, H * D:(H + Hkv) * D][:, loud] *= 6
        st["q_out"] = torch.empty(T, H * D, dtype=dt, device="cuda")
        st["past"] = _i32(past)
        st["table"] = _table(4096 + max(total), case["rot"], 1.0)
        at = [torch.arange(p, p + n) for p, n in zip(past, new)]
        st["pos"] = torch.cat(at).to(torch.int32).cuda()
        st["seq"] = torch.cat([torch.full((n,), b) for b, n in enumerate(new)]).cuda()
        # the touched blocks, from the first block's first token on
        first = [p // page * page for p in past]
        held = [t - f for t, f in zip(total, first)]
        st["first"], st["held_start"], st["max_held"] = _i32(first), _i32(_starts(held)), max(held)
        st["held_seq"] = torch.cat([torch.full((n,), b) for b, n in enumerate(held)]).cuda()
        st["held_slot"] = torch.cat([torch.arange(f, f + n) for f, n in zip(first, held)]).cuda()
        st["k_out"] = torch.empty(sum(held), Hkv * D, dtype=dt, device="cuda")
        st["v_out"] = torch.empty_like(st["k_out"])
        return st
    st["q"] = randn(T, H * D)
    st["len"] = _i32(total)
    st["max_len"] = max(total)
    st["mask"] = None
    if case["masked"]:
        st["mask"] = (torch.rand(case["batch"], max(total), generator=g, device="cuda") < 0.9).to(torch.uint8)
        st["mask"][-1] = 0                      # every cached position of the last sequence is dropped
        if case["batch"] == 1:
            st["mask"][0, : max(total) // 2 + 1] = 1
    st["out"] = torch.empty(T, H * D, dtype=dt, device="cuda")
    st["lse"] = torch.empty(T, H, device="cuda")
    return st


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _rotate(x, cs, rot, interleaved, inverse=False):
    """x [T][heads][D] in 32 bits, cs [T][rot / 2][2]: the first rot channels of each head turned by their angles."""
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if inverse:
        s = -s
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_rope(st):
    c, x = st["case"], st["x"]
    y = _rotate(x.float().view(c["tokens"], c["heads"], c["dim"]), st["table"][st["pos"].long()], c["rot"],
                c["interleaved"], c["inverse"])
    return y.reshape(x.shape).to(x.dtype)


def _plain_matvec(st):
    c = st["case"]
    w = st["w"].to(torch.int32)
    codes = torch.stack([w & 15, w >> 4], dim=-1).flatten(-2)
    codes = torch.where(codes > 7, codes - 16, codes).float()
    weight = (codes.view(c["n"], -1, c["group"]) * st["scales"][..., None]).view(c["n"], c["k"])
    y = st["x"].float() @ weight.T
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(st["x"].dtype)


def _store(codes, scales, x, page_of, slot, touched, kept, page):
    """Quantises the rows x [T][Hkv][D] into their blocks: a block's scale covers its new rows and is never less than the
    scale of the rows that it keeps, whose codes are rounded again to it."""
    top = torch.zeros_like(scales).index_reduce_(0, page_of, x.abs().amax(-1), "amax")
    old = torch.where(kept[:, None] > 0, scales, 0.0)
    new = torch.maximum(torch.maximum(old, top / 127.0), torch.full_like(old, SCALE_FLOOR))
    new = torch.where(touched[:, None], new, scales)
    at = touched.nonzero()[:, 0]
    ratio = torch.where(kept[at, None] > 0, old[at] / new[at], 1.0)[:, :, None, None]
    again = ((codes[at].float() - 128.0) * ratio).round() + 128.0
    keep = (torch.arange(page, device="cuda")[None, :] < kept[at, None])[:, None, :, None]
    codes[at] = torch.where(keep, again.to(torch.uint8), codes[at])
    rows = (x * (1.0 / new[page_of])[:, :, None]).round().clamp(-127, 127) + 128.0
    codes[page_of, :, slot % page] = rows.to(torch.uint8)
    scales.copy_(new)


def _plain_append(st):
    c, cache = st["case"], st["cache"]
    H, Hkv, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    T = st["qkv"].shape[0]
    x = st["qkv"].float().view(T, H + 2 * Hkv, D)
    cs = st["table"][st["pos"].long()]
    turned = _rotate(x[:, : H + Hkv], cs, c["rot"], c["interleaved"])
    slot = st["pos"].long()
    page_of = cache["table"][st["seq"], slot // page].long()
    touched = torch.zeros(cache["K"].shape[0], dtype=torch.bool, device="cuda").index_fill_(0, page_of, True)
    past = st["past"].long()
    kept = torch.zeros(cache["K"].shape[0], dtype=torch.long, device="cuda")
    part = cache["table"].gather(1, (past // page).clamp(max=cache["table"].shape[1] - 1)[:, None])[:, 0].long()
    kept[part] = past % page
    _store(cache["K"], cache["k_scale"], turned[:, H:], page_of, slot, touched, kept, page)
    _store(cache["V"], cache["v_scale"], x[:, H + Hkv:], page_of, slot, touched, kept, page)
    p = cache["table"][st["held_seq"], st["held_slot"] // page].long()
    s = st["held_slot"] % page
    dt = st["qkv"].dtype
    value = lambda codes, scales: ((codes[p, :, s].float() - 128.0) * scales[p][:, :, None]).flatten(1).to(dt)
    return {"q": turned[:, :H].reshape(T, H * D).to(dt), "k": value(cache["K"], cache["k_scale"]),
            "v": value(cache["V"], cache["v_scale"])}


def _plain_attend(st):
    c, cache = st["case"], st["cache"]
    B, n, H, Hkv, D, page = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    G = H // Hkv
    at = cache["table"].long().clamp(min=0)
    P = at.shape[1]
    value = lambda codes, scales: ((codes[at].float() - 128.0) * scales[at][..., None, None]) \
        .permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * page, D)
    q = st["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    s = (q @ value(cache["K"], cache["k_scale"]).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    j = torch.arange(P * page, device="cuda")
    length = st["len"].long()
    seen = (j[None, :] < length[:, None])[:, None, :].expand(B, n, -1)
    if c["causal"]:
        last = length[:, None] - n + torch.arange(n, device="cuda")[None, :]
        seen = seen & (j[None, None, :] <= last[:, :, None])
    if st["mask"] is not None:
        seen = seen & (torch.nn.functional.pad(st["mask"], (0, P * page - st["mask"].shape[1])) != 0)[:, None, :]
    seen = seen[:, None, :, None, :].expand(B, 1, n, G, P * page).reshape(B, 1, n * G, P * page)
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    del s
    total = p.sum(-1, keepdim=True)
    o = (p @ value(cache["V"], cache["v_scale"])) / torch.where(total > 0, total, 1.0)
    lse = (m + torch.log(total))[..., 0]
    back = lambda t: t.reshape(B, Hkv, n, G, -1).permute(0, 2, 1, 3, 4)
    return {"out": back(o).reshape(B * n, H * D).to(st["q"].dtype), "lse": back(lse).reshape(B * n, H)}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2606_04945_gb300 import abi

    c = st["case"]
    if c["op"] == "rope":
        abi.rope_apply(st["x"], c["heads"], st["pos"], st["table"], st["y"], interleaved=c["interleaved"],
                       inverse=c["inverse"])
        return st["y"]
    if c["op"] == "matvec":
        abi.w4g_linear(st["x"], st["w"], st["scales"], st["y"], bias=st["bias"])
        return st["y"]
    t = st["cache"]
    cache = abi.KVCache(t["K"], t["V"], t["k_scale"], t["v_scale"])
    if c["op"] == "append":
        H, Hkv, D = c["heads"], c["kv_heads"], c["dim"]
        qkv = st["qkv"]
        abi.kv_cache_append(cache, qkv[:, H * D:(H + Hkv) * D], qkv[:, (H + Hkv) * D:], st["start"], st["past"],
                            t["table"], st["pos"], st["table"], max_new=st["max_new"], Q=qkv[:, : H * D],
                            Q_out=st["q_out"], interleaved=c["interleaved"])
        abi.kv_cache_read(cache, t["table"], st["first"], st["held_start"], st["k_out"], st["v_out"],
                          max_rows=st["max_held"])
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    abi.kv_cache_attention(st["q"], cache, t["table"], st["len"], st["start"], st["out"], max_new=st["max_new"],
                           max_len=st["max_len"], causal=c["causal"], key_mask=st["mask"], lse=st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


PLAIN = {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "matvec": _plain_matvec}


def run(st):
    return _own(st) if own else PLAIN[st["case"]["op"]](st)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _turn64(x, table, pos, rot, interleaved, sign):
    """Pairs as complex numbers, multiplied by exp(i angle)."""
    t = table.double()[pos.long()]
    w = torch.complex(t[..., 0], sign * t[..., 1])[:, None, :]
    i = torch.arange(rot // 2, device="cuda")
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    out = x.double().clone()
    z = torch.complex(out[..., lo], out[..., hi]) * w
    out[..., lo], out[..., hi] = z.real, z.imag
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        x = st["x"].view(case["tokens"], case["heads"], case["dim"])
        y = _turn64(x, st["table"], st["pos"], case["rot"], case["interleaved"], -1.0 if case["inverse"] else 1.0)
        return y.reshape(st["x"].shape)
    if case["op"] == "matvec":
        n, k, gs = case["n"], case["k"], case["group"]
        x = st["x"].double()
        y = torch.zeros(case["rows"], n, dtype=torch.float64, device="cuda")
        for a in range(0, n, 4096):
            w = st["w"][a:a + 4096]
            codes = torch.empty(w.shape[0], k, dtype=torch.float64, device="cuda")
            codes[:, 0::2], codes[:, 1::2] = (w % 16).double(), (w // 16).double()
            codes = (codes + 8) % 16 - 8
            codes *= st["scales"][a:a + 4096].double().repeat_interleave(gs, dim=1)
            y[:, a:a + 4096] = x @ codes.T
        return y if st["bias"] is None else y + st["bias"].double()
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    new, past, total = _lengths(case)
    cache, at = st["cache"], _starts(new)
    pages = cache["table"].cpu()
    if case["op"] == "append":
        x = st["qkv"].double().view(-1, H + 2 * Hkv, D)
        turned = _turn64(x[:, : H + Hkv], st["table"], st["pos"], case["rot"], case["interleaved"], 1.0)
        held = {"k": [], "v": []}
        for b in range(case["batch"]):
            for name, codes, scales, rows in (("k", cache["K"], cache["k_scale"], turned[at[b]:at[b + 1], H:]),
                                              ("v", cache["V"], cache["v_scale"], x[at[b]:at[b + 1], H + Hkv:])):
                for blk in range(past[b] // page, (total[b] + page - 1) // page):
                    p, lo = int(pages[b, blk]), max(past[b], blk * page)
                    mine = rows[lo - past[b]: min(total[b], (blk + 1) * page) - past[b]].transpose(0, 1)
                    s = mine.abs().amax((1, 2)) / 127.0
                    kept = lo - blk * page
                    if kept:
                        old = scales[p].double()
                        s = torch.maximum(s, old)
                        before = codes[p, :, :kept].double() - 128
                        mine_codes = torch.cat([(before * (old / s)[:, None, None]).round(),
                                                (mine / s[:, None, None]).round()], dim=1)
                    else:
                        mine_codes = (mine / s[:, None, None]).round()
                    held[name].append((mine_codes * s[:, None, None]).transpose(0, 1).reshape(-1, Hkv * D))
        return {"q": turned[:, :H].reshape(-1, H * D), "k": torch.cat(held["k"]), "v": torch.cat(held["v"])}
    G = H // Hkv
    out = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(new), H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        L, n = total[b], new[b]
        p = pages[b, : (L + page - 1) // page].long().cuda()
        for h in range(Hkv):
            k = ((cache["K"][p, h].double() - 128) * cache["k_scale"][p, h].double()[:, None, None]).view(-1, D)[:L]
            v = ((cache["V"][p, h].double() - 128) * cache["v_scale"][p, h].double()[:, None, None]).view(-1, D)[:L]
            q = st["q"][at[b]:at[b + 1], h * G * D:(h + 1) * G * D].double().reshape(n, G, D)
            s = torch.einsum("ngd,ld->ngl", q, k) / math.sqrt(D)
            if case["causal"]:
                late = torch.arange(L, device="cuda")[None, :] > (L - n + torch.arange(n, device="cuda"))[:, None]
                s.masked_fill_(late[:, None, :], -math.inf)
            if st["mask"] is not None:
                s.masked_fill_(st["mask"][b, :L] == 0, -math.inf)
            row = torch.logsumexp(s, dim=-1)
            w = torch.exp(s - row.nan_to_num(neginf=0.0)[..., None])
            out[at[b]:at[b + 1], h * G:(h + 1) * G] = torch.einsum("ngl,ld->ngd", w, v)
            lse[at[b]:at[b + 1], h * G:(h + 1) * G] = row
    return {"out": out.reshape(-1, H * D), "lse": lse}
