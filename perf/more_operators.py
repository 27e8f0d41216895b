"""Cases of the operators that serve long contexts, answers that share a prompt, and rules on the tokens: attention over
the paged 8-bit cache with a sliding window behind a few first tokens, attention of sequences that share a long prefix,
logits under penalties, biases and masks, and the most likely token under them with its confidence.

Each case has a plain form (elementary torch operations in 32 bits, rounded once at the end), the call of the
library's operator, and a 64-bit value from the operator's definition.
"""

import math

import torch

own = False

DT = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}


def listed():
    return [
        # the next token of one running sequence whose layers see the last 1024 tokens and four first ones: latency
        dict(name="window_one", op="window", dtype="bfloat16", batch=1, new=1, len=20000, window=1024, sinks=4, heads=28,
             kv_heads=4, dim=128, page=64, causal=False, masked=False),
        # the next tokens of 64 running sequences on ragged caches, a wide window: the window's bytes
        dict(name="window_batch", op="window", dtype="bfloat16", batch=64, new=1, len=32768, window=4096, sinks=4,
             heads=28, kv_heads=4, dim=128, page=64, causal=False, masked=False),
        # five drafted tokens per sequence, causal among themselves, an odd window, heads of 64 on pages of 16
        dict(name="window_draft", op="window", dtype="float16", batch=16, new=5, len=4001, window=501, sinks=0, heads=16,
             kv_heads=2, dim=64, page=16, causal=True, masked=False),
        # a slice of a long prompt, causal, behind the slices before it
        dict(name="window_prompt", op="window", dtype="bfloat16", batch=1, new=2048, len=8192, window=1024, sinks=16,
             heads=28, kv_heads=4, dim=128, page=64, causal=True, masked=False),
        # one token each of three answers to one short prompt: latency
        dict(name="shared_few", op="shared", dtype="bfloat16", batch=3, groups=1, new=1, shared=1024, own=100, heads=28,
             kv_heads=4, dim=128, page=64, causal=False, masked=False),
        # the next tokens of 64 requests behind two long system prompts
        dict(name="shared_requests", op="shared", dtype="bfloat16", batch=64, groups=2, new=1, shared=32768, own=500,
             heads=28, kv_heads=4, dim=128, page=64, causal=False, masked=False),
        # eight answers under denoising in blocks of 32 positions behind one prompt, with dropped positions
        dict(name="shared_blocks", op="shared", dtype="float16", batch=8, groups=1, new=32, shared=8192, own=777, heads=32,
             kv_heads=8, dim=128, page=32, causal=False, masked=True),
        # the logits of one new token for each of 64 requests with settings of their own, on their way to a sampler
        dict(name="rules_requests", op="rules", dtype="float32", batch=64, new=1, vocab=50257, pad=0, history=777, biases=40,
             by_row=False, masked=True),
        # drafted runs of five tokens, a grammar's mask for each position, 16-bit logits
        dict(name="rules_draft", op="rules", dtype="bfloat16", batch=16, new=5, vocab=131072, pad=0, history=2000, biases=0,
             by_row=True, masked=True),
        # greedy choice of one sequence's next token: latency
        dict(name="pick_one", op="pick", dtype="float32", batch=1, new=1, vocab=32000, pad=0, history=300, biases=5,
             by_row=False, masked=False, kind="probability"),
        # which of 32 masked positions of eight answers to fix: the margin between the two best tokens, a padded head
        dict(name="pick_blocks", op="pick", dtype="float32", batch=8, new=32, vocab=131072, pad=64, history=1500, biases=40,
             by_row=False, masked=True, kind="margin"),
        # the same by entropy over 16-bit logits of an odd vocabulary, a grammar's mask for each position
        dict(name="pick_entropy", op="pick", dtype="bfloat16", batch=4, new=61, vocab=50257, pad=0, history=4096, biases=0,
             by_row=True, masked=True, kind="entropy"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = ((28, 4), (32, 32), (32, 8), (16, 2), (12, 3), (8, 8), (5, 5), (24, 1))


def draw(rng):
    op = rng.choice(("window", "window", "shared", "shared", "rules", "pick", "pick"))
    if op in ("rules", "pick"):
        vocab = _log(rng, 17, 131072)
        new = rng.choice((1, 1, 2, 5, 16, 32, 61))
        batch = _log(rng, 1, max(1, min(64, (256 if op == "pick" else 80) * 131072 // (vocab * new))))
        case = dict(op=op, dtype=rng.choice(("float32", "float32", "bfloat16", "float16")), batch=batch, new=new,
                    vocab=vocab, pad=rng.choice((0, 0, 1, 64)), history=_log(rng, 1, 5000) - 1,
                    biases=rng.choice((0, 1, 40, 300)), by_row=rng.random() < 0.5, masked=rng.random() < 0.6)
        if op == "pick":
            case["kind"] = rng.choice(("probability", "margin", "entropy"))
        return case
    heads, kv_heads = rng.choice(HEADS)
    dim, page = rng.choice((64, 128, 128)), rng.choice((16, 32, 64, 128))
    new = rng.choice((1, 1, 2, 5, 7, 16, 32, 61))
    case = dict(op=op, dtype=rng.choice(("float16", "bfloat16")), new=new, heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, causal=rng.random() < 0.5, masked=rng.random() < 0.3)
    # no more cache bytes, and no more products, than the largest listed cases have
    room = 64 * 20000 * 4 * 128 // (kv_heads * dim)
    pairs = 2048 * 28 * 128 * 1024 // (heads * dim)
    if op == "window":
        if rng.random() < 0.2:
            case["new"] = new = _log(rng, 100, 2048)
        batch = _log(rng, 1, max(1, min(64, 4096 // new)))
        length = min(_log(rng, 1, 32768), room // batch)
        window = _log(rng, 1, 8192)
        window = min(window, max(1, pairs // (batch * new)))
        return dict(case, batch=batch, len=max(new, length), window=window, sinks=rng.choice((0, 1, 4, 16, 130)))
    batch = _log(rng, 1, 64)
    shared = min(_log(rng, page, 32768), room // batch, pairs // (batch * new))
    return dict(case, batch=batch, groups=rng.randint(1, max(1, min(4, batch))), shared=max(1, shared),
                own=max(new, min(_log(rng, 1, 1000), room // (8 * batch))))


# ---------------------------------------------------------------------------
# Lengths: functions of the case alone, ragged over the batch.
# ---------------------------------------------------------------------------
def _ragged(top, b, lowest):
    """top for the first sequence, then spread over [top / 4, top]."""
    return top if b == 0 else max(lowest, int(top * (0.25 + 0.75 * ((b * 0.6180339887) % 1.0))))


def _starts(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _groups(case):
    """(first sequence of every group and the end, shared tokens of every group)."""
    B, P, page = case["batch"], case["groups"], case["page"]
    first = [B * g // P for g in range(P + 1)]
    # prompts end with a page, but for the odd one
    shared = [_ragged(case["shared"], g, 1) for g in range(P)]
    return first, [s // page * page if s > page and g % 3 != 2 else s for g, s in enumerate(shared)]


def _lengths(case):
    """Cached tokens of every sequence, the new ones among them."""
    B, n = case["batch"], case["new"]
    if case["op"] == "window":
        return [_ragged(case["len"], b, n) for b in range(B)]
    first, shared = _groups(case)
    group = [max(g for g in range(case["groups"]) if first[g] <= b) for b in range(B)]
    return [shared[group[b]] + _ragged(case["own"], b, n) for b in range(B)]


def _rules_lengths(case):
    """Tokens of every sequence's history, entries of its list of biases."""
    B = case["batch"]
    history = [_ragged(case["history"], b, 0) for b in range(B)]
    return history, [case["biases"] - (b % 3 if case["biases"] > 2 else 0) for b in range(B)]


def work(case):
    B, n = case["batch"], case["new"]
    T = B * n
    if case["op"] in ("rules", "pick"):
        size = 4 if case["dtype"] == "float32" else 2
        history, biases = _rules_lengths(case)
        values = T * case["vocab"]
        bytes_ = values * size + 4 * sum(history) + 8 * sum(biases) + 16 * B + 8 * B
        if case["masked"]:
            bytes_ += (T if case["by_row"] else B) * ((case["vocab"] + 31) // 32) * 4
        if case["op"] == "rules":
            return {"bytes": bytes_ + values * size, "flops": 2 * values}
        return {"bytes": bytes_ + 12 * T, "flops": (6 if case["kind"] == "entropy" else 4) * values}
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    total = _lengths(case)
    pairs = held = blocks = 0
    for t in total:
        for i in range(n):
            end = max(0, t - n + i + 1) if case["causal"] else t
            if case["op"] == "window":
                low = max(0, min(end, t - n + i - case["window"] + 1))
                pairs += end - low + min(low, case["sinks"])
            else:
                pairs += end
        if case["op"] == "window":
            low = max(0, min(t, t - n - case["window"] + 1))
            keys = t - low + min(low, case["sinks"])
            held += keys
            blocks += (keys + page - 1) // page
    if case["op"] == "shared":
        first, shared = _groups(case)
        # a group's prefix once, and what each sequence has of its own
        held = sum(total) - sum(s * (first[g + 1] - first[g] - 1) for g, s in enumerate(shared))
        blocks = (held + page - 1) // page
    mask = 0
    if case["masked"]:
        mask = held
    return {"bytes": held * 2 * Hkv * D + blocks * (2 * Hkv * 4 + 4) + 2 * T * H * D * 2 + T * H * 4 + mask,
            "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(case, g, total):
    """A paged cache: codes (byte = code + 128), scales and page table. Pages lie in a random order; the sequences of a
    group have the pages of their shared tokens in common; pages that nothing uses hold stale codes and no valid scale."""
    Hkv, D, page, B = case["kv_heads"], case["dim"], case["page"], case["batch"]
    need = [(t + page - 1) // page for t in total]
    width = max(need)
    names, used = torch.full((B, width), -1, dtype=torch.long), 0
    if case["op"] == "shared":
        first, shared = _groups(case)
        for p in range(case["groups"]):
            common = (shared[p] + page - 1) // page
            for b in range(first[p], first[p + 1]):
                names[b, :common] = torch.arange(used, used + common)
            used += common
            for b in range(first[p], first[p + 1]):
                names[b, common:need[b]] = torch.arange(used, used + need[b] - common)
                used += need[b] - common
    else:
        for b in range(B):
            names[b, :need[b]] = torch.arange(used, used + need[b])
            used += need[b]
    pages = used + 3
    order = torch.randperm(pages, generator=g, device="cuda")
    names = names.cuda()
    table = torch.where(names >= 0, order[names.clamp(min=0)], -1).to(torch.int32).contiguous()
    codes, scales = [], []
    for _ in range(2):
        c = torch.empty(pages, Hkv, page, D, device="cuda", dtype=torch.float16).normal_(0.0, 36.0, generator=g)
        codes.append(c.round_().clamp_(-127, 127).add_(128).to(torch.uint8))
        s = (torch.rand(pages, Hkv, generator=g, device="cuda") + 0.5) / 36.0
        s[order[used:]] = float("nan")
        scales.append(s)
    return dict(K=codes[0], V=codes[1], k_scale=scales[0], v_scale=scales[1], table=table)


def _prepare_rules(case, g):
    B, n, V = case["batch"], case["new"], case["vocab"]
    T, dt = B * n, DT[case["dtype"]]
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")
    st = dict(case=case, start=_i32(_starts([n] * B)))
    rows = torch.randn(T, V + case["pad"], generator=g, device="cuda") * 2.5
    lengths, biases = _rules_lengths(case)
    # what was written before: common tokens often, and the model likes to write them again
    ld = max(1, max(lengths))
    st["history"] = (rand(B, ld) ** 3 * V).long().clamp(max=V - 1).to(torch.int32)
    st["history_len"] = _i32(lengths)
    again = st["history"].long().repeat_interleave(n, 0)
    rows.scatter_add_(1, again, torch.full_like(again, 0.05, dtype=torch.float32))
    # temperature, repetition, presence and frequency penalties of every request; the first asks for none
    st["params"] = torch.stack([rand(B) * 1.2 + 0.3, rand(B) * 0.5 + 1.0, rand(B) * 0.6, rand(B) * 0.3], 1)
    st["params"][0] = torch.tensor([1.0, 1.0, 0.0, 0.0], device="cuda")
    st["params"] = st["params"].contiguous()
    st["bias_ids"] = st["bias_values"] = st["bias_len"] = None
    if case["biases"]:
        # ids of a list differ, but for one that is given again: then the later value counts
        ids = (rand(B, case["biases"]) * V).long().clamp(max=V - 1)
        st["bias_ids"] = ids.to(torch.int32)
        st["bias_values"] = torch.randn(B, case["biases"], generator=g, device="cuda") * 4
        st["bias_len"] = _i32(biases)
    st["allowed"] = None
    if case["masked"]:
        R = T if case["by_row"] else B
        words = (V + 31) // 32
        density = torch.tensor([0.02, 0.5, 0.98], device="cuda")[(rand(R) * 3).long().clamp(max=2)]
        bits = rand(R, words * 32) < density[:, None]
        bits[R - 1] = R == 1                    # the last mask leaves nothing
        v = (bits.view(R, words, 32).long() << torch.arange(32, device="cuda")).sum(-1)
        st["allowed"] = torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(torch.int32).contiguous()
    st["x"] = rows.to(dt)[:, :V]
    if case["op"] == "rules":
        st["y"] = torch.empty(T, V + case["pad"], dtype=dt, device="cuda")[:, :V]
    else:
        st["token"] = torch.empty(T, dtype=torch.int32, device="cuda")
        st["confidence"] = torch.empty(T, device="cuda")
        st["lse"] = torch.empty(T, device="cuda")
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    if case["op"] in ("rules", "pick"):
        return _prepare_rules(case, g)
    B, n, H, D = case["batch"], case["new"], case["heads"], case["dim"]
    T, dt = B * n, DT[case["dtype"]]
    total = _lengths(case)
    st = dict(case=case, cache=_cache(case, g, total), start=_i32(_starts([n] * B)), len=_i32(total), max_len=max(total))
    st["q"] = torch.randn(T, H * D, generator=g, device="cuda").to(dt)
    st["mask"] = None
    if case["masked"]:
        st["mask"] = (torch.rand(B, max(total), generator=g, device="cuda") < 0.9).to(torch.uint8)
        if case["op"] == "window":
            st["mask"][-1] = B == 1             # every cached position of the last sequence is dropped
    if case["op"] == "shared":
        first, shared = _groups(case)
        st["group_start"], st["shared_len"] = _i32(first), _i32(shared)
        st["max_rows"] = max(b - a for a, b in zip(first, first[1:])) * n
        st["max_shared"] = max(shared)
        if st["mask"] is not None:              # a group's sequences agree on what they drop of the prefix
            for p, s in enumerate(shared):
                st["mask"][first[p]:first[p + 1], :s] = st["mask"][first[p], :s].clone()
    st["out"] = torch.empty(T, H * D, dtype=dt, device="cuda")
    st["lse"] = torch.empty(T, H, device="cuda")
    return st


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _plain_attend(st):
    c, cache = st["case"], st["cache"]
    B, n, H, Hkv, D, page = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    G = H // Hkv
    at = cache["table"].long().clamp(min=0)
    P = at.shape[1]
    there = (cache["table"] >= 0)[..., None]
    value = lambda codes, scales: ((codes[at].float() - 128.0) * torch.where(there, scales[at], 0.0)[..., None, None]) \
        .permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * page, D)
    q = st["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    s = (q @ value(cache["K"], cache["k_scale"]).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    j = torch.arange(P * page, device="cuda")
    length = st["len"].long()
    seen = (j[None, :] < length[:, None])[:, None, :].expand(B, n, -1)
    own_slot = length[:, None] - n + torch.arange(n, device="cuda")[None, :]
    if c["causal"]:
        seen = seen & (j[None, None, :] <= own_slot[:, :, None])
    if c["op"] == "window":
        seen = seen & ((j[None, None, :] > own_slot[:, :, None] - c["window"]) | (j < c["sinks"])[None, None, :])
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


def _plain_logits(st):
    """Logits in 32 bits after the penalties and biases, and which tokens may be taken: [T][V] both."""
    c = st["case"]
    B, n, V = c["batch"], c["new"], c["vocab"]
    x = st["x"].float()
    written = torch.arange(st["history"].shape[1], device="cuda")[None, :] < st["history_len"][:, None]
    count = torch.zeros(B, V, device="cuda").scatter_add_(1, st["history"].long(), written.float())
    count = count.repeat_interleave(n, 0)
    _, repetition, presence, frequency = (t[:, None] for t in st["params"].repeat_interleave(n, 0).unbind(1))
    scaled = torch.where(x > 0, x / repetition, x * repetition)
    x = torch.where(count > 0, scaled - (frequency * count + presence), x)
    if st["bias_ids"] is not None:
        k = torch.arange(c["biases"], device="cuda")[None, :]
        given = torch.where(k < st["bias_len"][:, None], k, -1)
        last = torch.full((B, V), -1, dtype=torch.long, device="cuda")
        last.scatter_reduce_(1, st["bias_ids"].long(), given, "amax")
        bias = torch.where(last >= 0, st["bias_values"].gather(1, last.clamp(min=0)), 0.0)
        x = x + bias.repeat_interleave(n, 0)
    if st["allowed"] is None:
        return x, torch.ones_like(x, dtype=torch.bool)
    v = torch.arange(V, device="cuda")
    allowed = (st["allowed"][:, v // 32] >> (v % 32)[None, :] & 1) != 0
    return x, allowed if c["by_row"] else allowed.repeat_interleave(n, 0)


def _plain_rules(st):
    x, allowed = _plain_logits(st)
    x = x * (1.0 / st["params"][:, 0]).repeat_interleave(st["case"]["new"])[:, None]
    return torch.where(allowed, x, -math.inf).to(st["x"].dtype)


def _plain_pick(st):
    c = st["case"]
    z, allowed = _plain_logits(st)
    z = torch.where(allowed, z, -math.inf)
    some = allowed.any(-1)
    best = z.amax(-1, keepdim=True)
    v = torch.arange(c["vocab"], device="cuda")
    token = torch.where((z == best) & allowed, v, c["vocab"]).amin(-1)
    warm = (1.0 / st["params"][:, 0]).repeat_interleave(c["new"])[:, None]
    d = torch.where(allowed, (z - torch.where(some[:, None], best, 0.0)) * warm, -math.inf)
    p = torch.exp(d)
    total = p.sum(-1)
    lse = best[:, 0] * warm[:, 0] + torch.log(total)
    if c["kind"] == "probability":
        confidence = 1.0 / total
    elif c["kind"] == "margin":
        second = torch.where(v[None, :] == token[:, None], -math.inf, d).amax(-1)
        confidence = (1.0 - torch.exp(second)) / total
    else:
        confidence = torch.where(allowed, p * d, 0.0).nan_to_num(nan=0.0).sum(-1) / total - torch.log(total)
    return {"token": torch.where(some, token, -1).to(torch.int32), "confidence": torch.where(some, confidence, 0.0),
            "lse": torch.where(some, lse, -math.inf)}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2606_04945_gb300 import abi

    c = st["case"]
    if c["op"] in ("rules", "pick"):
        rules = abi.LogitsRules(c["vocab"], params=st["params"], history=st["history"], history_len=st["history_len"],
                                bias_ids=st["bias_ids"], bias_values=st["bias_values"], bias_len=st["bias_len"],
                                allowed=st["allowed"], allowed_by_row=c["by_row"])
        if c["op"] == "rules":
            abi.logits_apply_rules(st["x"], st["start"], rules, max_new=c["new"], Y=st["y"])
            return st["y"]
        abi.logits_pick(st["x"], st["start"], rules, st["token"], st["confidence"], max_new=c["new"], kind=c["kind"],
                        lse=st["lse"])
        return {"token": st["token"], "confidence": st["confidence"], "lse": st["lse"]}
    t = st["cache"]
    cache = abi.KVCache(t["K"], t["V"], t["k_scale"], t["v_scale"])
    if c["op"] == "window":
        abi.kv_cache_attention_window(st["q"], cache, t["table"], st["len"], st["start"], st["out"], max_new=c["new"],
                                      max_len=st["max_len"], window=c["window"], sinks=c["sinks"], causal=c["causal"],
                                      key_mask=st["mask"], lse=st["lse"])
    else:
        abi.kv_cache_attention_shared(st["q"], cache, t["table"], st["len"], st["start"], st["out"], max_new=c["new"],
                                      max_len=st["max_len"], group_start=st["group_start"], shared_len=st["shared_len"],
                                      max_rows=st["max_rows"], max_shared=st["max_shared"], causal=c["causal"],
                                      key_mask=st["mask"], lse=st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


PLAIN = {"window": _plain_attend, "shared": _plain_attend, "rules": _plain_rules, "pick": _plain_pick}


def run(st):
    return _own(st) if own else PLAIN[st["case"]["op"]](st)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_logits(st, b):
    """One sequence's logits [new][V] after penalties and biases, before the temperature, and its masks."""
    c = st["case"]
    n, V = c["new"], c["vocab"]
    x = st["x"][b * n:(b + 1) * n].double()
    _, repetition, presence, frequency = st["params"][b].double().tolist()
    tokens = st["history"][b, :int(st["history_len"][b])].long()
    seen, times = torch.unique(tokens, return_counts=True)
    if seen.numel():
        y = x[:, seen]
        x[:, seen] = torch.where(y > 0, y / repetition, y * repetition) - presence - frequency * times.double()
    if st["bias_ids"] is not None:
        entries = int(st["bias_len"][b])
        values = dict(zip(st["bias_ids"][b, :entries].tolist(), st["bias_values"][b, :entries].double().tolist()))
        if values:
            x[:, torch.tensor(list(values), device="cuda")] += torch.tensor(list(values.values()), dtype=torch.float64,
                                                                             device="cuda")
    ok = torch.ones(n, V, dtype=torch.bool, device="cuda")
    if st["allowed"] is not None:
        rows = st["allowed"][b * n:(b + 1) * n] if c["by_row"] else st["allowed"][b:b + 1]
        words = rows.long() % 2 ** 32
        bits = torch.stack([words // 2 ** k % 2 for k in range(32)], -1).flatten(1)[:, :V]
        ok &= bits == 1
    return x, ok


def _exact_tokens(case, st):
    out, token, confidence, lses = [], [], [], []
    for b in range(case["batch"]):
        x, ok = _exact_logits(st, b)
        t = float(st["params"][b, 0])
        y = (x / t).masked_fill(~ok, -math.inf)
        if case["op"] == "rules":
            out.append(y)
            continue
        some = ok.any(-1)
        z = x.masked_fill(~ok, -math.inf)
        top2 = torch.sort(z, dim=-1, descending=True, stable=True)
        token.append(torch.where(some, top2.indices[:, 0], -1))
        lse = torch.logsumexp(y, -1)
        p = torch.where(ok, torch.exp(y - lse.nan_to_num(neginf=0.0)[:, None]), 0.0)
        if case["kind"] == "probability":
            conf = p.gather(1, top2.indices[:, :1])[:, 0]
        elif case["kind"] == "margin":
            conf = p.gather(1, top2.indices[:, :1])[:, 0]
            if case["vocab"] > 1:
                conf = conf - p.gather(1, top2.indices[:, 1:2])[:, 0]
        else:
            conf = torch.special.xlogy(p, p).sum(-1)
        confidence.append(torch.where(some, conf, 0.0))
        lses.append(lse)
    if case["op"] == "rules":
        return torch.cat(out)
    return {"token": torch.cat(token).to(torch.int32), "confidence": torch.cat(confidence), "lse": torch.cat(lses)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("rules", "pick"):
        return _exact_tokens(case, st)
    B, n, H, Hkv, D, page = (case[k] for k in ("batch", "new", "heads", "kv_heads", "dim", "page"))
    total, cache, G = _lengths(case), st["cache"], H // Hkv
    pages = cache["table"].cpu()
    out = torch.zeros(B * n, H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B * n, H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        L = total[b]
        slot = torch.arange(L, device="cuda")
        mine = torch.arange(L - n, L, device="cuda")
        hidden = torch.zeros(n, L, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= slot[None, :] > mine[:, None]
        if case["op"] == "window":
            far = mine[:, None] - slot[None, :] >= case["window"]
            far[:, :case["sinks"]] = False
            hidden |= far
        if st["mask"] is not None:
            hidden |= st["mask"][b, :L] == 0
        # keys that some row of the sequence sees
        met = torch.nonzero(~hidden.all(0))[:, 0]
        if not met.numel():
            continue
        hidden = hidden[:, met]
        p, at = pages[b][(met // page).cpu()].long().cuda(), met % page
        for h in range(Hkv):
            k = (cache["K"][p, h, at].double() - 128) * cache["k_scale"][p, h].double()[:, None]
            v = (cache["V"][p, h, at].double() - 128) * cache["v_scale"][p, h].double()[:, None]
            q = st["q"][b * n:(b + 1) * n, h * G * D:(h + 1) * G * D].double().reshape(n, G, D)
            s = torch.einsum("ngd,ld->ngl", q, k) / math.sqrt(D)
            s.masked_fill_(hidden[:, None, :], -math.inf)
            row = torch.logsumexp(s, dim=-1)
            w = torch.exp(s - row.nan_to_num(neginf=0.0)[..., None])
            out[b * n:(b + 1) * n, h * G:(h + 1) * G] = torch.einsum("ngl,ld->ngd", w, v)
            lse[b * n:(b + 1) * n, h * G:(h + 1) * G] = row
    return {"out": out.reshape(-1, H * D), "lse": lse}
