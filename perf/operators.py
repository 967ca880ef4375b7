"""Workloads of the operators between the qkv and the o projection of a layer: head norms with rotary positions,
the 8-bit paged cache, attention over it, and cross attention to an encoder's states.

``listed()`` and ``draw()`` describe cases, ``prepare()`` makes what a program holds before the call, ``run()`` makes one
call -- of the library where ``own`` is true, of the same formula in elementary torch operations where it is not --
and ``exact()`` evaluates the definition in 64 bits.

The cache holds int8 codes, k as [pages, heads, page, head_dim], v as [pages, heads, head_dim, page], and one scale for
each page and head.  What a code stands for is code * scale.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FLT_MIN = 2.0 ** -126


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # one denoising step of the action expert: 50 tokens, width 1024 in 16 heads; latency counts
        dict(name="rope_expert_step", op="rope", tokens=50, q_heads=16, k_heads=16, head_dim=64, rotary=64, layout="half", norm=True, dtype="bf16", context=1024),
        # the backbone's prefix (816 tokens, hidden 2048, one kv head of 256) of sixteen robots
        dict(name="rope_prefix_batch", op="rope", tokens=13056, q_heads=8, k_heads=1, head_dim=256, rotary=256, layout="half", norm=True, dtype="bf16", context=816),
        # a long batch in binary32: interleaved pairs, half of the head rotated, far positions
        dict(name="rope_long_f32", op="rope", tokens=16383, q_heads=16, k_heads=4, head_dim=128, rotary=64, layout="interleaved", norm=True, dtype="f32", context=131072),
        # one new token for each of 32 sequences
        dict(name="append_tokens", op="append", batch=32, longest=4096, new_most=1, heads=4, head_dim=128, page=64, dtype="bf16"),
        # the backbone's prefix of 64 robots written into fresh pages
        dict(name="append_prefix", op="append", batch=64, longest=0, new_most=816, heads=1, head_dim=256, page=64, dtype="bf16", even=True),
        # ragged chunks in binary32 behind what the pages hold, short pages
        dict(name="append_ragged_f32", op="append", batch=19, longest=700, new_most=901, heads=5, head_dim=96, page=16, dtype="f32"),
        # one token of one robot over its prefix and chunk; latency counts
        dict(name="cache_token", op="cache", batch=1, shortest=866, longest=866, queries=1, q_heads=8, kv_heads=1, head_dim=256, page=64, causal=True, dtype="bf16"),
        # single tokens of a ragged batch over long caches
        dict(name="cache_tokens_ragged", op="cache", batch=48, shortest=1, longest=16384, queries=1, q_heads=32, kv_heads=8, head_dim=128, page=64, causal=True, dtype="bf16"),
        # the action expert's 50 tokens over the prefix and themselves, both directions, 32 robots
        dict(name="cache_expert_chunk", op="cache", batch=32, shortest=866, longest=866, queries=50, q_heads=8, kv_heads=1, head_dim=256, page=64, causal=False, dtype="bf16"),
        # ragged chunks of a long prompt over what is cached before them
        dict(name="cache_prefill", op="cache", batch=3, shortest=5000, longest=8192, queries=4096, q_heads=16, kv_heads=4, head_dim=128, page=32, causal=True, dtype="bf16"),
        # the action expert's tokens to the encoder's 816 states, a part of them masked
        dict(name="cross_expert", op="cross", batch=1, queries=50, keys=816, q_heads=16, kv_heads=16, head_dim=64, mask=True, dtype="bf16"),
        # the same for a batch of long sequences of another length
        dict(name="cross_batch", op="cross", batch=16, queries=1023, keys=4100, q_heads=16, kv_heads=16, head_dim=64, mask=False, dtype="bf16"),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "cache", "cache", "cross"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "rope":
        head_dim = rng.choice([64, 80, 96, 128, 256])
        k_heads = rng.choice([1, 2, 4, 8])
        q_heads = k_heads * rng.randint(1, 4)
        tokens = _log(rng, 1, max(1, 16384 * 2560 // ((q_heads + k_heads) * head_dim)))
        rotary = rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(1, head_dim // 2)])
        return dict(op=op, tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=head_dim, rotary=rotary, layout=rng.choice(["half", "interleaved"]), norm=rng.random() < 0.8, dtype=dtype, context=_log(rng, 1024, 1 << 20))
    if op == "append":
        heads, head_dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 80, 128, 256])
        batch = _log(rng, 1, 64)
        most = max(1, min(4096, 52224 * 256 // (batch * heads * head_dim)))
        return dict(op=op, batch=batch, longest=rng.choice([0, _log(rng, 1, 4096)]), new_most=rng.choice([1, _log(rng, 1, most)]), heads=heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]), dtype=dtype)
    head_dim = rng.choice([64, 80, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
    if op == "cache":
        queries = rng.choice([1, 1, _log(rng, 2, 1024)])
        longest = _log(rng, max(queries, 16), 16384)
        # bounds: the bytes of the cache, and the products of queries and keys (fewer of them in binary32)
        pairs = (1 << 33) if dtype == "bf16" else (1 << 28)
        batch = _log(rng, 1, max(1, min(64, (1 << 28) // (longest * kv_heads * head_dim), pairs // (queries * longest * q_heads))))
        return dict(op=op, batch=batch, shortest=rng.randint(0, longest), longest=longest, queries=queries, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]), causal=rng.random() < 0.6, dtype=dtype)
    queries, keys = rng.choice([1, _log(rng, 2, 2048)]), _log(rng, 1, 8192)
    pairs = (1 << 31) if dtype == "bf16" else (1 << 28)
    batch = _log(rng, 1, max(1, min(64, (1 << 27) // (keys * kv_heads * head_dim), pairs // (queries * keys * q_heads))))
    return dict(op=op, batch=batch, queries=queries, keys=keys, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, mask=rng.random() < 0.5, dtype=dtype)


# ---------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _lengths(seed, batch, low, high):
    import random
    rng = random.Random(seed)
    out = [rng.randint(low, high) for _ in range(batch)]
    out[rng.randrange(batch)] = high
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _pages(g, lengths, longest, heads, page, head_dim):
    """A cache that holds `lengths` tokens of each sequence in pages of a random order, with room for `longest` of each."""
    counts = [-(-n // page) for n in lengths]
    need = max(1, len(lengths) * -(-longest // page))
    x = torch.randn(need, heads, page, head_dim, device="cuda", generator=g)
    x[..., ::17] *= 4.0                                   # channels of a larger amplitude
    scale_k = x.abs().amax((2, 3)) / 127.0
    k = torch.round(x / scale_k[..., None, None]).to(torch.int8)
    x = torch.randn(need, heads, head_dim, page, device="cuda", generator=g)
    scale_v = x.abs().amax((2, 3)) / 127.0
    v = torch.round(x / scale_v[..., None, None]).to(torch.int8)
    order = torch.randperm(need, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros(len(lengths), max(1, max(counts)), dtype=torch.int32, device="cuda")
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return k, v, scale_k, scale_v, table


def _plan(table, held, new, page):
    """The pages that new tokens go to, with the first and the end of the places they take there, and each token's place."""
    which, first, end, block, offset = [], [], [], [], []
    for b, (h, n) in enumerate(zip(held, new)):
        for i in range(h // page, (h + n - 1) // page + 1):
            lo, hi = max(h, i * page), min(h + n, (i + 1) * page)
            block += [len(which)] * (hi - lo)
            offset += range(lo - i * page, hi - i * page)
            which.append((b, i))
            first.append(lo - i * page)
            end.append(hi - i * page)
    where = torch.tensor(which, device="cuda")
    rest = [torch.tensor(x, device="cuda") for x in (first, end, block, offset)]
    return [table[where[:, 0], where[:, 1]].long()] + rest


def _frequencies(case):
    """Per pair, in radians a position: base 10000, those that turn less than once within 8192 positions slowed by 8,
    those that turn more than 4 times kept, a ramp between."""
    r = case["rotary"]
    f = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if case["context"] > 8192:
        turns = f * 8192 / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f * keep + f / 8.0 * (1.0 - keep)
    return f.cuda()


def prepare(case, seed):
    g = _generator(seed)
    t = DTYPES[case["dtype"]]
    s = dict(case=case)
    if case["op"] == "rope":
        M, D, hq, hk = case["tokens"], case["head_dim"], case["q_heads"], case["k_heads"]
        # q, k and v next to each other, as the fused projection writes them
        s["qkv"] = (torch.randn(M, (hq + 2 * hk) * D, device="cuda", generator=g) * 1.5).to(t)
        s["positions"] = torch.randint(0, case["context"], (M,), device="cuda", generator=g, dtype=torch.int32)
        s["frequencies"] = _frequencies(case)
        s["q_gain"] = 1.0 + 0.2 * torch.randn(D, device="cuda", generator=g) if case["norm"] else None
        s["k_gain"] = 1.0 + 0.2 * torch.randn(D, device="cuda", generator=g) if case["norm"] else None
    elif case["op"] == "append":
        B, H, D, P = case["batch"], case["heads"], case["head_dim"], case["page"]
        new = [case["new_most"]] * B if case.get("even") else _lengths(seed + 1, B, 1, case["new_most"])
        held = _lengths(seed + 2, B, 0, case["longest"])
        most_held = case["longest"] + case["new_most"]
        k, v, sk, sv, table = _pages(g, [a + b for a, b in zip(held, new)], most_held, H, P, D)
        T = sum(new)
        kv = torch.randn(T, 2 * H * D, device="cuda", generator=g) * 1.3
        kv[:, :H * D:17] *= 4.0
        kv = kv.to(t)
        s.update(k=kv[:, :H * D], v=kv[:, H * D:], held=held, new=new, offsets=_ints(_offsets(new)), lengths=_ints(held), most=max(new))
        s.update(ck=k, cv=v, sk=sk, sv=sv, table=table, plan=_plan(table, held, new, P))
    elif case["op"] == "cache":
        B, hq, hk, D, P = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
        held = _lengths(seed + 1, B, case["shortest"], case["longest"])
        queries = [case["queries"]] * B
        k, v, sk, sv, table = _pages(g, held, case["longest"], hk, P, D)
        s.update(q=(torch.randn(sum(queries), hq * D, device="cuda", generator=g) * 1.5).to(t), held=held, queries=queries,
                 offsets=_ints(_offsets(queries)), lengths=_ints(held), ck=k, cv=v, sk=sk, sv=sv, table=table)
    else:
        B, hq, hk, D = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
        s["q"] = (torch.randn(B * case["queries"], hq * D, device="cuda", generator=g) * 1.5).to(t)
        # keys and values next to each other, as a fused projection of the encoder's states writes them
        kv = torch.randn(B * case["keys"], 2 * hk * D, device="cuda", generator=g).to(t)
        s["k"], s["v"] = kv[:, :hk * D], kv[:, hk * D:]
        s["mask"] = None
        if case["mask"]:                                  # a run of states left out (an absent camera) and a few single ones
            m = torch.rand(B, case["keys"], device="cuda", generator=g) > 0.02
            m[:, case["keys"] // 3:2 * case["keys"] // 3] = False
            s["mask"] = m
    if own:
        from paper_2609_24433_b200 import fq
        if "ck" in s:
            s["cache"] = fq.KV8Cache(s["ck"], s["cv"], s["sk"], s["sv"])
    return s


# ---------------------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2609_24433_b200 import fq
    c = s["case"]
    if c["op"] == "rope":
        q, k = fq.qk_norm_rope(s["qkv"], c["q_heads"], c["k_heads"], c["head_dim"], s["positions"], s["frequencies"], q_gain=s["q_gain"], k_gain=s["k_gain"],
                               eps=1e-6, layout=fq.ROPE_HALF if c["layout"] == "half" else fq.ROPE_INTERLEAVED)
        return dict(q=q, k=k)
    if c["op"] == "append":
        fq.kv8_append(s["k"], s["v"], s["cache"], s["table"], s["lengths"], s["offsets"], max_new=s["most"])
        return dict(k=s["ck"], v=s["cv"], k_scale=s["sk"], v_scale=s["sv"])
    if c["op"] == "cache":
        return fq.attention_kv8(s["q"], c["q_heads"], s["cache"], s["table"], s["lengths"], s["offsets"], max_q=c["queries"], causal=c["causal"])
    return fq.cross_attention(s["q"], s["k"], s["v"], c["q_heads"], c["kv_heads"], c["batch"], key_mask=s["mask"])


def _run_plain(s):
    return {"rope": _plain_rope, "append": _plain_append, "cache": _plain_cache, "cross": _plain_cross}[s["case"]["op"]](s)


def _plain_rope(s):
    c = s["case"]
    M, D, hq, hk, r = c["tokens"], c["head_dim"], c["q_heads"], c["k_heads"], c["rotary"]
    angle = torch.remainder(s["positions"].double()[:, None] * s["frequencies"], 2 * math.pi)
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]

    def one(x, gain):
        x = x.float()
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
        if c["layout"] == "half":
            a, b = x[..., :r // 2], x[..., r // 2:r]
        else:
            a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -2 if c["layout"] == "half" else -1).flatten(-2)
        return torch.cat([turned, x[..., r:]], -1).to(s["qkv"].dtype).view(M, -1)

    heads = s["qkv"].view(M, -1, D)
    return dict(q=one(heads[:, :hq], s["q_gain"]), k=one(heads[:, hq:hq + hk], s["k_gain"]))


def _plain_append(s):
    c = s["case"]
    H, D, P = c["heads"], c["head_dim"], c["page"]
    page, first, end, block, offset = s["plan"]           # of each page that tokens go to; of each token
    slot = torch.arange(P, device="cuda")[None]
    fresh = ((slot >= first[:, None]) & (slot < end[:, None]))[:, None, :, None]
    held = (slot < first[:, None])[:, None, :, None]
    for x, codes, scales, last in ((s["k"], s["ck"], s["sk"], False), (s["v"], s["cv"], s["sv"], True)):
        new = torch.zeros(len(page), P, H, D, device="cuda")
        new[block, offset] = x.float().view(-1, H, D)
        new = new.transpose(1, 2)                         # [pages, heads, page, head_dim]
        most = new.abs().amax((2, 3))
        cand = most / 127.0
        cand = torch.where(cand < FLT_MIN, torch.zeros_like(cand), cand)
        was = torch.where(first[:, None] > 0, scales[page], torch.zeros_like(cand))
        now = torch.maximum(was, cand)
        # quotients in 64 bits: values next to a border between two codes
        sets = (cand >= was)[:, :, None, None]
        wide = lambda t: t.double()[:, :, None, None]
        quotient = torch.where(sets, new.double() * 127.0, new.double()) / torch.where(sets, wide(most), wide(was))
        filled = torch.where(wide(now) > 0, torch.round(quotient), torch.zeros_like(quotient)).to(torch.int8)
        old = codes[page]
        old = old.transpose(2, 3) if last else old
        kept = torch.where((now > was)[:, :, None, None], torch.round(old.double() * wide(was) / wide(now)).to(torch.int8), old)
        out = torch.where(fresh, filled, torch.where(held, kept, old))
        codes[page] = out.transpose(2, 3) if last else out
        scales[page] = now
    return dict(k=s["ck"], v=s["cv"], k_scale=s["sk"], v_scale=s["sv"])


def _held(codes, scales, pages, n, tokens_last):
    x = codes.index_select(0, pages).float() * scales.index_select(0, pages)[..., None, None]
    if tokens_last:
        x = x.transpose(2, 3)
    return x.transpose(0, 1).flatten(1, 2)[:, :n]          # [heads, n, head_dim]


def _softmax_sum(q, k, v, seen):
    """q [Hq, T, D], k and v [Hk, L, D] in 32 bits, seen [T or 1, L] or None -> [Hq, T, D]; a row that sees nothing gives zeros."""
    hq, T, D = q.shape
    hk, L = k.shape[0], k.shape[1]
    if L == 0:
        return torch.zeros_like(q)
    a = torch.matmul(q.view(hk, -1, D), k.transpose(1, 2)).view(hq, T, L) * (1.0 / math.sqrt(D))
    if seen is not None:
        a = a.masked_fill(~seen, -math.inf)
    top = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(hk, -1, L), v).view(hq, T, D)
    return torch.where(total > 0, out / total, torch.zeros_like(out))


def _plain_cache(s):
    c = s["case"]
    hq, D, P = c["q_heads"], c["head_dim"], c["page"]
    out, at = torch.empty_like(s["q"]), 0
    for b, (n, T) in enumerate(zip(s["held"], s["queries"])):
        pages = s["table"][b, :-(-n // P)].long()
        k, v = _held(s["ck"], s["sk"], pages, n, False), _held(s["cv"], s["sv"], pages, n, True)
        for t0 in range(0, T, 1024):
            t1 = min(T, t0 + 1024)
            q = s["q"][at + t0:at + t1].float().view(t1 - t0, hq, D).transpose(0, 1)
            seen = None
            if c["causal"]:
                last = torch.arange(t0, t1, device="cuda")[:, None] + (n - T)
                seen = torch.arange(n, device="cuda")[None] <= last
            o = _softmax_sum(q.contiguous(), k, v, seen)
            out[at + t0:at + t1] = o.transpose(0, 1).reshape(t1 - t0, hq * D).to(out.dtype)
        at += T
    return out


def _plain_cross(s):
    c = s["case"]
    hq, hk, D, T, L = c["q_heads"], c["kv_heads"], c["head_dim"], c["queries"], c["keys"]
    out = torch.empty_like(s["q"])
    for b in range(c["batch"]):
        k = s["k"][b * L:(b + 1) * L].float().view(L, hk, D).transpose(0, 1)
        v = s["v"][b * L:(b + 1) * L].float().view(L, hk, D).transpose(0, 1)
        q = s["q"][b * T:(b + 1) * T].float().view(T, hq, D).transpose(0, 1).contiguous()
        o = _softmax_sum(q, k, v, None if s["mask"] is None else s["mask"][b][None])
        out[b * T:(b + 1) * T] = o.transpose(0, 1).reshape(T, hq * D).to(out.dtype)
    return out


# ---------------------------------------------------------------------------- what a pass cannot do without
def _pairs(held, T, causal):
    if not causal:
        return held * T
    first = held - T + 1                                  # keys that the first query sees
    if first >= 1:
        return T * (first + held) // 2
    return held * (held + 1) // 2


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rope":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        return dict(bytes=2 * e * n + 4 * case["tokens"] + 4 * case["rotary"] + 8 * case["head_dim"], flops=7 * n)
    if case["op"] == "append":
        # (the mean of the drawn lengths: what a seed draws lies around it)
        T = case["batch"] * (case["new_most"] if case.get("even") else (1 + case["new_most"]) / 2)
        n = 2 * T * case["heads"] * case["head_dim"]
        return dict(bytes=(e + 1) * n + 8 * case["heads"] * (T / case["page"] + case["batch"]), flops=4 * n)
    D, hq, hk = case["head_dim"], case["q_heads"], case["kv_heads"]
    if case["op"] == "cache":
        L = (case["shortest"] + case["longest"]) / 2
        T, B = case["queries"], case["batch"]
        if case["causal"]:
            pairs = B * T * (2 * L - T + 1) / 2 if L >= T else B * L * (L + 1) / 2
        else:
            pairs = B * T * L
        return dict(bytes=2 * e * B * T * hq * D + B * L * hk * 2 * (D + 4 / case["page"]), flops=4 * D * hq * pairs)
    T, L, B = case["queries"], case["keys"], case["batch"]
    seen = L * 0.65 if case["mask"] else L
    return dict(bytes=2 * e * B * T * hq * D + 2 * e * B * seen * hk * D + (B * L if case["mask"] else 0), flops=4 * D * hq * B * T * seen)


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    if case["op"] == "append":
        return _exact_append(case, s)
    if case["op"] == "cache":
        P, out, at = case["page"], [], 0
        for b, n in enumerate(s["held"]):
            T = s["queries"][b]
            dense = []
            for codes, scales, perm in ((s["ck"], s["sk"], (1, 0, 2, 3)), (s["cv"], s["sv"], (1, 0, 3, 2))):
                idx = s["table"][b, :(n + P - 1) // P].long()
                x = codes[idx].double() * scales[idx].double().unsqueeze(-1).unsqueeze(-1)
                dense.append(x.permute(*perm).reshape(case["kv_heads"], -1, case["head_dim"])[:, :n])
            limit = torch.arange(n - T, n, device="cuda") if case["causal"] else torch.full((T,), n - 1, device="cuda")
            out.append(_exact_rows(s["q"][at:at + T].double().view(T, case["q_heads"], -1), dense[0], dense[1], limit, None))
            at += T
        return torch.cat(out)
    out = []
    T, L = case["queries"], case["keys"]
    for b in range(case["batch"]):
        k, v = (s[x][b * L:(b + 1) * L].double().reshape(L, case["kv_heads"], -1).permute(1, 0, 2) for x in "kv")
        out.append(_exact_rows(s["q"][b * T:(b + 1) * T].double().view(T, case["q_heads"], -1), k, v, torch.full((T,), L - 1, device="cuda"), None if s["mask"] is None else s["mask"][b]))
    return torch.cat(out)


def _exact_rows(q, k, v, limit, mask):
    """Softmax-weighted sums by their definition, head by head; query i sees keys 0 .. limit[i] that the mask leaves."""
    T, hq, D = q.shape
    hk, L, _ = k.shape
    out = torch.zeros(T, hq, D, dtype=torch.float64, device="cuda")
    if L == 0:
        return out.view(T, hq * D)
    index = torch.arange(L, device="cuda")
    for h in range(hq):
        kh, vh = k[h // (hq // hk)], v[h // (hq // hk)]
        for t in range(0, T, 512):
            see = index[None, :] <= limit[t:t + 512, None]
            if mask is not None:
                see = see & mask[None, :]
            w = torch.where(see, torch.einsum("td,ld->tl", q[t:t + 512, h], kh) / D ** 0.5, -1e300)
            w = torch.where(see, (w - w.max(1, keepdim=True).values).exp(), 0.0)
            out[t:t + 512, h] = torch.einsum("tl,ld->td", w, vh) / w.sum(1, keepdim=True).clamp_min(1e-300)
    return out.view(T, hq * D)


def _exact_rope(case, s):
    M, D, r = case["tokens"], case["head_dim"], case["rotary"]
    x = s["qkv"].double().view(M, -1, D)[:, :case["q_heads"] + case["k_heads"]].clone()
    if case["norm"]:
        x /= ((x ** 2).sum(-1, keepdim=True) / D + 1e-6).sqrt()
        x[:, :case["q_heads"]] *= s["q_gain"].double()
        x[:, case["q_heads"]:] *= s["k_gain"].double()
    turn = torch.exp(1j * (s["positions"].double()[:, None, None] * s["frequencies"]))
    first = torch.arange(r // 2, device="cuda") * (1 if case["layout"] == "half" else 2)
    second = first + (r // 2 if case["layout"] == "half" else 1)
    z = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return dict(q=x[:, :case["q_heads"]].reshape(M, -1), k=x[:, case["q_heads"]:].reshape(M, -1))


def _exact_append(case, s):
    H, D, P = case["heads"], case["head_dim"], case["page"]
    table = s["table"].tolist()
    out = {}
    for name, x, codes, scales in (("k", s["k"], s["ck"], s["sk"]), ("v", s["v"], s["cv"], s["sv"])):
        tokens_first = codes.clone() if name == "k" else codes.transpose(2, 3).clone()
        held_scale = scales.double().clone()
        row = 0
        for b in range(case["batch"]):
            start, end = s["held"][b], s["held"][b] + s["new"][b]
            for i in range(start // P, (end - 1) // P + 1):
                lo, hi = max(start, i * P), min(end, (i + 1) * P)
                page, a, z = table[b][i], lo - i * P, hi - i * P
                new = x[row:row + hi - lo].double().view(hi - lo, H, D).permute(1, 0, 2)
                row += hi - lo
                peak = new.abs().flatten(1).max(1).values
                step = (peak / 127).float().double()      # the scale is held in 32 bits
                step = torch.where(step < FLT_MIN, 0.0, step)
                before = held_scale[page] if a else torch.zeros(H, dtype=torch.float64, device="cuda")
                after = torch.maximum(before, step)
                grown = (after > before).view(H, 1, 1)
                sets = (step >= before).view(H, 1, 1)
                q = torch.where(sets, new * 127 / peak.view(H, 1, 1), new / before.view(H, 1, 1))
                tokens_first[page, :, a:z] = torch.where(after.view(H, 1, 1) > 0, q.round(), 0.0).to(torch.int8)
                if a:
                    old = tokens_first[page, :, :a].double()
                    tokens_first[page, :, :a] = torch.where(grown, (old * before.view(H, 1, 1) / after.view(H, 1, 1)).round(), old).to(torch.int8)
                held_scale[page] = after
        out[name] = tokens_first if name == "k" else tokens_first.transpose(2, 3).contiguous()
        out[name + "_scale"] = held_scale
    return dict(k=out["k"], v=out["v"], k_scale=out["k_scale"], v_scale=out["v_scale"])
