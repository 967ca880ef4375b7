"""The operators between the projections of a layer against their formulas in 64 bits: head norms with rotary positions, the
8-bit paged cache, attention over it, cross attention.

Bounds (u = 2^-24, the half step of binary32; h = half a step of the output's type: 2^-8 in bf16, u in binary32):
  rope       sum of squares, root, gain, angle, sine, product: at most 32 roundings of u on a pair's |a| + |b|, then h |y|
  append     codes equal (each is the rounding of an exact quotient), scales within u
  attention  a score is off by at most (D + 8) u A, A = scale max_j sum_d |q_d k_jd|, which scales a probability by e^(that);
             numerator and denominator each: 2 ((D + 8) u A) + (L + 16) u; bf16 calls may take the exponential to 2^-18,
             and their rounded probabilities add 2^-8 (bf16) or 2^-11 (binary16) of W = sum_j p_j |v_j|; then h |y|.  A probability beside the largest, 1, may underflow: each
             of L terms loses at most 2^-126 of V = max_j |v_j| -- or, over the cache, where p vs 2^(7-e) goes as one binary16 term
             (binary32 rows, 16 at most: two), a multiple of 2^-24: 2^-25, times a code of at most 127 and 2^(e-7), with the largest value
             127 vs >= 127 2^(e-1): 2^-31 of the largest value of any channel of the head, seen or not.  Two terms keep 2^-22 of p
"""
import math
import os
import random
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2609_24433_b200 import fq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _watchdog_clean(request):
    yield
    if "gpu" in request.keywords and torch.cuda.is_available():
        st, word = fq.device_status()
        assert st == fq.OK, f"device wait watchdog fired: {word:#x}"


def rand(shape, seed, dtype=torch.float32, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) * gain).to(dtype)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def offsets_of(counts):
    return ints([0] + list(np.cumsum(counts)))


# ------------------------------------------------------------------------------------------- rotary positions
def rope_reference(x, heads, D, positions, freq, gain, eps, layout, amplitude):
    """x [M, heads D] -> (values, |a| + |b| of each channel's pair) in 64 bits"""
    M, r = x.shape[0], 2 * freq.numel()
    x = x.double().reshape(M, heads, D)
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    w = positions.double()[:, None, None] * freq
    c, s = amplitude * torch.cos(w), amplitude * torch.sin(w)
    i = torch.arange(r // 2, device=x.device)
    first, second = (i, i + r // 2) if layout == fq.ROPE_HALF else (2 * i, 2 * i + 1)
    y, size = x.clone(), x.abs()
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    size[..., first] = size[..., second] = abs(amplitude) * (a.abs() + b.abs())
    return y.reshape(M, -1), size.reshape(M, -1)


ROPES = [   # M, q heads, k heads, D, rotary, layout, gains, input, output
    (1, 1, 1, 64, 64, fq.ROPE_HALF, True, "bf16", "bf16"),
    (50, 16, 16, 64, 64, fq.ROPE_HALF, True, "bf16", "bf16"),
    (17, 8, 1, 256, 256, fq.ROPE_HALF, True, "bf16", "f32"),
    (33, 3, 2, 128, 64, fq.ROPE_INTERLEAVED, True, "f32", "f32"),
    (700, 5, 3, 80, 80, fq.ROPE_HALF, True, "f32", "bf16"),
    (9, 7, 0, 96, 20, fq.ROPE_HALF, False, "bf16", "bf16"),           # halves that no lane boundary separates
    (9, 0, 7, 8, 2, fq.ROPE_HALF, True, "f32", "f32"),
    (5, 2, 2, 256, 254, fq.ROPE_HALF, True, "bf16", "bf16"),
    (5, 2, 2, 248, 6, fq.ROPE_INTERLEAVED, False, "bf16", "bf16"),
    (5, 2, 2, 64, 0, fq.ROPE_HALF, True, "bf16", "bf16"),             # the norm alone
    (3001, 12, 4, 128, 128, fq.ROPE_HALF, True, "bf16", "bf16"),      # several tokens per CTA, a ragged end
    (2000, 32, 8, 64, 32, fq.ROPE_INTERLEAVED, True, "bf16", "bf16"),
]


@gpu
@pytest.mark.parametrize("M,hq,hk,D,r,layout,norm,xt,yt", ROPES)
def test_qk_norm_rope_against_64_bits(M, hq, hk, D, r, layout, norm, xt, yt):
    qkv = rand((M, (hq + 2 * hk) * D + 8), M + D, TYPES[xt])
    g = random.Random(M)
    positions = ints([g.choice([0, 1, -3, 815, 131071, 2 ** 31 - 1, g.randrange(1 << 20)]) for _ in range(M)])
    freq = fq.rope_frequencies(r, 10000.0)
    qg = 1 + 0.2 * rand(D, 1) if norm else None
    kg = 1 + 0.2 * rand(D, 2) if norm else None
    q, k = fq.qk_norm_rope(qkv, hq, hk, D, positions, freq, qg, kg, 1e-6, layout, 1.25, TYPES[yt])
    assert q.shape == (M, hq * D) and k.shape == (M, hk * D) and q.dtype == k.dtype == TYPES[yt]
    for got, x, heads, gain in ((q, qkv[:, :hq * D], hq, qg), (k, qkv[:, hq * D:(hq + hk) * D], hk, kg)):
        if heads:
            want, size = rope_reference(x, heads, D, positions, freq, gain, 1e-6, layout, 1.25)
            assert ((got.double() - want).abs() <= HALF[TYPES[yt]] * want.abs() + 32 * U * size).all()


@gpu
@pytest.mark.parametrize("D,r", [(64, 64), (96, 20), (256, 256)])
def test_qk_norm_rope_in_place_and_strided(D, r):
    M, hq, hk = 300, 4, 2
    base = rand((M, 8 * D), 5, torch.bfloat16)
    positions, freq, gain = ints(range(M)), fq.rope_frequencies(r), 1 + 0.2 * rand(D, 3)
    want = fq.qk_norm_rope(base, hq, hk, D, positions, freq, gain, gain)
    x = base.clone()
    fq.qk_norm_rope(x, hq, hk, D, positions, freq, gain, gain, q=x[:, :hq * D], k=x[:, hq * D:(hq + hk) * D])
    assert torch.equal(x[:, :hq * D], want[0]) and torch.equal(x[:, hq * D:(hq + hk) * D], want[1])
    assert torch.equal(x[:, (hq + hk) * D:], base[:, (hq + hk) * D:])
    out = torch.full((M, 8 * D), 7.0, dtype=torch.bfloat16, device="cuda")
    fq.qk_norm_rope(base[:, D:], hq, hk, D, positions, freq, q=out[:, 8:8 + hq * D], k=out[:, 16 + hq * D:16 + (hq + hk) * D])
    want, size = rope_reference(base[:, D:(1 + hq) * D], hq, D, positions, freq, None, 0, fq.ROPE_HALF, 1.0)
    assert ((out[:, 8:8 + hq * D].double() - want).abs() <= 2.0 ** -8 * want.abs() + 32 * U * size).all()
    assert (out[:, :8] == 7).all() and (out[:, 8 + hq * D:16 + hq * D] == 7).all() and (out[:, 16 + (hq + hk) * D:] == 7).all()


def test_rope_frequencies_by_their_formulas():
    r, base = 128, 10000.0
    i = np.arange(r // 2)
    plain = base ** (-2.0 * i / r)
    near = lambda t, w: np.allclose(t.numpy(), w, rtol=1e-14, atol=0)
    assert near(fq.rope_frequencies(r, base, device="cpu"), plain)
    assert near(fq.rope_frequencies(r, base, fq.ROPE_LINEAR, 4.0, device="cpu"), plain / 4)
    changed = fq.rope_frequencies(r, base, fq.ROPE_BASE, 4.0, device="cpu").numpy()
    assert changed[0] == 1.0 and math.isclose(changed[-1], plain[-1] / 4, rel_tol=1e-12)
    turns = plain * 8192 / (2 * math.pi)
    keep = np.clip((turns - 1) / 3, 0, 1)
    assert near(fq.rope_frequencies(r, base, fq.ROPE_PARTS, 8.0, 8192, 1.0, 4.0, device="cpu"), plain * keep + plain / 8 * (1 - keep))
    assert fq.rope_frequencies(0, device="cpu").numel() == 0


# ------------------------------------------------------------------------------------------- the cache
class Model:
    """A cache in 64 bits on the host, by the definition."""

    def __init__(self, cache):
        self.k, self.v = cache.k.cpu().numpy().copy(), cache.v.cpu().numpy().transpose(0, 1, 3, 2).copy()
        self.ks, self.vs = cache.k_scale.cpu().numpy().copy(), cache.v_scale.cpu().numpy().copy()
        self.P = cache.page

    def append(self, k, v, table, held, new):
        row = 0
        for b, (h, n) in enumerate(zip(held, new)):
            for i in range(h // self.P, -(-(h + n) // self.P)):
                lo, hi = max(h, i * self.P), min(h + n, (i + 1) * self.P)
                if hi <= lo or i >= table.shape[1] or not 0 <= table[b, i] < len(self.k):
                    continue
                for x, codes, scales in ((k, self.k, self.ks), (v, self.v, self.vs)):
                    self._block(x[row + lo - h:row + hi - h], codes[table[b, i]], scales[table[b, i]], lo - i * self.P)
            row += n

    @staticmethod
    def _block(x, codes, scales, first):
        H, _, D = codes.shape
        x = x.astype(np.float64).reshape(len(x), H, D).transpose(1, 0, 2)
        for h in range(H):
            a = np.abs(x[h]).max()
            c = np.float32(np.float32(a) / np.float32(127))
            c = np.float32(0) if c < np.float32(2.0 ** -126) else c
            s = scales[h] if first else np.float32(0)
            now = max(s, c)
            if now == 0:
                new = np.zeros_like(x[h])
            else:
                new = np.rint(x[h] * 127 / a) if c >= s else np.rint(x[h] / np.float64(s))
            if first and now > s:
                codes[h, :first] = np.rint(codes[h, :first].astype(np.float64) * np.float64(s) / np.float64(now))
            codes[h, first:first + x.shape[1]] = new
            scales[h] = now

    def check(self, cache):
        assert np.array_equal(cache.k_scale.cpu().numpy(), self.ks) and np.array_equal(cache.v_scale.cpu().numpy(), self.vs)
        assert np.array_equal(cache.k.cpu().numpy(), self.k)
        assert np.array_equal(cache.v.cpu().numpy(), self.v.transpose(0, 1, 3, 2))


def filled_cache(pages, heads, D, page, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = fq.KV8Cache.empty(pages, heads, D, page)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(-127, 128, t.shape, device="cuda", generator=g, dtype=torch.int8))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.rand(t.shape, device="cuda", generator=g) * 0.03 + 0.003)
    return cache


def table_of(pages, batch, width, seed):
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    return ints(order[:batch * width]).view(batch, width)


def host(t):
    return t.float().cpu().numpy()


APPENDS = [   # heads, D, page, held, new, input
    (1, 16, 16, [0], [1], "bf16"),
    (4, 128, 64, [0, 63, 64, 100, 127], [1, 1, 1, 1, 1], "bf16"),
    (1, 256, 64, [0, 0, 0], [816, 64, 63], "bf16"),
    (5, 96, 16, [3, 0, 31, 16, 200], [100, 0, 1, 17, 16], "f32"),
    (2, 80, 32, [31, 1, 30, 0], [2, 31, 33, 95], "f32"),
    (3, 64, 128, [5, 127, 128, 129], [7, 130, 1, 255], "bf16"),
]


@gpu
@pytest.mark.parametrize("H,D,P,held,new,dtype", APPENDS)
def test_kv8_append_by_the_definition(H, D, P, held, new, dtype):
    B = len(held)
    width = max(-(-(h + n) // P) for h, n in zip(held, new)) + 1
    cache = filled_cache(B * width + 3, H, D, P, 1)
    table = table_of(cache.pages, B, width, 2)
    T = sum(new)
    kv = rand((T, 2 * H * D), 3, gain=1.5)
    kv[::3] *= 0.05                                     # tokens that do not set the scale
    kv = kv.to(TYPES[dtype])
    k, v = kv[:, :H * D], kv[:, H * D:]
    model = Model(cache)
    model.append(host(k), host(v), table.cpu().numpy(), held, new)
    lens = ints(held)
    fq.kv8_append(k, v, cache, table, lens, offsets_of(new), max_new=max(new))
    model.check(cache)
    assert lens.tolist() == held
    # a hint below the truth changes nothing but the launch; the same tokens again change nothing
    fq.kv8_append(k, v, cache, table, lens, offsets_of(new), max_new=1)
    model.check(cache)


@gpu
def test_kv8_append_ties_zeros_and_tiny_values():
    H, D, P = 1, 16, 16
    cache = filled_cache(4, H, D, P, 9)
    table = ints([[2, 0]])
    x = torch.zeros(20, D, device="cuda")
    x[0, 0], x[0, 1:9] = 127.0, torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, 62.5, 63.5, -126.5])   # exact ties: to even
    x[16:, :] = 0.0                                     # a page of zeros
    x[17, 3] = 1e-42                                    # ... and one below the smallest step
    model = Model(cache)
    model.append(host(x), host(x), table.cpu().numpy(), [0], [20])
    fq.kv8_append(x, x, cache, table, ints([0]))
    model.check(cache)
    assert cache.k[2, 0, 0, :9].tolist() == [127, 0, 2, 2, 0, -2, 62, 64, -126] and cache.k_scale[0, 0] == 0


@gpu
def test_kv8_append_token_by_token():
    H, D, P, B = 2, 64, 16, 3
    cache = filled_cache(12, H, D, P, 4)
    table = table_of(12, B, 3, 4)
    model = Model(cache)
    held = [0, 5, 15]
    for step in range(20):
        kv = rand((B, 2 * H * D), 100 + step, torch.bfloat16, gain=1.0 + 0.3 * step)
        model.append(host(kv[:, :H * D]), host(kv[:, H * D:]), table.cpu().numpy(), held, [1] * B)
        fq.kv8_append(kv[:, :H * D], kv[:, H * D:], cache, table, ints(held))
        held = [h + 1 for h in held]
    model.check(cache)


@gpu
def test_kv8_append_leaves_what_is_not_its_own():
    H, D, P = 2, 32, 16
    cache = filled_cache(6, H, D, P, 5)
    table = ints([[1, -1, 3, 99], [4, 6, 2, 0]])        # no pages: -1, 6 and 99; the third page of sequence 1 is not reached
    before = [t.clone() for t in cache.tensors]
    x = rand((90, H * D), 6)
    held, new = [10, 20], [60, 10]                      # rows 70 .. 89 belong to nobody; 10 + 60 passes four pages
    model = Model(cache)
    model.append(host(x), host(x), table.cpu().numpy(), held, new)
    fq.kv8_append(x, x, cache, table, ints(held), offsets_of(new))
    model.check(cache)
    for t, was in zip(cache.tensors, before):
        for page in (0, 2, 4, 5):
            assert torch.equal(t[page], was[page])
    # offsets that leave the rows, or fall, are cut: nothing is read or written out of range
    fq.kv8_append(x, x, cache, table, ints([0, 0]), ints([80, 500, 10]))
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- attention
def attention_reference(q, k, v, scale, seen):
    """q [T, Hq, D], k, v [L, Hk, D] in 64 bits, seen [T, L] -> (o, A, W, V), each [T, Hq, D] or [T, Hq, 1]"""
    T, Hq, D = q.shape
    L, Hk = k.shape[:2]
    if L == 0:
        z = torch.zeros(T, Hq, D, dtype=torch.float64, device=q.device)
        return z, z[..., :1], z, z
    k, v = (t.repeat_interleave(Hq // Hk, 1) for t in (k, v))
    s = torch.einsum("thd,lhd->htl", q, k) * scale
    size = torch.einsum("thd,lhd->htl", q.abs(), k.abs()) * scale
    s = torch.where(seen[None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.where(seen[None], torch.exp(s - torch.where(top.isinf(), 0.0, top)), 0.0)
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-300)
    A = torch.where(seen[None], size, 0.0).amax(-1)
    return (torch.einsum("htl,lhd->thd", p, v), A.transpose(0, 1)[..., None], torch.einsum("htl,lhd->thd", p, v.abs()),
            v.abs().amax(0)[None])


def assert_attention(got, want, A, W, V, L, rounded, two_terms=False):
    D = want.shape[-1]
    bound = (2 * (2 * (D + 8) * U * A + (L + 16) * U + (2.0 ** -18 if rounded else 0.0)) + rounded) * W + HALF[got.dtype] * want.abs()
    bound = bound + L * 2.0 ** -126 * V + (2.0 ** -22 * W if two_terms else 0.0)
    if rounded == 2.0 ** -11 or two_terms:
        bound = bound + L * 2.0 ** -31 * V.amax(-1, keepdim=True)
    off = (got.double().view_as(want) - want).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), f"{(off / bound.clamp_min(1e-300)).max().item():.3g} of the bound"


def dense(cache, table, b, n):
    """What the codes of a sequence's first n tokens stand for, and which of them lie in pages that there are."""
    P = cache.page
    ids = [table[b, j // P].item() for j in range(n)]
    ok = torch.tensor([0 <= i < cache.pages for i in ids], dtype=torch.bool, device="cuda")
    idx = torch.tensor([max(0, min(i, cache.pages - 1)) for i in ids], dtype=torch.long, device="cuda")
    off = torch.arange(n, device="cuda") % P
    k = cache.k[idx, :, off].double() * cache.k_scale[idx].double()[..., None]
    v = cache.v.transpose(2, 3)[idx, :, off].double() * cache.v_scale[idx].double()[..., None]
    return k, v, ok


def check_cache_attention(cache, table, lens, queries, Hq, dtype, causal, scale=None, seed=0, max_kv=0, two_terms=False, **kw):
    D, rows = cache.head_dim, sum(queries)
    q = rand((rows + 3, Hq * D), seed, TYPES[dtype], gain=1.5)
    y = torch.full((rows + 3, Hq * D), 7.0, dtype=TYPES[dtype], device="cuda")
    got = fq.attention_kv8(q, Hq, cache, table, ints(lens), offsets_of(queries), max_kv=max_kv, causal=causal, scale=scale, y=y, **kw)
    assert got is y and (y[rows:] == 7).all()          # rows that belong to no sequence
    scale = D ** -0.5 if scale is None else scale
    at = 0
    for b, (n, T) in enumerate(zip(lens, queries)):
        n = min(n, table.shape[1] * cache.page, max_kv or n)
        k, v, ok = dense(cache, table, b, n)
        last = torch.arange(T, device="cuda")[:, None] + (n - T if causal else n)
        seen = ok[None] & (torch.arange(n, device="cuda")[None] <= last)
        want, A, W, V = attention_reference(q[at:at + T].double().view(T, Hq, D), k, v, scale, seen)
        assert_attention(y[at:at + T], want, A, W, V, n, 2.0 ** -11 if dtype == "bf16" else 0.0, two_terms)
        empty = ~seen.any(1)
        assert (y[at:at + T][empty] == 0).all()
        at += T


CACHES = [   # q heads, kv heads, D, page, lengths, queries, causal, type
    (1, 1, 16, 16, [1], [1], True, "bf16"),
    (8, 1, 256, 64, [866], [1], True, "bf16"),
    (8, 1, 256, 64, [866, 50, 1], [50, 50, 1], False, "bf16"),
    (8, 2, 128, 64, [0, 1, 63, 64, 65, 1000], [1, 1, 1, 1, 1, 1], True, "bf16"),
    (16, 1, 64, 32, [300, 31, 33], [1, 1, 1], True, "bf16"),
    (24, 1, 64, 16, [300, 31, 33], [1, 1, 1], True, "bf16"),          # more heads in a group than a tile of sixteen
    (4, 4, 128, 16, [700, 40, 0], [33, 50, 4], True, "bf16"),         # queries that see nothing: 50 on 40 keys, 4 on none
    (6, 2, 80, 32, [500, 129], [130, 129], True, "bf16"),
    (5, 1, 112, 128, [257, 1], [7, 2], False, "bf16"),
    (2, 1, 192, 64, [400], [300], True, "bf16"),
    (32, 8, 128, 64, [4100, 17, 2050], [1, 1, 1], True, "bf16"),      # chunks of keys that meet
    (4, 2, 64, 64, [3000, 5], [3, 2], True, "bf16"),
    (8, 1, 256, 64, [866, 3], [1, 1], True, "f32"),
    (4, 2, 128, 16, [700, 40, 0], [33, 50, 4], True, "f32"),
    (6, 2, 80, 32, [2500, 129], [3, 2], False, "f32"),
]


@gpu
@pytest.mark.parametrize("Hq,Hk,D,P,lens,queries,causal,dtype", CACHES)
def test_attention_kv8_against_64_bits(Hq, Hk, D, P, lens, queries, causal, dtype):
    width = max(1, max(-(-n // P) for n in lens)) + 1
    cache = filled_cache(len(lens) * width + 2, Hk, D, P, 11)
    cache.k_scale[0], cache.v_scale[0] = 0.0, 0.0       # a page of zeros
    table = table_of(cache.pages, len(lens), width, 12)
    used = set()
    for b, n in enumerate(lens):
        used |= set(table[b, :-(-n // P)].tolist())
    for page in set(range(cache.pages)) - used:         # what no sequence reaches may hold anything
        cache.k_scale[page], cache.v_scale[page] = math.nan, math.inf
    check_cache_attention(cache, table, lens, queries, Hq, dtype, causal, seed=13)
    check_cache_attention(cache, table, lens, queries, Hq, dtype, causal, scale=0.02, seed=14, max_q=max(queries))


@gpu
@pytest.mark.parametrize("queries", [[1, 1, 1], [40, 2, 70]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_kv8_pages_that_are_none_and_cut_lengths(queries, dtype):
    cache = filled_cache(40, 2, 64, 16, 21)
    table = table_of(40, 3, 12, 22)
    table[0, 3] = -1
    table[1, 0:2] = 40                                  # all of a short sequence's pages
    table[2, 5] = 2 ** 31 - 1
    check_cache_attention(cache, table, [150, 32, 500], queries, 4, dtype, False, seed=23)       # 500 > 12 pages of 16
    check_cache_attention(cache, table, [150, 32, 500], queries, 4, dtype, True, seed=24, max_kv=100)


@gpu
@pytest.mark.parametrize("Hq,Hk,D,P,dtype", [(4, 2, 64, 64, "bf16"), (16, 1, 128, 32, "bf16"), (8, 1, 256, 128, "bf16"), (3, 1, 128, 64, "f32")])
def test_attention_kv8_few_queries_of_many_sequences(Hq, Hk, D, P, dtype):
    """Equal shares of a ragged batch: tiles inside a share, across two, over many; sequences without keys or queries; more
    sequences than a CTA has threads; hints of max_q that are too small."""
    lens = [0, 1, 255, 256, 257, 511, 513, 90] * 37 + [9000, 0, 20]
    queries = [1, 0, 2, 1, 1, 1, 1, 3] * 37 + [1, 0, 1]
    rows = sum(queries)
    cache = filled_cache(400, Hk, D, P, 61)
    gen = torch.Generator().manual_seed(62)
    table = torch.randint(0, 400, (len(lens), -(-9000 // P)), generator=gen).int().cuda()
    check_cache_attention(cache, table, lens, queries, Hq, dtype, True, seed=63, max_q=3)
    check_cache_attention(cache, table, lens, queries, Hq, dtype, True, seed=64, max_q=1)
    q, offsets = rand((rows, Hq * D), 65, TYPES[dtype]), offsets_of(queries)
    one, other = (fq.attention_kv8(q, Hq, cache, table, ints(lens), offsets, max_q=3) for _ in range(2))
    assert torch.equal(one, other)


@gpu
@pytest.mark.parametrize("Hq,D,lens", [(8, 128, [16384]), (8, 256, [16384]), (1, 64, [0, 0, 16384, 0]), (8, 128, [100] * 500)])
def test_attention_kv8_shares_of_one_long_or_many_short_sequences(Hq, D, lens):
    cache = filled_cache(300, 1, D, 64, 66)
    gen = torch.Generator().manual_seed(67)
    table = torch.randint(0, 300, (len(lens), -(-max(lens) // 64)), generator=gen).int().cuda()
    check_cache_attention(cache, table, lens, [1] * len(lens), Hq, "bf16", True, seed=68, max_q=1)


@gpu
@pytest.mark.parametrize("Hq,Hk,D,P,queries", [(2, 1, 16, 16, [300, 70]), (4, 2, 48, 32, [200, 5]), (2, 2, 64, 64, [300, 129]), (4, 1, 128, 64, [300, 40]),
                                               (8, 1, 256, 128, [50, 50])])
def test_attention_kv8_many_queries_of_every_width(Hq, Hk, D, P, queries):
    lens = [2100, 300]
    width = -(-2100 // P)
    cache = filled_cache(2 * width, Hk, D, P, 69)
    table = table_of(2 * width, 2, width, 70)
    table[0, 400 // P] = -1                             # a page that is none
    check_cache_attention(cache, table, lens, queries, Hq, "bf16", True, seed=71, max_q=max(queries))
    check_cache_attention(cache, table, lens, queries, Hq, "bf16", False, seed=72)


@gpu
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("scale", [0.999, 0.51, 1.0, 3e-30])
def test_attention_kv8_rows_that_see_nothing_whatever_the_scales(D, scale):
    """Causal, more queries than keys, of few and of many tiles: the first rows are zeros."""
    cache = filled_cache(64, 2, D, 16, 76)
    cache.v_scale.fill_(scale)
    table = table_of(64, 3, 20, 77)
    check_cache_attention(cache, table, [119, 300, 1], [123, 700, 40], 4, "bf16", True, seed=78)
    check_cache_attention(cache, table, [1, 2, 0], [2, 3, 2], 4, "bf16", True, seed=79, max_q=3)


@gpu
def test_attention_kv8_widens_in_several_passes():
    """More (sequence, head) pairs than the widened codes of one pass hold."""
    cache = filled_cache(60, 4, 256, 128, 73)
    gen = torch.Generator().manual_seed(74)
    table = torch.randint(0, 60, (3, 260), generator=gen).int().cuda()
    lens, queries = [33000, 40, 300], [20, 17, 33]
    assert 12 * 33280 * 256 * 4 > 256 << 20
    check_cache_attention(cache, table, lens, queries, 4, "bf16", True, seed=75, max_q=33)


@gpu
def test_attention_kv8_peaked_scores_and_repeated_pages():
    """Scores far apart (the running maximum rises late, most terms vanish); a prefix page that two sequences share."""
    cache = filled_cache(70, 1, 128, 64, 31)
    table = table_of(70, 2, 33, 32)
    table[1, :10] = table[0, :10]
    cache.k_scale[table[0, 30].item()] *= 30
    check_cache_attention(cache, table, [2100, 700], [1, 1], 8, "bf16", True, scale=1.0, seed=33)
    check_cache_attention(cache, table, [2100, 700], [20, 30], 8, "bf16", True, scale=1.0, seed=34)


@gpu
def test_attention_kv8_peaked_scores_of_binary32_rows():
    """Channels where the value beside the largest probability is next to nothing, so that only small terms are left."""
    for D, Hq, Hk, T in ((64, 3, 1, 2), (128, 12, 3, 1), (192, 8, 1, 2)):
        cache = filled_cache(41, Hk, D, 16, 44)
        table = table_of(41, 2, 20, 45)
        check_cache_attention(cache, table, [27, 300], [T, T], Hq, "f32", True, scale=1.0, seed=46, two_terms=True)


@gpu
def test_attention_kv8_scales_far_apart():
    cache = filled_cache(20, 1, 64, 16, 35)
    cache.v_scale.copy_(10.0 ** torch.linspace(-30, 30, 20, device="cuda")[:, None])
    cache.k_scale.mul_(0.1)
    table = table_of(20, 1, 20, 36)
    for T in (1, 30):
        check_cache_attention(cache, table, [320], [T], 4, "bf16", True, seed=37 + T)
        check_cache_attention(cache, table, [320], [T], 4, "f32", True, seed=38 + T)


@gpu
def test_attention_kv8_queries_of_any_size():
    """A row's largest channel from 1e-30 to 1e30, with the scale that keeps the scores ordinary."""
    cache = filled_cache(8, 1, 64, 64, 41)
    table = table_of(8, 1, 8, 42)
    for T in (1, 40):
        base = rand((T, 4 * 64), 43, torch.bfloat16)
        for size in (2.0 ** -100, 2.0 ** -20, 2.0 ** 20, 2.0 ** 100):
            q, scale = (base.double() * size).to(torch.bfloat16), 0.125 / size
            got = fq.attention_kv8(q, 4, cache, table, ints([500]), causal=False, scale=scale)
            k, v, ok = dense(cache, table, 0, 500)
            want, A, W, V = attention_reference(q.double().view(T, 4, 64), k, v, scale, ok[None].expand(T, -1))
            assert_attention(got, want, A, W, V, 500, 2.0 ** -11)


@gpu
def test_attention_kv8_behind_2_to_the_31_bytes():
    pages = (1 << 31) // (8 * 128 * 64) + 40
    cache = fq.KV8Cache.empty(pages, 8, 128, 64)
    small = filled_cache(40, 8, 128, 64, 51)
    for big, s in zip(cache.tensors, small.tensors):
        big[-40:] = s
    table = table_of(40, 2, 16, 52) + (pages - 40)
    for queries in ([1, 1], [70, 20]):
        check_cache_attention(cache, table, [1000, 90], queries, 16, "bf16", True, seed=53)
    x = rand((3, 8 * 128), 54, torch.bfloat16)
    fq.kv8_append(x, x, cache, table, ints([900, 90]), offsets_of([1, 2]))
    fq.kv8_append(x, x, small, table - (pages - 40), ints([900, 90]), offsets_of([1, 2]))
    for big, s in zip(cache.tensors, small.tensors):
        assert torch.equal(big[-40:], s)


def check_cross(Hq, Hk, D, q_counts, k_counts, dtype, lens=None, mask=None, padded=False, seed=0, poison=True, scale=None, ld=0):
    """padded: counts are uniform and no offsets are passed."""
    B, Tq, Tk = len(q_counts), sum(q_counts), sum(k_counts)
    t = TYPES[dtype]
    q = rand((Tq, Hq * D + ld), seed, t, gain=1.5)[:, :Hq * D]
    kv = rand((Tk, 2 * Hk * D + ld), seed + 1, t)
    k, v = kv[:, :Hk * D], kv[:, Hk * D:2 * Hk * D]
    seen = torch.ones(Tk, dtype=torch.bool, device="cuda") if mask is None else mask.clone()
    starts = [0] + list(np.cumsum(k_counts))
    if lens is not None:
        for b in range(B):
            seen[starts[b] + min(lens[b], k_counts[b]):starts[b + 1]] = False
    if poison:                                          # what masked rows hold does not matter
        k[~seen], v[~seen] = math.nan, math.inf
    got = fq.cross_attention(q, k, v, Hq, Hk, B, None if padded else offsets_of(q_counts), None if padded else offsets_of(k_counts),
                             None if lens is None else ints(lens), mask, scale=scale)
    scale = D ** -0.5 if scale is None else scale
    k, v = k.double().masked_fill(~seen[:, None], 0.0), v.double().masked_fill(~seen[:, None], 0.0)
    at = 0
    for b in range(B):
        T, L = q_counts[b], k_counts[b]
        see = seen[starts[b]:starts[b + 1]][None].expand(T, -1)
        want, A, W, V = attention_reference(q[at:at + T].double().reshape(T, Hq, D), k[starts[b]:starts[b + 1]].reshape(L, Hk, D),
                                         v[starts[b]:starts[b + 1]].reshape(L, Hk, D), scale, see)
        assert_attention(got[at:at + T], want, A, W, V, L, 2.0 ** -8 if dtype == "bf16" else 0.0)
        if not see.any():
            assert (got[at:at + T] == 0).all()
        at += T


CROSSES = [   # q heads, kv heads, D, queries, keys, type
    (1, 1, 16, [1], [1], "bf16"),
    (16, 16, 64, [50], [816], "bf16"),
    (8, 2, 128, [1, 1, 1], [400, 400, 400], "bf16"),
    (4, 4, 64, [130, 130], [257, 257], "bf16"),
    (8, 1, 256, [17, 17], [300, 300], "bf16"),
    (6, 3, 80, [33, 33], [129, 129], "bf16"),
    (2, 2, 128, [3, 3], [5000, 5000], "bf16"),          # chunks of keys that meet
    (2, 1, 192, [260], [100], "bf16"),
    (4, 2, 64, [40, 40], [200, 200], "f32"),
    (8, 1, 256, [5], [900], "f32"),
    (3, 3, 48, [1, 1], [3000, 3000], "f32"),
]


@gpu
@pytest.mark.parametrize("Hq,Hk,D,queries,keys,dtype", CROSSES)
def test_cross_attention_against_64_bits(Hq, Hk, D, queries, keys, dtype):
    check_cross(Hq, Hk, D, queries, keys, dtype, padded=True, seed=61, ld=16)
    g = torch.Generator(device="cuda").manual_seed(62)
    mask = torch.rand(sum(keys), device="cuda", generator=g) > 0.4
    lens = [max(0, n - 7 * b - 3) for b, n in enumerate(keys)]
    check_cross(Hq, Hk, D, queries, keys, dtype, lens=lens, mask=mask, padded=True, seed=63)


@gpu
@pytest.mark.parametrize("D,queries", [(16, 300), (48, 300), (64, 300), (64, 40), (128, 300), (128, 40), (256, 300)])
def test_cross_attention_masks_over_many_tiles(D, queries):
    """Tiles of keys that are whole, that miss a few keys, that are all masked, in no regular order; more of them than stages."""
    mask = torch.ones(3 * 2100, dtype=torch.bool, device="cuda")
    mask[130:390], mask[700:701], mask[1023:1025], mask[1400:2099], mask[2100:2300], mask[3000:3512] = False, False, False, False, False, False
    mask[4200:6300:7] = False
    check_cross(4, 2, D, [queries] * 3, [2100] * 3, "bf16", mask=mask, padded=True, seed=74)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cross_attention_packed_empty_and_masked_sequences(dtype):
    q_counts, k_counts = [5, 0, 130, 1, 64], [70, 30, 0, 129, 300]       # no queries; no keys
    mask = torch.ones(sum(k_counts), dtype=torch.bool, device="cuda")
    mask[100:229] = False                               # all keys of the fourth sequence
    check_cross(4, 2, 64, q_counts, k_counts, dtype, seed=71)
    check_cross(4, 2, 64, q_counts, k_counts, dtype, mask=mask, seed=72)
    check_cross(4, 2, 64, q_counts, k_counts, dtype, lens=[0, 5, 7, 128, 400], mask=mask, seed=73)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_sequence_stay_and_bad_offsets_stay_inside(dtype):
    q, k = rand((20, 128), 81, TYPES[dtype]), rand((50, 128), 82, TYPES[dtype])
    y = torch.full_like(q, 7.0)
    fq.cross_attention(q, k, k, 2, 2, 2, ints([2, 5, 9]), ints([0, 10, 40]), y=y)
    assert (y[:2] == 7).all() and (y[9:] == 7).all() and not (y[2:9] == 7).all(1).any()
    fq.cross_attention(q, k, k, 2, 2, 2, ints([-5, 15, 900]), ints([30, 700, 10]), y=y)        # cut to the rows that there are
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- together
def _layer_step(x, held, steps_of, cache, table, freq, gain, kv_len, positions, offsets, W):
    """What a layer does between its residuals: qkv projection, norms and positions, cache, attention, o projection."""
    B, T = steps_of
    hq, D = 4, 64
    qkv = fq.linear_w8a8(x, W[0], out_dtype=torch.bfloat16)
    q, k = fq.qk_norm_rope(qkv, hq, 1, D, positions, freq, gain, gain)
    fq.kv8_append(k, qkv[:, (hq + 1) * D:], cache, table, held, offsets, max_new=T)
    o = fq.attention_kv8(q, hq, cache, table, kv_len, offsets, max_q=T, causal=True)
    return fq.linear_w8a8(o, W[1], out_dtype=torch.bfloat16), q, o


@gpu
@pytest.mark.parametrize("T", [1, 37])
def test_the_operators_as_a_layer_runs_them_captured_and_replayed(T):
    """Steps of a decoder layer in one captured graph whose lengths advance on the device, against eager calls; the attention of
    the last step against 64 bits."""
    B, hq, D, P = 3, 4, 64, 16
    width = 16
    W = [fq.fold_weights(rand((n, k), s) * 0.1, None, None, 64, 8) for n, k, s in (((hq + 2) * D, 256, 1), (256, hq * D, 2))]
    freq, gain = fq.rope_frequencies(D), 1 + 0.2 * rand(D, 3)
    offsets = offsets_of([T] * B)
    xs = [rand((B * T, 256), 90 + i, torch.bfloat16) for i in range(4)]

    def fresh():
        c = filled_cache(B * width, 1, D, P, 5)
        return c, table_of(B * width, B, width, 6), ints([0, 7, 20])

    def call(x, c, table, held):
        kv_len = held + T
        positions = (held[:, None] + torch.arange(T, device="cuda", dtype=torch.int32)[None]).flatten()
        out = _layer_step(x, held, (B, T), c, table, freq, gain, kv_len, positions, offsets, W)
        held += T
        return out

    cache, table, held = fresh()
    want = [call(x, cache, table, held) for x in xs]
    lens = held.tolist()
    k, v, ok = dense(cache, table, 1, lens[1])
    seen = torch.arange(lens[1], device="cuda")[None] <= torch.arange(T, device="cuda")[:, None] + lens[1] - T
    o, A, Wt, V = attention_reference(want[-1][1][T:2 * T].double().view(T, hq, D), k, v, D ** -0.5, seen)
    assert_attention(want[-1][2][T:2 * T], o, A, Wt, V, lens[1], 2.0 ** -11)

    cache2, table2, held2 = fresh()
    x = torch.empty_like(xs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(xs[0], *fresh())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(x, cache2, table2, held2)
    for xi, (y, _, _) in zip(xs, want):
        x.copy_(xi)
        graph.replay()
        assert torch.equal(out[0], y)
    for a, b in zip(cache.tensors, cache2.tensors):
        assert torch.equal(a, b)
    st, word = fq.device_status()
    assert st == fq.OK, hex(word)


@gpu
def test_two_graphs_and_two_streams_on_one_and_two_workspaces():
    cache = filled_cache(300, 8, 128, 64, 101)
    table = table_of(300, 2, 100, 102)
    lens = ints([6000, 3333])
    qs = [rand((2, 32 * 128), 103 + i, torch.bfloat16) for i in range(2)]
    want = [fq.attention_kv8(q, 32, cache, table, lens) for q in qs]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    ys = [torch.empty_like(q) for q in qs]
    graphs = [torch.cuda.CUDAGraph() for _ in qs]
    for q, y, g in zip(qs, ys, graphs):
        with torch.cuda.graph(g):
            fq.attention_kv8(q, 32, cache, table, lens, y=y, workspace=ws)
    for _ in range(3):
        ws.fill_(255)                                   # a workspace's contents do not matter
        for g in graphs:
            g.replay()
        for y, w in zip(ys, want):
            assert torch.equal(y, w)
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(fq.attention_kv8(qs[i], 32, cache, table, lens))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


@gpu
def test_attention_returns_the_same_bits_every_time():
    cache = filled_cache(200, 2, 256, 64, 111)
    table = table_of(200, 4, 50, 112)
    lens = ints([3100, 40, 866, 2000])
    for T in (1, 50):
        q = rand((4 * T, 16 * 256), 113, torch.bfloat16)
        first = fq.attention_kv8(q, 16, cache, table, lens, causal=False)
        for _ in range(50):
            assert torch.equal(fq.attention_kv8(q, 16, cache, table, lens, causal=False), first)
    q, k, v = rand((200, 1024), 114, torch.bfloat16), rand((6000, 1024), 115, torch.bfloat16), rand((6000, 1024), 116, torch.bfloat16)
    first = fq.cross_attention(q, k, v, 16, 16, 2)
    for _ in range(50):
        assert torch.equal(fq.cross_attention(q, k, v, 16, 16, 2), first)


@gpu
def test_first_calls_inside_a_capture():
    """A process whose first call of each operator is captured: nothing is set up behind the capture's back."""
    code = """
import torch
from paper_2609_24433_b200 import fq
bf = torch.bfloat16
for T in (1, 40):
    x = torch.randn(2 * T, 6 * 64, device="cuda").to(bf)
    cache = fq.KV8Cache.empty(40, 1, 64, 16)
    table = torch.arange(40, device="cuda", dtype=torch.int32).view(2, 20)
    held = torch.zeros(2, dtype=torch.int32, device="cuda")
    lens, pos, f = held + T, torch.arange(2 * T, device="cuda", dtype=torch.int32), fq.rope_frequencies(64)
    def run():
        q, k = fq.qk_norm_rope(x, 4, 1, 64, pos, f)
        fq.kv8_append(k, x[:, 320:], cache, table, held)
        return fq.attention_kv8(q, 4, cache, table, lens), fq.cross_attention(q, k, k, 4, 1, 2), fq.cross_attention(q.float(), k.float(), k.float(), 4, 1, 2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    g.replay()
    for a, b in zip(out, run()):
        assert torch.equal(a, b)
assert fq.device_status()[0] == fq.OK
print("fine")
"""
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert got.returncode == 0 and "fine" in got.stdout, got.stderr[-2000:]


# ------------------------------------------------------------------------------------------- numbers that are not finite
def plain_attention(q, k, v, scale, seen):
    """The formula in 64 bits, whatever the numbers: q [T, Hq, D], k, v [L, Hk, D], seen [T, L] -> [T, Hq, D].  A query without a key
    gives zeros; values of keys that no query sees do not enter."""
    Hq, Hk = q.shape[1], k.shape[1]
    k, v = (t.masked_fill(~seen.any(0)[:, None, None], 0.0).repeat_interleave(Hq // Hk, 1) for t in (k, v))
    s = torch.where(seen[None], (q.transpose(0, 1)[:, :, None] * k.transpose(0, 1)[:, None]).sum(-1) * scale, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = torch.where(seen[None], p, 0.0)
    o = (p[..., None] * v.transpose(0, 1)[:, None]).sum(2) / p.sum(-1)[..., None]
    return torch.where(seen.any(1)[None, :, None], o, 0.0).transpose(0, 1)


def assert_same_kind(got, want):
    """NaN where the formula has it, and infinities with its signs."""
    got = got.double().view_as(want)
    assert torch.equal(got.isnan(), want.isnan()), f"{(got.isnan() != want.isnan()).sum().item()} of {got.numel()} numbers are NaN on one side only"
    assert torch.equal(got.isposinf(), want.isposinf()) and torch.equal(got.isneginf(), want.isneginf())


NOT_FINITE = [math.nan, math.inf, -math.inf]


@gpu
@pytest.mark.parametrize("bad", NOT_FINITE)
@pytest.mark.parametrize("Hq,Hk,D,T,dtype", [
    (8, 1, 64, 1, "bf16"), (8, 1, 256, 2, "bf16"), (3, 1, 128, 1, "f32"),                   # few queries: one and two tiles of columns, two terms
    (4, 2, 64, 40, "bf16"), (2, 1, 64, 300, "bf16"), (2, 1, 128, 300, "bf16"), (8, 1, 256, 40, "bf16"),
    (4, 2, 64, 40, "f32")])
@pytest.mark.parametrize("n", [1, 200, 2100])
def test_attention_kv8_of_queries_that_are_not_finite(bad, Hq, Hk, D, T, dtype, n):
    """A row with a channel that is not finite is NaN where it sees a key (every score is NaN or infinite, and the largest less itself
    is NaN), zeros where it sees none; all other rows are what they were."""
    cache = filled_cache(70, Hk, D, 32, 121)
    table = table_of(70, 1, 70, 122)
    q = rand((T, Hq * D), 123, TYPES[dtype])
    kv = ints([n])
    for causal in (True, False):
        want = fq.attention_kv8(q, Hq, cache, table, kv, causal=causal)
        x = q.clone()
        rows = sorted({0, T // 3, T - 1})
        for i, r in enumerate(rows):
            x[r, (Hq - 1) * D + (5 + 17 * i) % D] = bad
        got = fq.attention_kv8(x, Hq, cache, table, kv, causal=causal)
        for r in rows:
            sees = n > 0 and (not causal or n - T + r >= 0)
            tail = got[r, (Hq - 1) * D:]
            assert tail.isnan().all() if sees else (tail == 0).all(), (r, tail[:4])
            want[r, (Hq - 1) * D:] = got[r, (Hq - 1) * D:] = 0
        assert torch.equal(got, want)


@gpu
@pytest.mark.parametrize("Hq,Hk,D,T,L,B,dtype", [
    (4, 2, 64, 40, 200, 2, "bf16"), (2, 2, 64, 300, 250, 1, "bf16"), (2, 1, 128, 300, 200, 1, "bf16"), (4, 1, 256, 40, 200, 2, "bf16"),
    (4, 2, 64, 40, 2100, 2, "bf16"), (2, 1, 64, 300, 2100, 1, "bf16"), (2, 1, 128, 300, 2100, 1, "bf16"), (4, 1, 256, 40, 2100, 1, "bf16"),   # chunks
    (4, 4, 64, 9, 700, 40, "bf16"),                                                                                                         # long, one chunk
    (4, 2, 64, 3, 200, 2, "f32"), (4, 2, 64, 40, 200, 2, "f32"), (4, 2, 128, 40, 2100, 2, "f32")])
def test_cross_attention_of_numbers_that_are_not_finite(Hq, Hk, D, T, L, B, dtype):
    q, k, v = (rand((B * n, h * D), 131 + i, TYPES[dtype]) for i, (n, h) in enumerate(((T, Hq), (L, Hk), (L, Hk))))
    mask = torch.rand(B * L, device="cuda", generator=torch.Generator(device="cuda").manual_seed(134)) > 0.1
    clean = fq.cross_attention(q, k, v, Hq, Hk, B, key_mask=mask)

    def check(q, k, v, mask, touched):
        got = fq.cross_attention(q, k, v, Hq, Hk, B, key_mask=mask)
        want = torch.cat([plain_attention(q[b * T:(b + 1) * T].double().view(T, Hq, D), k[b * L:(b + 1) * L].double().view(L, Hk, D),
                                          v[b * L:(b + 1) * L].double().view(L, Hk, D), D ** -0.5, mask[b * L:(b + 1) * L][None].expand(T, -1))
                          for b in touched])
        rows = torch.cat([torch.arange(b * T, (b + 1) * T, device="cuda") for b in touched])
        assert_same_kind(got[rows], want)
        rest = torch.ones(B * T, dtype=torch.bool, device="cuda")
        rest[rows] = False
        assert torch.equal(got[rest], clean[rest])
        # what is finite is near: a score loses (D + 8) u A, a probability 2^-8 at most, the store half a step (see the top of this file)
        fine = want.isfinite()
        size = v.double().masked_fill(~v.isfinite(), 0.0).abs().max()
        assert ((got[rows].double().view_as(want) - want)[fine].abs() <= 2.0 ** -6 * size).all()
        return got

    for bad in NOT_FINITE:
        x = q.clone()
        x[0, 3] = x[T - 1, Hq * D - 1] = x[T // 2, D] = bad
        check(x, k, v, mask, [0])
        for j in (0, 1, 2, 15, 16 * (L // 32) + 1, L - 1):
            seen = mask.clone()
            seen[j] = True
            clean = fq.cross_attention(q, k, v, Hq, Hk, B, key_mask=seen)
            x = k.clone()
            x[j, D - 2] = bad
            check(q, x, v, seen, [0])
            x = v.clone()
            x[j, Hk * D - 3] = bad
            check(q, k, x, seen, [0])
            seen[j] = False                             # behind the mask it does not matter
            x, z = k.clone(), v.clone()
            x[j], z[j] = bad, bad
            assert torch.equal(fq.cross_attention(q, x, z, Hq, Hk, B, key_mask=seen), fq.cross_attention(q, k, v, Hq, Hk, B, key_mask=seen))
        clean = fq.cross_attention(q, k, v, Hq, Hk, B, key_mask=mask)


@gpu
@pytest.mark.parametrize("bad", NOT_FINITE)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,D,T,L", [(2, 64, 40, 200), (2, 64, 300, 200), (2, 128, 300, 250), (1, 256, 40, 200), (2, 64, 40, 1500), (2, 128, 300, 1500)])
def test_attention_of_numbers_that_are_not_finite_ahead_of_keys_that_are_masked(Hq, D, T, L, dtype, bad):
    """The last tiles of keys, and the last chunks, hold nothing that a row sees, whatever it saw ahead of them."""
    q, k, v = (rand((n, Hq * D), 221 + i, TYPES[dtype]) for i, n in enumerate((T, L, L)))
    mask = torch.ones(L, dtype=torch.bool, device="cuda")
    mask[100:] = False
    x = k.clone()
    x[50, 7] = bad
    want = plain_attention(q.double().view(T, Hq, D), x.double().view(L, Hq, D), v.double().view(L, Hq, D), D ** -0.5, mask[None].expand(T, -1))
    assert_same_kind(fq.cross_attention(q, x, v, Hq, Hq, 1, key_mask=mask), want)
    x = q.clone()
    x[T // 2, 7] = bad
    want = plain_attention(x.double().view(T, Hq, D), k.double().view(L, Hq, D), v.double().view(L, Hq, D), D ** -0.5, mask[None].expand(T, -1))
    assert_same_kind(fq.cross_attention(x, k, v, Hq, Hq, 1, key_mask=mask), want)
    cache = filled_cache(100, Hq, D, 16, 224)
    table = table_of(100, 1, 100, 225)
    table[0, 6:] = -1                                   # no pages behind 96 keys
    got = fq.attention_kv8(x, Hq, cache, table, ints([L]), causal=False)
    assert got[T // 2, :D].isnan().all() and torch.isfinite(got[T // 2, D:]).all()
    rest = torch.arange(T, device="cuda") != T // 2
    assert torch.equal(got[rest], fq.attention_kv8(q, Hq, cache, table, ints([L]), causal=False)[rest])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,D,T,L", [(2, 64, 40, 200), (2, 64, 300, 2100), (2, 128, 300, 2100), (1, 256, 40, 2100), (2, 64, 3, 1)])
def test_cross_attention_of_scores_that_are_all_minus_infinity(Hq, D, T, L, dtype):
    """exp(-inf - (-inf)): NaN, as the formula has it, and not the zeros of a query without a key; keys at minus infinity beside others
    count for nothing, a whole chunk of them too."""
    q, k, v = (rand((n, Hq * D), 141 + i, TYPES[dtype]) for i, n in enumerate((T, L, L)))
    q[:, 0] = 1.0
    low = k.clone()
    low[:, 0] = -math.inf
    got = fq.cross_attention(q, low, v, Hq, Hq, 1)
    assert got[:, :D].isnan().all()
    assert torch.equal(got[:, D:], fq.cross_attention(q, k, v, Hq, Hq, 1)[:, D:])
    if L > 1:
        keep = torch.zeros(L, dtype=torch.bool, device="cuda")
        keep[[L - 1, L // 3]] = True
        low = k.clone()
        low[~keep, 0] = -math.inf
        got = fq.cross_attention(q, low, v, Hq, Hq, 1)[:, :D]
        want = plain_attention(q.double().view(T, Hq, D), k.double().view(L, Hq, D), v.double().view(L, Hq, D), D ** -0.5, keep[None].expand(T, -1))[:, 0]
        assert ((got.double() - want).abs() <= 2.0 ** -6 * v.double().abs().max()).all()


@gpu
@pytest.mark.parametrize("size", [1e5, 1e8, 1e12, 1e25])
@pytest.mark.parametrize("D,T,dtype", [(64, 40, "bf16"), (64, 300, "bf16"), (128, 300, "bf16"), (256, 40, "bf16"), (64, 1, "bf16"), (64, 1, "f32"), (64, 40, "f32")])
def test_attention_of_huge_scores_takes_the_largest(D, T, dtype, size):
    """Scores whose binary32 steps are large, and further apart than their error, which is (D + 8) u A: the key with the largest one has
    probability 1.  It takes one rounding of at most 2^-8 (rows; over the cache 2^-11), the store half a step; exponentials are good to 2^-18."""
    L = 700
    q = rand((T, 2 * D), 151, TYPES[dtype], gain=size)
    cache = filled_cache(30, 2, D, 32, 152)
    table = table_of(30, 1, 22, 153)
    k, v, _ = dense(cache, table, 0, L)
    ks, vs = (rand((L, 2 * D), 154 + i, TYPES[dtype]) for i in range(2))
    calls = [(fq.attention_kv8(q, 2, cache, table, ints([L]), causal=False), k, v, 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22),
             (fq.cross_attention(q, ks, vs, 2, 2, 1), ks.double().view(L, 2, D), vs.double().view(L, 2, D), 2.0 ** -8 if dtype == "bf16" else 0.0)]
    for got, k, v, rounded in calls:
        x = q.double().view(T, 2, D)
        s = torch.einsum("thd,lhd->thl", x, k) * D ** -0.5
        A = (torch.einsum("thd,lhd->thl", x.abs(), k.abs()) * D ** -0.5).amax(-1)
        two = s.topk(2, -1)
        clear = two.values[..., 0] - two.values[..., 1] > 4 * (D + 8) * U * A + 64
        assert clear.sum() > 0.5 * clear.numel()
        want = torch.stack([v[two.indices[:, h, 0], h] for h in range(2)], 1)
        off = (got.double().view(T, 2, D) - want).abs()
        assert (off <= (rounded + 2.0 ** -16 + HALF[got.dtype]) * want.abs())[clear].all()


@gpu
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -140, 2.0 ** -127])
@pytest.mark.parametrize("D,T,dtype", [(64, 40, "bf16"), (64, 300, "bf16"), (128, 300, "bf16"), (256, 40, "bf16"), (64, 40, "f32")])
def test_attention_of_scales_below_the_smallest_normal_number(D, T, dtype, scale):
    """Products up to the largest binary32 numbers: no scale is raised to what would tell them apart."""
    L, g = 300, 2.2e18 * (64 / D) ** 0.25
    q, k = (rand((n, 2 * D), 161 + i, TYPES[dtype], gain=g) for i, n in enumerate((T, L)))
    v = rand((L, 2 * D), 163, TYPES[dtype])
    got = fq.cross_attention(q, k, v, 2, 2, 1, scale=scale)
    want, A, W, V = attention_reference(q.double().view(T, 2, D), k.double().view(L, 2, D), v.double().view(L, 2, D), scale,
                                     torch.ones(T, L, dtype=torch.bool, device="cuda"))
    assert_attention(got, want, A, W, V, L, 2.0 ** -8 if dtype == "bf16" else 0.0)
    cache = filled_cache(12, 2, D, 32, 164)
    check_cache_attention(cache, table_of(12, 1, 10, 165), [L], [T], 2, dtype, False, scale=scale, seed=166)


@gpu
def test_positions_frequencies_and_page_scales_begin_anywhere():
    """Views that start inside an allocation: these arrays are read one element at a time."""
    M, D = 40, 64
    x = rand((M, 4 * D), 171, torch.bfloat16)
    positions, freq = ints(range(M + 1)), torch.cat([torch.zeros(1, dtype=torch.float64, device="cuda"), fq.rope_frequencies(D)])
    want = fq.qk_norm_rope(x, 2, 1, D, positions[1:].clone(), freq[1:].clone())
    got = fq.qk_norm_rope(x, 2, 1, D, positions[1:], freq[1:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    aligned = filled_cache(6, 1, D, 16, 172)
    scales = torch.empty(2, 7, device="cuda")
    other = fq.KV8Cache(aligned.k.clone(), aligned.v.clone(), scales[0, 1:].view(6, 1), scales[1, :6].view(6, 1))
    other.k_scale.copy_(aligned.k_scale)
    other.v_scale.copy_(aligned.v_scale)
    table, new = ints([[2, 0, 1, 5]]), rand((M, D), 173, torch.bfloat16)
    for c in (aligned, other):
        fq.kv8_append(new, new, c, table, ints([3]))
    for a, b in zip(aligned.tensors, other.tensors):
        assert torch.equal(a, b)
    for T, t in ((1, torch.bfloat16), (M, torch.bfloat16), (M, torch.float32)):
        q = rand((T, 2 * D), 174, t)
        assert torch.equal(*(fq.attention_kv8(q, 2, c, table, ints([M + 3])) for c in (aligned, other)))


@gpu
def test_binary32_rows_with_leading_dimensions_of_four():
    """16 bytes are four binary32 channels."""
    D, T, L = 48, 40, 300

    def rows(n, width, seed):
        t = torch.full((n, width + 4), 7.0, device="cuda")
        t[:, :width] = rand((n, width), seed)
        return t[:, :width]

    qkv, positions, freq = rows(T, 4 * D, 181), ints(range(T)), fq.rope_frequencies(D)
    q, k = rows(T, 2 * D, 182), rows(T, D, 183)
    fq.qk_norm_rope(qkv, 2, 1, D, positions, freq, q=q, k=k)
    for got, want in zip((q, k), fq.qk_norm_rope(qkv.contiguous(), 2, 1, D, positions, freq)):
        assert torch.equal(got, want)
    new, caches, table = rows(L, D, 184), [filled_cache(20, 1, D, 16, 185) for _ in range(2)], table_of(20, 1, 20, 186)
    for x, c in zip((new, new.contiguous()), caches):
        fq.kv8_append(x, x, c, table, ints([5]))
    for a, b in zip(caches[0].tensors, caches[1].tensors):
        assert torch.equal(a, b)
    for n in (1, T):
        y = rows(n, 2 * D, 187)
        fq.attention_kv8(q[:n], 2, caches[0], table, ints([L]), y=y)
        assert torch.equal(y, fq.attention_kv8(q[:n].contiguous(), 2, caches[0], table, ints([L])))
        fq.cross_attention(q[:n], new, new, 2, 1, 1, y=y)
        assert torch.equal(y, fq.cross_attention(q[:n].contiguous(), new.contiguous(), new.contiguous(), 2, 1, 1))
        assert (y._base[:, 2 * D:] == 7).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_kv8_single_tokens_of_more_sequences_than_a_grid_has_rows(dtype):
    B, H, D = 8200, 8, 16                               # 65600 (sequence, head) pairs
    cache = filled_cache(300, H, D, 16, 191)
    table = torch.randint(0, 300, (B, 2), generator=torch.Generator().manual_seed(192)).int().cuda()
    lens = torch.randint(0, 33, (B,), generator=torch.Generator().manual_seed(193)).int().cuda()
    q = rand((B, H * D), 194, TYPES[dtype])
    got = fq.attention_kv8(q, H, cache, table, lens)
    for rows in (slice(0, B // 2), slice(B // 2, B)):
        assert torch.equal(got[rows], fq.attention_kv8(q[rows], H, cache, table[rows], lens[rows]))
    with pytest.raises(fq.FqError) as e:                # (other kernels have a grid of them)
        fq.attention_kv8(rand((3 * B, 8 * H * D), 195, TYPES[dtype]), 8 * H, cache, table, lens)
    assert e.value.status == fq.ERR_UNSUPPORTED


# ------------------------------------------------------------------------------------------- offsets that nobody has checked
def inside(t, edge):
    """t as an inner slice of a larger tensor, with `edge` in 40 rows on either side of it: (slice, whole)."""
    whole = torch.full((len(t) + 80, *t.shape[1:]), edge, dtype=t.dtype, device="cuda")
    whole[40:-40] = t
    return whole[40:-40], whole


def edges_are(whole, edge):
    return bool((whole[:40] == edge).all() and (whole[-40:] == edge).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_by_offsets_that_leave_the_rows_or_fall(dtype):
    """They are cut to the rows that there are: what is around the rows, the pages and the scales is neither read nor written."""
    H, D, P = 2, 32, 16
    start = filled_cache(8, H, D, P, 201)
    table = ints([[5, 1, 3], [0, 4, 6]])
    x = rand((90, 2 * H * D), 202, TYPES[dtype])
    for bad, cut in (([80, 500, 10], [80, 90, 90]), ([-30, 20, 2 ** 31 - 1], [0, 20, 90]), ([50, 40, 45], [50, 50, 50]), ([-9, -5, 3], [0, 0, 3])):
        kv, _ = inside(x, math.nan)
        parts = [inside(t, e) for t, e in zip(start.tensors, (77, 77, 9.0, 9.0))]
        cache = fq.KV8Cache(*(p[0] for p in parts))
        fq.kv8_append(kv[:, :H * D], kv[:, H * D:], cache, table, ints([3, 7]), ints(bad))
        want = fq.KV8Cache(*(t.clone() for t in start.tensors))
        # ([50, 40, 45]: the second sequence begins at row 40)
        if bad == [50, 40, 45]:
            fq.kv8_append(x[40:45, :H * D], x[40:45, H * D:], want, table[1:], ints([7]))
        else:
            fq.kv8_append(x[:, :H * D], x[:, H * D:], want, table, ints([3, 7]), ints(cut))
        for (got, whole), t, e in zip(parts, want.tensors, (77, 77, 9.0, 9.0)):
            assert torch.equal(got, t) and edges_are(whole, e)
        if bad[0] == 80:                                # ten rows behind three that were held: the first page of sequence 0
            changed = [p for p in range(8) if not torch.equal(cache.k[p], start.k[p]) or not torch.equal(cache.v[p], start.v[p])]
            assert changed == [5]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,D,max_q", [(2, 2, 64, 1), (4, 1, 64, 3), (2, 1, 128, 0), (4, 2, 256, 0), (2, 2, 64, 0)])
def test_attention_by_offsets_that_leave_the_rows_or_fall(Hq, Hk, D, max_q, dtype):
    t = TYPES[dtype]
    rows, keys = 300, 400
    xq, xk, xv = (rand((n, h * D), 211 + i, t) for i, (n, h) in enumerate(((rows, Hq), (keys, Hk), (keys, Hk))))
    start = filled_cache(40, Hk, D, 16, 214)
    table = table_of(40, 2, 20, 215)
    for bad, cut in (([-5, 130, 9000], [0, 130, 300]), ([250, 2 ** 31 - 1, 10], [250, 300, 300]), ([-8, -3, 70], [0, 0, 70])):
        for k_bad, k_cut in (([30, 700, 10], [30, 400, 400]), ([-40, 200, 401], [0, 200, 400])):
            (q, _), (k, _), (v, _), (y, around) = (inside(x, e) for x, e in ((xq, math.nan), (xk, math.nan), (xv, math.nan), (torch.full_like(xq, 7.0), 7.0)))
            fq.cross_attention(q, k, v, Hq, Hk, 2, ints(bad), ints(k_bad), max_q=max_q, y=y)
            want = fq.cross_attention(xq, xk, xv, Hq, Hk, 2, ints(cut), ints(k_cut), max_q=max_q, y=torch.full_like(xq, 7.0))
            assert torch.equal(y, want) and edges_are(around, 7.0)
        parts = [inside(x, e) for x, e in zip(start.tensors, (77, 77, math.nan, math.nan))]
        y, around = inside(torch.full_like(xq, 7.0), 7.0)
        fq.attention_kv8(q, Hq, fq.KV8Cache(*(p[0] for p in parts)), table, ints([290, 2 ** 31 - 1]), ints(bad), max_q=max_q, y=y)
        want = fq.attention_kv8(xq, Hq, start, table, ints([290, 320]), ints(cut), max_q=max_q, y=torch.full_like(xq, 7.0))
        assert torch.equal(y, want) and edges_are(around, 7.0)
        assert torch.isfinite(y).all() and (y[:max(0, cut[0])] == 7).all() and (y[cut[2]:] == 7).all()
