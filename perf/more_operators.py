"""Workloads of the projection in microscaled 4-bit floating point (quantisation of the activations, product, both in one
call) and of the RMS norm with the residual's addition that ends in a projection's codes.

``listed()`` and ``draw()`` describe cases, ``prepare()`` makes what a program holds before the call, ``run()`` makes one
call -- of the library where ``own`` is true, of the same formula in elementary torch operations where it is not --
and ``exact()`` evaluates the definition in 64 bits.

Codes are e2m1, two to a byte, the even channel in the low nibble.  Block scales are e8m0 for 32 channels ("mx") or e4m3 for
16 ("nv"), in tiles of 128 rows x 4 blocks: byte (row % 32) * 16 + (row % 128) / 32 * 4 + block % 4 of tile
(row / 128, block / 4); places past the last row or block hold 0.  A row's value is code * block scale * step.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = {"mx": 32, "nv": 16}


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # one denoising step of the action expert: 50 tokens of width 1024; latency counts
        dict(name="quantize_step", op="quantize", tokens=50, K=1024, hadamard=64, form="nv", dtype="bf16"),
        # the backbone's prefix (816 tokens, hidden 2048) of sixteen robots
        dict(name="quantize_prefix", op="quantize", tokens=13056, K=2048, hadamard=128, form="mx", dtype="bf16"),
        # a long binary32 batch without a rotation
        dict(name="quantize_long_f32", op="quantize", tokens=8191, K=8192, hadamard=1, form="nv", dtype="f32"),
        # one token through the backbone's fused q/k/v projection: weights are streamed, latency counts
        dict(name="product_token", op="product", tokens=1, K=2048, N=2560, form="nv", dtype="bf16"),
        # a padded batch of an odd size, few channels, binary32 outputs
        dict(name="product_ragged_f32", op="product", tokens=333, K=1120, N=1000, form="mx", dtype="f32"),
        # the throughput sweep's long batch
        dict(name="product_long", op="product", tokens=16384, K=8192, N=8192, form="nv", dtype="bf16"),
        # one step of the action expert through an MLP projection, quantisation included
        dict(name="linear_step", op="linear", tokens=50, K=1024, N=4096, hadamard=64, form="nv", dtype="bf16"),
        # the backbone's fused gate/up projection and its down projection
        dict(name="linear_gate_up", op="linear", tokens=816, K=2048, N=32768, hadamard=128, form="nv", dtype="bf16"),
        dict(name="linear_down", op="linear", tokens=816, K=16384, N=2048, hadamard=256, form="mx", dtype="bf16"),
        # residual and norm ahead of the action expert's q/k/v projection; latency counts
        dict(name="norm_step", op="norm", tokens=50, K=1024, hadamard=64, form="int8", dtype="bf16", residual=True),
        # ahead of the backbone's, for sixteen robots
        dict(name="norm_prefix", op="norm", tokens=13056, K=2048, hadamard=1, form="int8", dtype="bf16", residual=True),
        # a binary32 residual stream of an odd length
        dict(name="norm_long_f32", op="norm", tokens=4095, K=5120, hadamard=256, form="int8", dtype="f32", residual=True),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "linear", "norm"])
    hadamard = rng.choice([1, 1, 32, 64, 128, 256])
    unit = max(32, hadamard)
    K = unit * _log(rng, max(1, 256 // unit), 16384 // unit)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    form = rng.choice(["mx", "nv"])
    if op in ("quantize", "norm"):
        tokens = _log(rng, 1, min(16384, (1 << 26) // K))
        if op == "quantize":
            return dict(op=op, tokens=tokens, K=K, hadamard=hadamard, form=form, dtype=dtype)
        return dict(op=op, tokens=tokens, K=K, hadamard=hadamard, form=rng.choice(["int8", "int8", "mx", "nv"]), dtype=dtype, residual=rng.random() < 0.8)
    N = 8 * _log(rng, 8, min(4096, (1 << 26) // K // 8))
    tokens = rng.choice([rng.randint(1, 16), _log(rng, 1, min(16384, (1 << 39) // (N * K)))])
    if op == "product":
        return dict(op=op, tokens=tokens, K=K, N=N, form=form, dtype=dtype)
    return dict(op=op, tokens=tokens, K=K, N=N, hadamard=hadamard, form=form, dtype="bf16")


# ---------------------------------------------------------------------------- inputs
def _tokens(g, M, K, dtype):
    x = torch.randn(M, K, device="cuda", generator=g)
    loud = torch.rand(K, device="cuda", generator=g) < 0.005            # channels of a larger amplitude
    return (x * torch.where(loud, 30.0, 1.0)).to(DTYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, K, form = case["tokens"], case["K"], case["form"]
    s = dict(case=case)
    if case["op"] == "product":
        s["codes"], s["scales"], s["steps"] = _quantize(_tokens(g, M, K, "f32"), form)
    else:
        s["x"] = _tokens(g, M, K, case["dtype"])
        # smoothing scales and the rotation's norm, as a folded site keeps them
        s["mult"] = torch.exp(0.3 * torch.randn(K, device="cuda", generator=g)) * case["hadamard"] ** -0.5
    if case["op"] == "norm":
        s["residual"] = _tokens(g, M, K, case["dtype"]) if case["residual"] else None
    if "N" in case:
        W = torch.randn(case["N"], K, device="cuda", generator=g) * 0.02
        s["w_codes"], s["w_scales"], s["w_steps"] = _quantize(W, form)
        s["bias"] = 0.1 * torch.randn(case["N"], device="cuda", generator=g)
    if own:
        from paper_2609_24433_b200 import fq
        if "N" in case:
            s["handle"] = fq.weights_import_fp4(s["w_codes"], s["w_scales"], s["w_steps"], s.get("mult"), s["bias"], K, case.get("hadamard", 1), _format(form))
    return s


def _format(form):
    from paper_2609_24433_b200 import fq
    return {"mx": fq.MXFP4, "nv": fq.NVFP4}[form]


# ---------------------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2609_24433_b200 import fq
    c = s["case"]
    if c["op"] == "quantize":
        return fq.quantize_act_fp4(s["x"], s["mult"], c["hadamard"], _format(c["form"]))
    if c["op"] == "product":
        return fq.gemm_fp4(s["codes"], s["scales"], s["steps"], s["handle"], DTYPES[c["dtype"]])
    if c["op"] == "linear":
        return fq.linear_fp4(s["x"], s["handle"], DTYPES[c["dtype"]])
    if c["form"] == "int8":
        h, codes, steps = fq.rmsnorm_quantize_act(s["x"], s["residual"], s["mult"], c["hadamard"], 8, eps=1e-6)
        return h, codes.view(torch.int8), steps
    return fq.rmsnorm_quantize_act_fp4(s["x"], s["residual"], s["mult"], c["hadamard"], _format(c["form"]), eps=1e-6)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "quantize":
        return _quantize(_rotate(s["x"].float() * s["mult"], c["hadamard"]), c["form"])
    if c["op"] == "product":
        return _product(s, s["codes"], s["scales"], s["steps"])
    if c["op"] == "linear":
        return _product(s, *_quantize(_rotate(s["x"].float() * s["mult"], c["hadamard"]), c["form"]))
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    wide = h.float()
    r = torch.rsqrt((wide * wide).mean(1) + 1e-6)
    # the quantiser is homogeneous: a row's codes are those from before the division by its norm, which the step takes
    z = _rotate(wide * s["mult"], c["hadamard"])
    if c["form"] != "int8":
        codes, scales, steps = _quantize(z, c["form"])
        return h, codes, scales, steps * r
    step = z.abs().amax(1) / 127.0
    held = step >= 2.0 ** -126
    inverse = torch.where(held, 1.0 / step, torch.zeros_like(step))
    codes = torch.round(z * inverse[:, None]).to(torch.int8)
    return h, codes, torch.where(held, step, torch.zeros_like(step)) * r


def _rotate(v, block):
    """Butterflies of ascending strides in 32 bits (each rounding of theirs decides codes, so their order is part of the definition)."""
    shape, h = v.shape, 1
    while h < block:
        a, b = v.view(-1, 2, h).unbind(1)
        v = torch.stack([a + b, a - b], 1).view(shape)
        h *= 2
    return v


def _nibbles(v):
    """e2m1 of v, nearest with ties to the even mantissa, at most 6."""
    a = v.abs()
    n = (a > 0.25).to(torch.uint8)
    n = n.add_(a >= 0.75).add_(a > 1.25).add_(a >= 1.75).add_(a > 2.5).add_(a >= 3.5).add_(a > 5.0)
    n = n.add_(torch.signbit(v), alpha=8)
    return n[:, 0::2] + n[:, 1::2] * 16


def _tiles(scales):
    rows, blocks = scales.shape
    t, a = -(-rows // 128), -(-blocks // 4)
    out = torch.zeros(t * 128, a * 4, dtype=torch.uint8, device="cuda")
    out[:rows, :blocks] = scales
    return out.view(t, 4, 32, a, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _quantize(z, form):
    M, K = z.shape
    parts = z.view(M, -1, BLOCK[form])
    most = parts.abs().amax(2)
    if form == "mx":
        e = ((most.view(torch.int32) >> 23) - 2).clamp_min(0)
        v = parts * ((254 - e) << 23).view(torch.float32)[:, :, None]
        return _nibbles(v.view(M, K)), _tiles(e.to(torch.uint8)), torch.ones(M, device="cuda")
    step = most.amax(1) / 2688.0
    held = step >= 2.0 ** -100
    inverse = torch.where(held, 1.0 / step, torch.zeros_like(step))
    scale = ((most * inverse[:, None]) * 0.1666666716337204).clamp_max(448.0).to(torch.float8_e4m3fn)
    wide = scale.float()
    v = parts * torch.where(wide > 0, inverse[:, None] / wide, torch.zeros_like(wide))[:, :, None]
    return _nibbles(v.view(M, K)), _tiles(scale.view(torch.uint8)), torch.where(held, step, torch.zeros_like(step))


def _values(codes, scales, form):
    """What codes and block scales stand for, in 32 bits (each product is exact)."""
    M, K, blocks = codes.shape[0], 2 * codes.shape[1], 2 * codes.shape[1] // BLOCK[form]
    e2m1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    e2m1 = torch.cat([e2m1, -e2m1])
    pairs = torch.stack([e2m1.repeat(16), e2m1.repeat_interleave(16)], 1)
    v = pairs[codes.int()].view(M, blocks, -1)
    a = -(-blocks // 4)
    flat = scales.view(-1, a, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, a * 4)[:M, :blocks]
    wide = torch.exp2(flat.float() - 127.0) if form == "mx" else flat.contiguous().view(torch.float8_e4m3fn).float()
    return (v * wide[:, :, None]).view(M, K)


def _product(s, codes, scales, steps):
    c = s["case"]
    a, w = _values(codes, scales, c["form"]), _values(s["w_codes"], s["w_scales"], c["form"])
    y = torch.matmul(a, w.T) * (steps[:, None] * s["w_steps"]) + s["bias"]
    return y.to(DTYPES[c["dtype"]])


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    M, K, e = case["tokens"], case["K"], 4 if case["dtype"] == "f32" else 2
    held = 0.5 + 1.0 / BLOCK[case["form"]] if case["form"] in BLOCK else 1.0      # bytes of a quantised channel
    turns = max(1, case.get("hadamard", 1)).bit_length() - 1
    if case["op"] == "quantize":
        return dict(bytes=(e + held) * M * K + 4 * K + 4 * M, flops=(turns + 3) * M * K)
    if case["op"] == "norm":
        reads, writes = (2, 1) if case["residual"] else (1, 0)                     # (without a residual the stream stays as it is)
        return dict(bytes=((reads + writes) * e + held) * M * K + 4 * K + 4 * M, flops=(turns + 6) * M * K)
    N = case["N"]
    tokens = e * M * K if case["op"] == "linear" else held * M * K
    return dict(bytes=tokens + held * N * K + e * M * N + 4 * M + 8 * N, flops=2 * M * N * K)


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "product":
        return _exact_product(s, _decoded(s["codes"], s["scales"], case["form"]) * s["steps"].double()[:, None])
    x = s["x"].double()
    if case["op"] == "norm":
        if s["residual"] is not None:
            x = x + s["residual"].double()
        h = x.to(s["x"].dtype).double()
        z = _turned(h * s["mult"].double(), case["hadamard"])
        norm = (h.square().sum(1) / case["K"] + 1e-6).sqrt()
        steps = 1.0 / norm if case["form"] == "mx" else z.abs().max(1).values / {"int8": 127, "nv": 2688}[case["form"]] / norm
        return (x, None, steps) if case["form"] == "int8" else (x, None, None, steps)
    z = _turned(x * s["mult"].double(), case["hadamard"])
    if case["op"] == "quantize":
        return None, None, torch.ones(case["tokens"], dtype=torch.float64, device="cuda") if case["form"] == "mx" else z.abs().max(1).values / 2688
    return _exact_product(s, _rounded(z, case["form"]))


def _turned(v, block):
    h = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    while h.shape[0] < block:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return (v.view(-1, block) @ h).view(v.shape)


def _rounded(z, form):
    """z as its codes, block scales and steps have it."""
    parts = z.view(z.shape[0], -1, BLOCK[form])
    peak = parts.abs().max(2, keepdim=True).values
    if form == "mx":
        unit = torch.pow(2.0, torch.floor(torch.log2(peak.clamp_min(2.0 ** -124))) - 2)
    else:
        step = peak.max(1, keepdim=True).values / 2688
        unit = (peak / 6 / step).float().to(torch.float8_e4m3fn).double() * step
    a = (parts / unit).abs().nan_to_num(0.0).clamp_max(6.0)
    grid = torch.pow(2.0, torch.floor(torch.log2(a.clamp_min(1.0))) - 1)        # distance of the e2m1 numbers around a
    return (torch.round(a / grid) * grid * unit * torch.sign(parts)).view(z.shape)


def _decoded(codes, scales, form):
    rows, K = codes.shape[0], 2 * codes.shape[1]
    n = torch.stack([codes % 16, codes // 16], 2).view(rows, K).long()
    exponent, half = (n // 2) % 4, (n % 2).double()
    v = torch.where(exponent == 0, half / 2, (1 + half / 2) * torch.pow(2.0, (exponent - 1).double())) * (1 - 2 * (n // 8)).double()
    r, b = torch.arange(rows, device="cuda")[:, None], torch.arange(K // BLOCK[form], device="cuda")[None]
    across = -(-(K // BLOCK[form]) // 4)
    byte = scales[((r // 128) * across + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4].double()
    if form == "mx":
        scale = torch.pow(2.0, byte - 127)
    else:
        scale = torch.where(byte < 8, byte / 512, (1 + byte % 8 / 8) * torch.pow(2.0, torch.floor(byte / 8) - 7))
    return (v.view(rows, -1, BLOCK[form]) * scale[:, :, None]).view(rows, K)


def _exact_product(s, tokens):
    w = _decoded(s["w_codes"], s["w_scales"], s["case"]["form"]) * s["w_steps"].double()[:, None]
    return tokens @ w.T + s["bias"].double()
