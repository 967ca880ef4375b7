"""Projections in microscaled 4-bit floating point, and the RMS norm that ends in codes, on the GPU: codes, scales and steps bit
for bit against the stated binary32 sequence in numpy, products against 64 bits, the norm against the calls that it fuses."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_24433_b200 import fq

pytestmark = pytest.mark.gpu

FORMATS = {"mx": fq.MXFP4, "nv": fq.NVFP4}
BLOCK = {"mx": 32, "nv": 16}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------- the definitions, apart from the library's code
def nearest_even(v, grid):
    """Index of the grid value nearest to each v >= 0, ties to the even index, saturating (64 bits: distances are exact)."""
    v = np.minimum(v.astype(np.float64), grid[-1])
    hi = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = v - grid[lo], grid[hi] - v
    return np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))


def rotate(x, g, block):
    """Multiplier and butterflies, one binary32 operation at a time."""
    v = (x.astype(np.float32) * g.astype(np.float32)).astype(np.float32)
    h = 1
    while h < block:
        p = v.reshape(v.shape[0], -1, 2, h)
        v = np.stack([p[:, :, 0] + p[:, :, 1], p[:, :, 0] - p[:, :, 1]], 2).reshape(v.shape)
        h *= 2
    return v


def tiles(scales):
    rows, blocks = scales.shape
    t, a = -(-rows // 128), -(-blocks // 4)
    out = np.zeros((t * 128, a * 4), np.uint8)
    out[:rows, :blocks] = scales
    return out.reshape(t, 4, 32, a, 4).transpose(0, 3, 2, 1, 4).reshape(-1)


def quantize(z, form):
    """(codes u8 [M, K/2], scale bytes [M, blocks], steps) of transformed rows."""
    f = np.float32
    parts = z.reshape(z.shape[0], -1, BLOCK[form])
    most = np.abs(parts).max(2)
    with np.errstate(all="ignore"):
        if form == "mx":
            scale = np.maximum((most.view(np.uint32) >> 23).astype(np.int64) - 2, 0)
            q = (2.0 ** (127 - scale)).astype(f)
            step = np.ones(z.shape[0], f)
        else:
            step = (most.max(1) * (f(1) / f(2688))).astype(f)
            step = np.where(step >= f(2.0 ** -100), step, f(0))
            inv = np.where(step > 0, f(1) / step, f(0)).astype(f)
            scale = nearest_even((most * inv[:, None]).astype(f) * f(1 / 6), E4M3)
            held = E4M3[scale].astype(f)
            q = np.where(held > 0, inv[:, None] / held, f(0)).astype(f)
        v = (parts * q[:, :, None]).astype(f).reshape(z.shape)
    n = nearest_even(np.abs(v), E2M1) + 8 * np.signbit(v)
    return (n[:, 0::2] + 16 * n[:, 1::2]).astype(np.uint8), scale.astype(np.uint8), step


def integers(z, bits, clip=1.0):
    """(codes u8, steps before the norm) of the integer quantiser behind a norm."""
    f, q = np.float32, 7 if bits == 4 else 127
    step = (f(clip) * np.abs(z).max(1)).astype(f) * (f(1) / f(q))
    step = np.where(step >= f(2.0 ** -126), step, f(0)).astype(f)
    with np.errstate(all="ignore"):
        inv = np.where(step > 0, f(1) / step, f(0)).astype(f)
    n = np.clip(np.rint((z * inv[:, None]).astype(f)), -q, q).astype(np.int64) if clip < 1 else np.rint((z * inv[:, None]).astype(f)).astype(np.int64)
    return ((n[:, 0::2] & 15 | (n[:, 1::2] & 15) << 4) if bits == 4 else n & 255).astype(np.uint8), step


def values(codes, scales, steps, form):
    """What codes stand for, in 64 bits."""
    rows, K = codes.shape[0], 2 * codes.shape[1]
    n = np.stack([codes & 15, codes >> 4], 2).reshape(rows, K)
    v = E2M1[n & 7] * np.where(n & 8, -1.0, 1.0)
    s = 2.0 ** (scales.astype(np.float64) - 127) if form == "mx" else E4M3[scales]
    return (v.reshape(rows, -1, BLOCK[form]) * s[:, :, None]).reshape(rows, K) * steps.astype(np.float64)[:, None]


def tokens(rng, M, K):
    x = rng.standard_normal((M, K)).astype(np.float32)
    x[:, rng.random(K) < 0.02] *= 30
    return x


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(TYPES[dtype])


def host(t):
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def check_status():
    st, word = fq.device_status()
    assert st == fq.OK, hex(word)


# ---------------------------------------------------------------------------- quantiser
@pytest.mark.parametrize("form", ["mx", "nv"])
@pytest.mark.parametrize("M,K,block,dtype", [
    (1, 32, 1, "f32"), (3, 32, 32, "bf16"), (2, 96, 16, "bf16"), (127, 256, 256, "f32"), (128, 160, 8, "bf16"), (129, 512, 64, "bf16"),
    (300, 1120, 32, "f32"), (50, 1024, 64, "bf16"), (5, 2080, 4, "f32"), (33, 4096, 128, "bf16"), (7, 8192, 256, "f32"),
    (4, 8224, 32, "bf16"), (3, 16384, 256, "bf16"), (3, 16384, 2, "f32"), (2, 16416, 32, "bf16"), (2, 32768, 256, "f32"), (1000, 64, 64, "bf16"),
    # batches that stream through shared memory
    (700, 2048, 128, "bf16"), (600, 2048, 256, "f32"), (1301, 1024, 64, "bf16"), (1500, 960, 32, "f32"), (1297, 1088, 16, "bf16"), (300, 5120, 1, "bf16"),
    (301, 5120, 256, "f32"), (297, 8192, 128, "f32"), (296, 16384, 256, "bf16"), (2500, 512, 2, "bf16")])
def test_quantize_bits(form, M, K, block, dtype):
    rng = np.random.default_rng(M * 7 + K)
    x = dev(tokens(rng, M, K), dtype)
    g = np.exp(0.3 * rng.standard_normal(K)).astype(np.float32) * np.float32(block ** -0.5)
    codes, scales, steps = fq.quantize_act_fp4(x, dev(g), block, FORMATS[form])
    c, s, d = quantize(rotate(host(x), g, block), form)
    assert np.array_equal(host(steps), d)
    assert np.array_equal(host(scales), tiles(s))
    assert np.array_equal(host(codes), c)


@pytest.mark.parametrize("form", ["mx", "nv"])
def test_quantize_special_rows(form):
    """Zero rows and blocks, signed zeros, ties, the smallest and largest numbers, steps next to the limit."""
    K = 128
    rng = np.random.default_rng(3)
    x = tokens(rng, 14, K)
    x[0] = 0.0
    x[1] = -0.0
    x[2, 32:64] = 0.0
    x[2, 16:32] *= 1e-6                                          # e4m3's subnormal numbers and below
    x[3] = np.tile([0.25, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, 6.0, -6.0, 0.125, 0.3, 4.0, 4.9999995, 5.0000005, 7.0], 8)
    x[4] *= 1e-38
    x[5] = np.float32(1e-45)
    x[6] *= 1e36
    x[7] = 0.0
    x[7, 5] = 3.4e38
    x[8] = rng.choice([2.0 ** -100 * 2688, 2.0 ** -101 * 2688], K)
    x[9] = 2.0 ** -101 * 2688
    x[10, ::2] = -0.0
    x[11] = 6.0 * 448
    x[12] = np.float32(2.0 ** -126) * rng.integers(0, 8, K)
    for mult in (None, np.ones(K, np.float32)):
        codes, scales, steps = fq.quantize_act_fp4(dev(x), None if mult is None else dev(mult), 1, FORMATS[form])
        c, s, d = quantize(rotate(x, np.ones(K, np.float32), 1), form)
        assert np.array_equal(host(steps), d)
        assert np.array_equal(host(scales), tiles(s))
        assert np.array_equal(host(codes), c)


@pytest.mark.parametrize("M,K", [(70, 224), (1300, 1024), (400, 4160)])
@pytest.mark.parametrize("form", ["mx", "nv"])
def test_quantize_strides_and_bounds(form, M, K):
    """Rows inside a wider matrix, outputs inside wider memory: nothing else is written, every place of the scales is."""
    wide = dev(tokens(np.random.default_rng(1), M, K + 40))
    x = wide[:, 16:16 + K]
    sb = fq.fp4_scale_bytes(M, K, FORMATS[form])
    code_mem, scale_mem, step_mem = torch.full((M * K // 2 + 64,), 77, dtype=torch.uint8, device="cuda"), torch.full((sb + 64,), 77, dtype=torch.uint8, device="cuda"), torch.full((M + 2,), 77.0, device="cuda")
    codes, scales, steps = code_mem[32:-32].view(M, K // 2), scale_mem[32:-32], step_mem[1:-1]
    fq.quantize_act_fp4(x, None, 32, FORMATS[form], codes, scales, steps)
    c, s, d = quantize(rotate(host(x), np.full(K, np.float32(32 ** -0.5)), 32), form)
    assert np.array_equal(host(codes), c) and np.array_equal(host(scales), tiles(s)) and np.array_equal(host(steps), d)
    for m in (code_mem[:32], code_mem[-32:], scale_mem[:32], scale_mem[-32:], step_mem[:1], step_mem[-1:]):
        assert bool((m == 77).all())


# ---------------------------------------------------------------------------- handles
@pytest.mark.parametrize("form", ["mx", "nv"])
def test_fold_export_import(form):
    rng = np.random.default_rng(5)
    N, K, block = 136, 320, 64
    W, smooth, bias = rng.standard_normal((N, K)).astype(np.float32), np.exp(rng.standard_normal(K)).astype(np.float32), rng.standard_normal(N).astype(np.float32)
    h = fq.fold_weights_fp4(dev(W), dev(smooth), dev(bias), block, FORMATS[form])
    assert (h.N, h.K, h.block, h.format) == (N, K, block, FORMATS[form])
    codes, scales, ws, g, b = h.export()
    cn = np.float32(1 / np.sqrt(block))
    c, s, d = quantize(rotate(W, smooth * cn, block), form)
    assert np.array_equal(host(codes), c) and np.array_equal(host(scales), tiles(s)) and np.array_equal(host(ws), d)
    assert np.array_equal(host(g), (np.float32(1) / smooth) * cn) and np.array_equal(host(b), bias)
    dirty = scales.view(-1, scales.numel() // 512 // 2, 32, 4, 4).clone() if form == "nv" else scales.clone()
    again = fq.weights_import_fp4(codes, dirty.view(-1), ws, g, b, K, block, FORMATS[form])
    for x, y in zip(again.export(), (codes, scales, ws, g, b)):
        assert torch.equal(x, y)
    plain = fq.weights_import_fp4(codes, scales, None, None, None, K, block, FORMATS[form]).export()
    assert bool((plain[2] == 1).all()) and bool((plain[3] == float(cn)).all()) and bool((plain[4] == 0).all())


@pytest.mark.parametrize("form", ["mx", "nv"])
def test_import_clears_unused_places(form):
    """Scales of a checkpoint whose unused places hold NaN: products do not see them."""
    N, K, M = 72, 96, 9
    rng = np.random.default_rng(8)
    c, s, d = quantize(tokens(rng, N, K), form)
    flat = tiles(s)
    used = tiles(np.ones_like(s)) == 1
    dirty = np.where(used, flat, 255).astype(np.uint8)
    h = fq.weights_import_fp4(dev(c), dev(dirty), dev(d), None, None, K, 1, FORMATS[form])
    assert np.array_equal(host(h.export()[1]), flat)
    a = fq.quantize_act_fp4(dev(tokens(rng, M, K)), None, 1, FORMATS[form])
    y = fq.gemm_fp4(*a, h)
    assert bool(torch.isfinite(y).all())


# ---------------------------------------------------------------------------- product
def product_case(form, M, N, K, seed=0, bias=True):
    rng = np.random.default_rng(seed + M + 3 * N + 5 * K)
    ac, as_, ad = quantize(tokens(rng, M, K), form)
    wc, ws, wd = quantize(0.02 * rng.standard_normal((N, K)).astype(np.float32), form)
    if form == "mx":
        ad = rng.uniform(0.5, 2, M).astype(np.float32)
        wd = rng.uniform(0.5, 2, N).astype(np.float32)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    handle = fq.weights_import_fp4(dev(wc), dev(tiles(ws)), dev(wd), None, None if b is None else dev(b), K, 1, FORMATS[form])
    A, W = dev(values(ac, as_, ad, form)), dev(values(wc, ws, wd, form))
    want = A @ W.T + (0.0 if b is None else dev(b).double())
    size = A.abs() @ W.abs().T + (0.0 if b is None else dev(b).double().abs())
    return (dev(ac), dev(tiles(as_)), dev(ad)), handle, want, size


def assert_product(y, want, size, K):
    """Each of K/16 partial sums is rounded or cut once in binary32 (2^-23 of what has been added up so far, at most the sum of
    magnitudes), then factor, product and sum of the epilogue, then half a step of the output."""
    bound = (K / 16 + 8) * 2.0 ** -23 * size + (2.0 ** -8 * want.abs() if y.dtype == torch.bfloat16 else 0.0)
    off = (y.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [
    (1, 8, 32), (1, 128, 64), (1, 2560, 2048), (2, 136, 96), (16, 128, 256), (17, 264, 288), (50, 1024, 1024), (64, 256, 512), (100, 512, 16384),
    (128, 128, 128), (129, 384, 320), (200, 2048, 8192), (255, 1000, 1120), (256, 256, 256), (257, 512, 544), (333, 1000, 1120), (300, 4104, 192),
    (816, 2048, 2048), (513, 10000, 352), (2100, 2600, 1056), (816, 1024, 8192), (130, 512, 32768), (3, 264, 32736)])
def test_product(form, M, N, K, dtype):
    a, handle, want, size = product_case(form, M, N, K)
    y = fq.gemm_fp4(*a, handle, TYPES[dtype])
    check_status()
    assert_product(y, want, size, K)


@pytest.mark.parametrize("seed", range(24))
def test_product_sizes_at_random(seed):
    """Whatever tiles, slices of K and pairs the sizes lead to."""
    import random
    rng = random.Random(seed)
    form = rng.choice(["mx", "nv"])
    K = 32 * max(1, int(2 ** rng.uniform(0, 9)))
    N = 8 * max(1, int(2 ** rng.uniform(0, min(9, 22 - np.log2(K)))))
    M = max(1, int(2 ** rng.uniform(0, min(11, 22 - np.log2(K)))))
    a, handle, want, size = product_case(form, M, N, K, seed)
    dtype = rng.choice(["f32", "bf16"])
    y = fq.gemm_fp4(*a, handle, TYPES[dtype])
    assert_product(y, want, size, K)
    assert torch.equal(fq.gemm_fp4(*a, handle, TYPES[dtype]), y)
    check_status()


def test_product_is_reproducible_and_each_row_its_own():
    """The same bits again, and a row does not depend on the batch around it where the plan is the same."""
    a, handle, want, size = product_case("nv", 60, 1024, 4096)
    y = fq.gemm_fp4(*a, handle)
    for _ in range(3):
        assert torch.equal(fq.gemm_fp4(*a, handle), y)
    codes = a[0].clone()
    codes[5] = 0x77
    other = fq.gemm_fp4(codes, a[1], a[2], handle)
    keep = torch.arange(60, device="cuda") != 5
    assert torch.equal(other[keep], y[keep]) and not torch.equal(other[5], y[5])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 72, 64), (50, 264, 512), (300, 520, 256), (700, 9480, 96)])
def test_product_writes_only_its_rows(M, N, K, dtype):
    a, handle, want, size = product_case("nv", M, N, K, bias=False)
    mem = torch.full((M + 2, N + 24), 3.5, dtype=TYPES[dtype], device="cuda")
    y = mem[1:-1, 8:8 + N]
    assert fq.gemm_fp4(*a, handle, y=y).data_ptr() == y.data_ptr()
    assert_product(y.clone(), want, size, K)
    mem[1:-1, 8:8 + N] = 3.5
    assert bool((mem == 3.5).all())


@pytest.mark.parametrize("form", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(513, 10000, 352), (2100, 2600, 1056), (816, 32776, 2048), (700, 9480, 96)])
def test_product_keeps_outputs_on_their_way(form, M, N, K):
    """Several tiles to a CTA, the last of them partly past N: what a warp has handed to the copy engine stays until it is read.
    Many launches one behind the other, each bit for bit the binary32 outputs rounded once (the same sums in the same order)."""
    a, handle, _, _ = product_case(form, M, N, K)
    want = fq.gemm_fp4(*a, handle).to(torch.bfloat16)
    for _ in range(4):
        got = [fq.gemm_fp4(*a, handle, torch.bfloat16) for _ in range(12)]
        for y in got:
            assert torch.equal(y, want)
    check_status()


def test_product_scales_past_the_last_row_do_not_matter():
    for form in ("mx", "nv"):
        a, handle, want, size = product_case(form, 37, 256, 512)
        scales = a[1].view(-1, 32, 4, 4).clone()
        rows = torch.arange(4, device="cuda")[None, :] * 32 + torch.arange(32, device="cuda")[:, None]
        scales[:, rows >= 37] = 255
        assert torch.equal(fq.gemm_fp4(a[0], scales.view(-1), a[2], handle), fq.gemm_fp4(*a, handle))


def test_product_slices_of_steps():
    """Steps may begin on any element."""
    a, handle, want, size = product_case("nv", 21, 128, 128)
    longer = torch.cat([a[2].new_zeros(3), a[2]])
    assert torch.equal(fq.gemm_fp4(a[0], a[1], longer[3:], handle), fq.gemm_fp4(*a, handle))


def test_product_large_and_small_scales():
    """e8m0 from 2^-120 to 2^120 in one product: magnitudes cancel in the accumulator exactly."""
    M, N, K = 8, 128, 64
    codes = torch.full((M, K // 2), 0x22, dtype=torch.uint8, device="cuda")            # ones
    wcodes = torch.full((N, K // 2), 0x22, dtype=torch.uint8, device="cuda")
    for ea, ew in ((7, 247), (247, 7), (127, 127), (67, 127)):
        h = fq.weights_import_fp4(wcodes, dev(tiles(np.full((N, 2), ew))), None, None, None, K, 1, fq.MXFP4)
        y = fq.gemm_fp4(codes, dev(tiles(np.full((M, 2), ea))), torch.ones(M, device="cuda"), h)
        assert bool((y == K * 2.0 ** (ea + ew - 254)).all())


# ---------------------------------------------------------------------------- both in one call
@pytest.mark.parametrize("form", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K,block,dtype", [(1, 256, 128, 64, "bf16"), (50, 1024, 1024, 64, "bf16"), (130, 264, 160, 32, "f32"), (816, 512, 2048, 128, "bf16"),
                                               (3, 128, 16384, 256, "f32")])
def test_linear_is_quantizer_and_product(form, M, N, K, block, dtype):
    rng = np.random.default_rng(M + K)
    x = dev(tokens(rng, M, K), dtype)
    W, smooth, bias = (dev(rng.standard_normal(s).astype(np.float32)) for s in ((N, K), K, N))
    for sm in (smooth.exp(), None):
        h = fq.fold_weights_fp4(W, sm, bias, block, FORMATS[form])
        for out in (torch.float32, torch.bfloat16):
            y = fq.linear_fp4(x, h, out)
            assert torch.equal(y, fq.gemm_fp4(*fq.quantize_act_fp4(x, h, block, FORMATS[form]), h, out))
    # against the float projection: W x is kept by the fold, and each operand's code is off by at most a quarter of its value or half
    # of the smallest distance (0.25 of 6) of its block's largest: one sixth of that at most, so the rounding's part stays a fraction
    ref = x.double() @ W.double().T + bias.double()
    err = (fq.linear_fp4(x, h).double() - ref).norm() / ref.norm()
    assert float(err) < 0.3
    check_status()


# ---------------------------------------------------------------------------- norm
def norm_reference(x, residual, dtype):
    t = TYPES[dtype]
    h = x if residual is None else (x.double() + residual.double()).to(torch.float32).to(t)
    return h


@pytest.mark.parametrize("form", ["int8", "int4", "mx", "nv"])
@pytest.mark.parametrize("M,K,block,dtype,residual", [
    (1, 32, 1, "f32", True), (50, 1024, 64, "bf16", True), (129, 96, 32, "bf16", False), (5, 2048, 1, "bf16", True), (33, 5120, 256, "f32", True),
    (3, 8192, 128, "bf16", True), (4, 8224, 8, "f32", True), (3, 16384, 256, "bf16", False), (2, 16416, 32, "f32", True), (2, 32768, 256, "bf16", True),
    (700, 64, 16, "f32", False),
    # batches that stream through shared memory
    (700, 2048, 128, "bf16", True), (601, 2048, 256, "f32", True), (1301, 1024, 1, "bf16", True), (1500, 960, 32, "f32", False), (1297, 1088, 16, "bf16", False),
    (301, 5120, 256, "f32", True), (297, 8192, 64, "f32", True), (300, 16384, 256, "bf16", True), (299, 5120, 1, "bf16", True)])
def test_norm(form, M, K, block, dtype, residual):
    rng = np.random.default_rng(M + K)
    x = dev(tokens(rng, M, K), dtype)
    r = dev(tokens(rng, M, K), dtype) if residual else None
    g = dev(np.exp(0.3 * rng.standard_normal(K)).astype(np.float32) * np.float32(block ** -0.5))
    eps = 1e-5
    h = x if r is None else (x.double() + r.double()).to(TYPES[dtype])       # (exact in 64 bits, rounded once)
    if form in FORMATS:
        got, codes, scales, steps = fq.rmsnorm_quantize_act_fp4(x, r, g, block, FORMATS[form], eps)
        c, s, d = fq.quantize_act_fp4(h, g, block, FORMATS[form])
        assert torch.equal(scales, s)
    else:
        bits = 8 if form == "int8" else 4
        got, codes, steps = fq.rmsnorm_quantize_act(x, r, g, block, bits, eps)
        c, d = (dev(a) for a in integers(rotate(host(h), host(g), block), bits))
    assert torch.equal(got, h) and (r is not None or got.data_ptr() == x.data_ptr())
    assert torch.equal(codes, c)
    want = d.double() / (h.double().square().mean(1) + eps).sqrt()
    # the squares' sum through at most 32 + 10 roundings (half of that behind the root), then five operations
    assert bool(((steps.double() - want).abs() <= 27 * 2.0 ** -24 * want).all())


@pytest.mark.parametrize("M,K", [(90, 288), (1400, 1024), (310, 8192)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_in_place_and_strided(dtype, M, K):
    rng = np.random.default_rng(2)
    x, r = dev(tokens(rng, M, K), dtype), dev(tokens(rng, M, K), dtype)
    h, codes, steps = fq.rmsnorm_quantize_act(x, r, None, 32, 8)
    for target in ("x", "r"):
        a, b = x.clone(), r.clone()
        out = fq.rmsnorm_quantize_act(a, b, None, 32, 8, h=a if target == "x" else b)
        assert out[0].data_ptr() == (a if target == "x" else b).data_ptr()
        assert torch.equal(out[0], h) and torch.equal(out[1], codes) and torch.equal(out[2], steps)
        assert torch.equal(b if target == "x" else a, r if target == "x" else x)
    wide = [torch.full((M + 2, K + 16), 9.0, dtype=TYPES[dtype], device="cuda") for _ in range(3)]
    va, vb, vh = (w[1:-1, 8:8 + K] for w in wide)
    va.copy_(x)
    vb.copy_(r)
    out = fq.rmsnorm_quantize_act(va, vb, None, 32, 8, h=vh)
    assert torch.equal(out[0], h) and torch.equal(out[1], codes) and torch.equal(out[2], steps)
    vh.fill_(9.0)
    assert bool((wide[2] == 9.0).all())


@pytest.mark.parametrize("K,repeat", [(96, 1), (4096, 1), (16416, 1), (4096, 60), (1024, 250)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("form", ["int8", "mx", "nv"])
def test_norm_extremes(form, K, repeat, residual):
    """Rows whose squares leave binary32, zero rows with and without eps, in short batches and in ones that stream."""
    rng = np.random.default_rng(4)
    base = np.tile(rng.standard_normal((6, K)).astype(np.float32), (repeat, 1))
    scale = np.tile(np.array([1e25, 1e-25, 0.0, 1.0, 1e19, 1e-19], np.float32), repeat)[:, None]
    x = dev(base * scale)
    zero = torch.zeros_like(x) if residual else None
    for eps in (0.0, 1e-6):
        out = fq.rmsnorm_quantize_act(x, zero, None, 1, 8, eps) if form == "int8" else fq.rmsnorm_quantize_act_fp4(x, zero, None, 1, FORMATS[form], eps)
        d = (fq.quantize_act(x, None, 1, 8) if form == "int8" else fq.quantize_act_fp4(x, None, 1, FORMATS[form]))[-1]
        rms = (x.double().square().mean(1) + eps).sqrt()
        want = torch.where(d > 0, d.double() / rms, 0.0)
        got = out[-1].double()
        assert bool(torch.isfinite(got).all())
        live = torch.tensor([i for i in range(6 * repeat) if i % 6 != 2], device="cuda")
        # (a result below binary32's normal numbers keeps a half of 2^-149)
        assert bool(((got - want)[live].abs() <= 27 * 2.0 ** -24 * want[live] + 2.0 ** -149).all())
        if form != "mx":
            assert bool((got[2::6] == 0.0).all())


# batches whose rows end in half a 128-byte line (bf16), have more than 256 lines, or both
ODD_ROWS = [(2100, 672, 32, "bf16"), (1300, 1056, 16, "bf16"), (800, 2080, 8, "bf16"), (600, 8224, 32, "bf16"), (330, 16416, 32, "bf16"), (297, 11296, 1, "bf16"),
            (298, 8224, 32, "f32"), (300, 16384, 256, "f32"), (299, 11296, 2, "f32"), (300, 16448, 64, "bf16"), (296, 32768, 256, "bf16")]


@pytest.mark.parametrize("form", ["mx", "nv"])
@pytest.mark.parametrize("M,K,block,dtype", ODD_ROWS)
def test_quantize_odd_rows(form, M, K, block, dtype):
    test_quantize_bits(form, M, K, block, dtype)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("form", ["int8", "int4", "mx", "nv"])
@pytest.mark.parametrize("M,K,block,dtype", ODD_ROWS)
def test_norm_odd_rows(form, M, K, block, dtype, residual):
    test_norm(form, M, K, block, dtype, residual)


@pytest.mark.parametrize("M,K,dtype", [(1400, 1056, "bf16"), (700, 4128, "bf16"), (300, 16416, "bf16"), (300, 11296, "f32")])
def test_norm_odd_rows_in_place_and_strided(M, K, dtype):
    test_norm_in_place_and_strided(dtype, M, K)


@pytest.mark.parametrize("form", ["int8", "nv"])
@pytest.mark.parametrize("K,repeat", [(1056, 250), (8224, 55)])
def test_norm_extremes_of_odd_rows(form, K, repeat):
    """Rows of bf16 whose squares leave binary32, whose last half line counts as the others do."""
    rng = np.random.default_rng(8)
    base = np.tile(rng.standard_normal((6, K)).astype(np.float32), (repeat, 1))
    base[:, -32:] *= 4.0
    scale = np.tile(np.array([1e25, 1e-25, 0.0, 1.0, 1e19, 1e-19], np.float32), repeat)[:, None]
    x = dev(base * scale, "bf16")
    out = fq.rmsnorm_quantize_act(x, torch.zeros_like(x), None, 1, 8, 0.0) if form == "int8" else fq.rmsnorm_quantize_act_fp4(x, torch.zeros_like(x), None, 1, FORMATS[form], 0.0)
    d = (fq.quantize_act(x, None, 1, 8) if form == "int8" else fq.quantize_act_fp4(x, None, 1, FORMATS[form]))[-1]
    live = torch.tensor([i for i in range(6 * repeat) if i % 6 != 2], device="cuda")
    want = (d.double() / x.double().square().mean(1).sqrt())[live]
    assert bool(((out[-1].double()[live] - want).abs() <= 27 * 2.0 ** -24 * want + 2.0 ** -149).all())
    assert bool((out[-1][2::6] == 0.0).all())


def test_norm_clip():
    x = dev(tokens(np.random.default_rng(6), 40, 512), "bf16")
    g = torch.ones(512, device="cuda")
    for bits in (4, 8):
        h, codes, steps = fq.rmsnorm_quantize_act(x, None, g, 1, bits, 0.0, clip_ratio=0.7)
        c, d = (dev(a) for a in integers(host(x), bits, 0.7))
        assert torch.equal(codes, c)
        want = d.double() / x.double().square().mean(1).sqrt()
        assert bool(((steps.double() - want).abs() <= 27 * 2.0 ** -24 * want).all())


def next_to_ties(rng, rows, K, bits, clip):
    """Rows of binary32 whose quotient z * (1/d), rounded to binary32, lies half way between two integers and unrounded beside it: the
    product's own rounding decides the code.  (Multiplied and rounded to an integer in one operation, they would go the other way.)"""
    f, q = np.float32, 7 if bits == 4 else 127
    x = np.zeros((rows, K), f)
    for r in range(rows):
        while True:
            m = f(rng.uniform(0.5, 4.0))
            d = (f(clip) * m) * (f(1) / f(q))
            inv = f(1) / d
            k = np.arange(q)
            z = ((k + 0.5) * np.float64(d)).astype(f)
            near = (z.view(np.int32)[:, None] + np.arange(-3, 4)[None]).view(f)
            exact = near.astype(np.float64) * np.float64(inv)         # (48 bits)
            fits = ((near * inv).astype(f) == (k + 0.5).astype(f)[:, None]) & (np.rint(exact) != np.rint(k + 0.5)[:, None]) & (near < m)
            if fits.any():
                break
        x[r] = rng.choice(near[fits], K) * rng.choice(np.array([-1, 1], f), K)
        x[r, rng.integers(K)] = m
    return x


@pytest.mark.parametrize("clip", [1.0, 0.75])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("K", [64, 4096, 8224, 16416])
def test_norm_rounds_the_quotient_and_then_the_code(K, bits, clip):
    """The same rows in a short batch and in one that streams: two operations, each rounded, in every kernel."""
    x = next_to_ties(np.random.default_rng(K + bits), 8, K, bits, clip)
    want, _ = integers(x, bits, clip)
    for repeat in (1, max(40, 160000 // K)):
        codes = fq.rmsnorm_quantize_act(dev(np.tile(x, (repeat, 1))), None, torch.ones(K, device="cuda"), 1, bits, clip_ratio=clip)[1]
        assert np.array_equal(host(codes), np.tile(want, (repeat, 1)))


STEP_ROWS = [(1024, "f32"), (1024, "bf16"), (8224, "bf16"), (16416, "f32")]     # short batches of all; the first three stream too


@pytest.mark.parametrize("repeat", [1, 240])
@pytest.mark.parametrize("K,dtype", STEP_ROWS)
@pytest.mark.parametrize("form", ["int8", "int4", "mx", "nv"])
def test_norm_steps_of_the_smallest_and_largest_rows(form, K, dtype, repeat):
    """Subnormal rows and rows at the end of binary32, without eps: d / rms, in 64 bits, rounded once (a half of 2^-149 where it ends
    below the normal numbers).  For MXFP4 a 1 / rms that binary32 does not have is a step of 0."""
    rng = np.random.default_rng(K)
    base = rng.uniform(0.5, 1.0, (8, K)).astype(np.float32) * rng.choice(np.array([-1, 1], np.float32), (8, K))
    base[7, 1:] = 0.0                                            # a single number
    scale = np.array([1e-40, 3e-44, 1e-38, 1e-30, 1e-20, 1e-41, 3e38, 1e37], np.float32)[:, None]
    for gain in (1.0, 2.0 ** 20, 2.0 ** -20):                    # (large: rows below the smallest step without it have one)
        eight = dev(base * np.where(scale > 1, scale / max(gain, 1.0), scale).astype(np.float32), dtype)
        x, g = eight.repeat(repeat, 1), torch.full((K,), gain, device="cuda")
        z = rotate(host(eight), host(g), 1)
        if form in FORMATS:
            got = fq.rmsnorm_quantize_act_fp4(x, None, g, 1, FORMATS[form], 0.0)[-1]
            d = quantize(z, form)[2]
        else:
            bits = 8 if form == "int8" else 4
            got = fq.rmsnorm_quantize_act(x, None, g, 1, bits, 0.0)[-1]
            d = integers(z, bits)[1]
        rms = np.sqrt(np.square(host(eight).astype(np.float64)).mean(1))
        want = d.astype(np.float64) / np.where(rms > 0, rms, np.inf)         # (bf16 does not have the smallest: rows of zeros, steps of 0)
        if form == "mx":
            want = np.where(want > float(np.finfo(np.float32).max), 0.0, want)
        want = np.tile(want, repeat)
        got = host(got).astype(np.float64)
        assert np.isfinite(got).all()
        # (rows in binary32's range: the sum of squares, its mean, root, reciprocal and product, as in the test of the norm)
        assert (np.abs(got - want) <= 27 * 2.0 ** -24 * want + 2.0 ** -149).all()
        if form in FORMATS:
            ones = torch.full((8, K // 2), 0x22, dtype=torch.uint8, device="cuda")
            scales = torch.full((fq.fp4_scale_bytes(8, K, FORMATS[form]),), 127 if form == "mx" else 56, dtype=torch.uint8, device="cuda")
            h = fq.weights_import_fp4(ones, scales, None, None, None, K, 1, FORMATS[form])
            y = fq.gemm_fp4(*fq.rmsnorm_quantize_act_fp4(x[:6], None, g, 1, FORMATS[form], 0.0)[1:], h)
            assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("repeat", [1, 240])
@pytest.mark.parametrize("K,dtype", STEP_ROWS)
@pytest.mark.parametrize("form", ["int8", "int4", "mx", "nv"])
def test_norm_steps_of_rows_that_are_not_finite(form, K, dtype, repeat, residual):
    """Such a row's step is NaN; the others' are as they were."""
    rng = np.random.default_rng(K + 1)
    a = np.tile(rng.standard_normal((6, K)).astype(np.float32), (repeat, 1))
    b = a.copy()
    b[0::6, K - 1] = np.nan
    b[2::6, 0] = np.inf
    b[4::6, K // 2] = -np.inf
    b[4::6, 3] = np.nan
    g = np.ones(K, np.float32)
    g[0] = 0.0
    for eps in (0.0, 1e-6):
        steps = []
        for rows in (a, b):
            x = dev(rows, dtype)
            r = torch.zeros_like(x) if residual else None
            out = fq.rmsnorm_quantize_act_fp4(x, r, dev(g), 1, FORMATS[form], eps) if form in FORMATS else fq.rmsnorm_quantize_act(x, r, dev(g), 1, 8 if form == "int8" else 4, eps)
            steps.append(out[-1])
        assert bool(torch.isfinite(steps[0]).all())
        assert torch.equal(steps[0][1::2], steps[1][1::2]) and bool(steps[1][0::2].isnan().all())


# ---------------------------------------------------------------------------- as they are used together
def test_a_layers_projections():
    """Residual and norm, 8-bit qkv; residual and norm, e2m1 gate/up and down: against the same layer from the plain calls."""
    M, K, F, block = 77, 512, 1024, 64
    rng = np.random.default_rng(9)
    t = lambda *s: dev(rng.standard_normal(s).astype(np.float32))
    x, r = t(M, K).to(torch.bfloat16), t(M, K).to(torch.bfloat16)
    qkv = fq.fold_weights(t(3 * K, K) * 0.05, t(K).exp(), None, block, 8)
    up, down = fq.fold_weights_fp4(t(F, K) * 0.05, t(K).exp(), t(F), block), fq.fold_weights_fp4(t(K, F) * 0.05, None, None, block, fq.MXFP4)
    h, codes, steps = fq.rmsnorm_quantize_act(x, r, qkv, block, 8)
    y = fq.gemm_w8a8(codes, steps, qkv, torch.bfloat16)
    hd = (x.double() + r.double()).to(torch.bfloat16)
    n = hd.double() / (hd.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    want = fq.linear_w8a8(n.float(), qkv, out_dtype=torch.float32).double()
    # (a code may differ where the plain call divides before it rounds: one step of 1/127 of the row's largest in few channels)
    assert float((y.double() - want).norm() / want.norm()) < 2.0 ** -8 + 1e-3
    h2, c2, s2, d2 = fq.rmsnorm_quantize_act_fp4(h, y[:, :K].contiguous(), up, block)
    z = fq.gemm_fp4(c2, s2, d2, up, torch.bfloat16)
    out = fq.linear_fp4(torch.nn.functional.silu(z), down, torch.bfloat16)
    n2 = h2.double() / (h2.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    z2 = fq.linear_fp4(n2.float(), up)
    # (the same argument with e2m1's steps: a quarter of a value, in few channels)
    assert float((z.double() - z2.double()).norm() / z2.double().norm()) < 2.0 ** -8 + 1e-2
    assert out.shape == (M, K) and bool(torch.isfinite(out).all())
    check_status()


def test_streams_and_graphs():
    """Calls on two streams at once, with a shared handle, and a captured run replayed on new inputs."""
    M, N, K, block = 64, 1024, 1024, 64
    rng = np.random.default_rng(11)
    W = dev(rng.standard_normal((N, K)).astype(np.float32))
    h = fq.fold_weights_fp4(W, None, None, block)
    xs = [dev(tokens(rng, M, K), "bf16") for _ in range(4)]
    want = [fq.linear_fp4(x, h) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None] * 4
    for rep in range(5):
        for i, x in enumerate(xs):
            with torch.cuda.stream(streams[i % 2]):
                got[i] = fq.linear_fp4(x, h)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    static, res = xs[0].clone(), xs[1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hh, c, s, d = fq.rmsnorm_quantize_act_fp4(static, res, h, block)
        y = fq.gemm_fp4(c, s, d, h)
        z = fq.linear_fp4(static, h)
    for a, b in ((xs[2], xs[3]), (xs[1], xs[0])):
        static.copy_(a)
        res.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        e = fq.rmsnorm_quantize_act_fp4(a, b, h, block)
        assert torch.equal(hh, e[0]) and torch.equal(y, fq.gemm_fp4(*e[1:], h)) and torch.equal(z, fq.linear_fp4(a, h))
    check_status()


def test_first_call_inside_a_capture():
    """A process whose first calls are captured: every set-up that a launch needs is allowed there."""
    import subprocess
    import sys
    code = """
import torch
from paper_2609_24433_b200 import fq
M, K, N = 640, 2048, 2560
h = fq.fold_weights_fp4(torch.randn(N, K, device="cuda"), None, None, 64)
x, r = (torch.randn(M, K, device="cuda").bfloat16() for _ in range(2))
short = x[:3].clone()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    n = fq.rmsnorm_quantize_act_fp4(x, r, h, 64)
    y = fq.gemm_fp4(*n[1:], h, torch.bfloat16)
    z = fq.linear_fp4(short, h)
    w = fq.linear_fp4(x[:200], h)
for _ in range(2):
    g.replay()
torch.cuda.synchronize()
n2 = fq.rmsnorm_quantize_act_fp4(x, r, h, 64)
assert all(torch.equal(a, b) for a, b in zip(n, n2))
assert torch.equal(y, fq.gemm_fp4(*n2[1:], h, torch.bfloat16)) and torch.equal(z, fq.linear_fp4(short, h)) and torch.equal(w, fq.linear_fp4(x[:200], h))
assert fq.device_status()[0] == fq.OK
print("captured")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]


def test_two_threads():
    """Calls from two Python threads on streams of their own, one handle."""
    import threading
    M, N, K, block = 300, 1024, 2048, 128
    rng = np.random.default_rng(12)
    h = fq.fold_weights_fp4(dev(rng.standard_normal((N, K)).astype(np.float32)), None, None, block, fq.MXFP4)
    xs = [dev(tokens(rng, M, K), "bf16") for _ in range(2)]
    want = [fq.linear_fp4(x, h) for x in xs]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(30):
                y = fq.linear_fp4(xs[i], h)
                torch.cuda.current_stream().synchronize()
                if not torch.equal(y, want[i]):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    check_status()


def test_empty_and_shapes():
    h = fq.fold_weights_fp4(torch.randn(16, 64, device="cuda"), None, None, 1)
    empty = torch.empty(0, 64, device="cuda")
    assert fq.linear_fp4(empty, h).shape == (0, 16)
    c, s, d = fq.quantize_act_fp4(empty, None, 1)
    assert c.shape == (0, 32) and s.numel() == 0 and d.numel() == 0 and fq.gemm_fp4(c, s, d, h).shape == (0, 16)
    assert fq.rmsnorm_quantize_act(empty, empty, None, 1, 8)[1].shape == (0, 64)
    none = fq.fold_weights_fp4(torch.empty(0, 64, device="cuda"), None, None, 1)
    assert fq.linear_fp4(torch.randn(3, 64, device="cuda"), none).shape == (3, 0)


def test_refusals():
    h = fq.fold_weights_fp4(torch.randn(16, 64, device="cuda"), None, None, 1)
    x = torch.randn(4, 64, device="cuda")
    c, s, d = fq.quantize_act_fp4(x, None, 1)
    for bad in (lambda: fq.linear_fp4(x[:, :32], h), lambda: fq.linear_fp4(x.cpu(), h), lambda: fq.gemm_fp4(c, s[:-1], d, h),
                lambda: fq.gemm_fp4(c.view(torch.int8), s, d, h), lambda: fq.gemm_fp4(c, s, d[:3], h), lambda: fq.gemm_fp4(c, s, d, h, y=torch.empty(3, 16, device="cuda")),
                lambda: fq.quantize_act_fp4(x, torch.ones(63, device="cuda"), 1), lambda: fq.quantize_act_fp4(x, None, 1, codes=c[:3]),
                lambda: fq.rmsnorm_quantize_act(x, x[:3], None, 1, 8), lambda: fq.rmsnorm_quantize_act(x, x.to(torch.bfloat16), None, 1, 8),
                lambda: fq.rmsnorm_quantize_act(x, None, None, 1, 8, h=x), lambda: fq.quantize_act_fp4(x, h if False else torch.ones(64), 1)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: fq.quantize_act_fp4(x, None, 3), fq.ERR_UNSUPPORTED), (lambda: fq.quantize_act_fp4(x, None, 1, 2), fq.ERR_INVALID_ARG),
                        (lambda: fq.rmsnorm_quantize_act(x, None, None, 1, 7), fq.ERR_INVALID_ARG), (lambda: fq.rmsnorm_quantize_act(x, None, None, 1, 8, -1.0), fq.ERR_INVALID_ARG),
                        (lambda: fq.linear_fp4(x, h, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), fq.ERR_NOMEM)):
        with pytest.raises(fq.FqError) as e:
            bad()
        assert e.value.status == status
    h.destroy()
    with pytest.raises(RuntimeError):
        fq.linear_fp4(x, h)


def test_multiplier_of_a_handle_goes_with_its_block():
    """A handle's multiplier carries its block's norm: calls with another block are refused."""
    x = torch.randn(4, 128, device="cuda")
    for h in (fq.fold_weights_fp4(torch.randn(16, 128, device="cuda"), None, None, 64), fq.fold_weights(torch.randn(16, 128, device="cuda"), None, None, 64, 8)):
        for call in (lambda block: fq.quantize_act_fp4(x, h, block), lambda block: fq.rmsnorm_quantize_act(x, None, h, block, 8),
                     lambda block: fq.rmsnorm_quantize_act_fp4(x, None, h, block)):
            call(64)
            for block in (1, 32, 128):
                with pytest.raises(ValueError):
                    call(block)


def test_parameters_are_tensors():
    """Multiplier, rows and outputs that a module holds as torch.nn.Parameter."""
    K = 256
    x, g = torch.randn(5, K, device="cuda"), torch.rand(K, device="cuda") + 0.5
    P = lambda t: torch.nn.Parameter(t)
    for a, b in zip(fq.quantize_act_fp4(P(x), P(g), 64), fq.quantize_act_fp4(x, g, 64)):
        assert torch.equal(a, b)
    for a, b in zip(fq.rmsnorm_quantize_act(P(x), P(x), P(g), 64, 8), fq.rmsnorm_quantize_act(x, x, g, 64, 8)):
        assert torch.equal(a, b)
    h = fq.fold_weights_fp4(P(torch.ones(16, K, device="cuda")), P(g), P(torch.zeros(16, device="cuda")), 64)
    assert torch.equal(fq.linear_fp4(P(x), h), fq.linear_fp4(x, h))


@pytest.mark.parametrize("M,K,F,block", [(77, 512, 1024, 64), (1, 512, 1024, 64), (300, 1056, 2080, 32)])
def test_a_layers_mlp_against_its_codes(M, K, F, block):
    """Residual and norm into NVFP4 gate/up, its activation into MXFP4 down, each product against 64 bits from the codes it was given."""
    rng = np.random.default_rng(M + F)
    t = lambda *s: dev(rng.standard_normal(s).astype(np.float32))
    up = fq.fold_weights_fp4(t(2 * F, K) * 0.05, t(K).exp(), t(2 * F), block)
    down = fq.fold_weights_fp4(t(K, F) * 0.05, t(F).exp(), t(K), block, fq.MXFP4)

    def product(a, handle, form):
        codes, scales, ws, _, bias = (host(v) for v in handle.export())
        def plain(c, sc, d, rows):
            blocks = handle.K // BLOCK[form]
            flat = sc.reshape(-(-rows // 128), -(-blocks // 4), 32, 4, 4).transpose(0, 3, 2, 1, 4).reshape(-1, -(-blocks // 4) * 4)
            return dev(values(c, flat[:rows, :blocks], d, form))
        A, W = plain(*(host(v) for v in a), M), plain(codes, scales, ws, handle.N)
        return A @ W.T + dev(bias).double(), A.abs() @ W.abs().T + dev(bias).double().abs()

    x, r = t(M, K).to(torch.bfloat16), t(M, K).to(torch.bfloat16)
    h, *a = fq.rmsnorm_quantize_act_fp4(x, r, up, block)
    for dtype in (torch.bfloat16, torch.float32):
        z = fq.gemm_fp4(*a, up, dtype)
        assert_product(z, *product(a, up, "nv"), K)
        y = torch.nn.functional.silu(z[:, :F]) * z[:, F:]
        out = fq.linear_fp4(y, down, dtype)
        assert_product(out, *product(fq.quantize_act_fp4(y, down, block, fq.MXFP4), down, "mx"), F)
    check_status()


def test_offsets_past_32_bits():
    """More than 2^32 numbers in rows, codes and outputs: the last rows are those of a short call, the last outputs those of 64 bits."""
    M, K, N, last, channels = 135000, 32768, 32768, 40, 512
    x = torch.randn(1000, K, device="cuda", dtype=torch.bfloat16).repeat(M // 1000, 1)
    x[-last:] = torch.randn(last, K, device="cuda", dtype=torch.bfloat16)
    tail = x[-last:].clone()

    def rows_of(scales, blocks, first, rows):                        # of the tiles from `first` on
        at = scales.view(-1, blocks // 4 * 512)[first // 128:(first + rows + 127) // 128]
        return at.reshape(-1, blocks // 4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, blocks)[first % 128:first % 128 + rows]

    for form in ("mx", "nv"):
        blocks = K // BLOCK[form]
        codes, scales, steps = fq.quantize_act_fp4(x, None, 64, FORMATS[form])
        short = fq.quantize_act_fp4(tail, None, 64, FORMATS[form])
        assert torch.equal(codes[-last:], short[0]) and torch.equal(steps[-last:], short[2])
        assert torch.equal(rows_of(scales, blocks, M - last, last), rows_of(short[1], blocks, 0, last))
    h = fq.weights_import_fp4(codes[:N], scales[:fq.fp4_scale_bytes(N, K, fq.NVFP4)], None, None, None, K, 64)
    y = fq.gemm_fp4(codes, scales, steps, h, torch.bfloat16)
    A = dev(values(host(short[0]), host(rows_of(short[1], blocks, 0, last)), host(short[2]), "nv"))
    W = dev(values(host(codes[N - channels:N]), host(rows_of(scales, blocks, N - channels, channels)), np.ones(channels, np.float32), "nv"))
    assert_product(y[-last:, -channels:], A @ W.T, A.abs() @ W.abs().T, K)
    check_status()
    del y, codes, scales, steps
    want = fq.rmsnorm_quantize_act(tail, tail, None, 64, 8)
    got = fq.rmsnorm_quantize_act(x, x, None, 64, 8, h=x)
    assert got[0].data_ptr() == x.data_ptr()
    assert torch.equal(x[-last:], want[0]) and torch.equal(got[1][-last:], want[1])
    check_status()
