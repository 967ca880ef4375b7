"""Refusals of the 4-bit floating-point projections and of the norm that ends in codes: argument checks run on the host, ahead
of any device work."""
import ctypes

import pytest

from paper_2609_24433_b200 import build as fq_build
from paper_2609_24433_b200 import fq

NULL = ctypes.c_void_p(0)
ONE = ctypes.c_void_p(4096)             # an address that is never touched
ODD = ctypes.c_void_p(4098)
L, F, Z = ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


@pytest.fixture(scope="module")
def lib():
    fq_build.build()
    return fq.lib()


def test_scale_bytes(lib):
    assert fq.fp4_scale_bytes(1, 32, fq.MXFP4) == 512 and fq.fp4_scale_bytes(1, 32, fq.NVFP4) == 512
    assert fq.fp4_scale_bytes(129, 160, fq.MXFP4) == 2 * 2 * 512 and fq.fp4_scale_bytes(128, 160, fq.NVFP4) == 3 * 512
    for bad in ((0, 64, 0), (-1, 64, 0), (1, 0, 0), (1, 48, 0), (1, 32800, 1), (1, 64, 2), ((1 << 31) + 1, 64, 1)):
        assert fq.fp4_scale_bytes(*bad) == 0, bad


def test_workspace_bytes(lib):
    need = lib.fq_linear_fp4_workspace_bytes(50, 1024, fq.NVFP4)
    assert need % 256 == 0 and need >= 50 * 512 + fq.fp4_scale_bytes(50, 1024, fq.NVFP4) + 200
    assert lib.fq_linear_fp4_workspace_bytes(0, 1024, 0) == 0 and lib.fq_linear_fp4_workspace_bytes(4, 1000, 0) == 0


def quantize(lib, x=ONE, xt=1, M=4, K=64, ldx=64, g=NULL, block=1, fmt=1, codes=ONE, scales=ONE, delta=ONE):
    return lib.fq_quantize_act_fp4(x, xt, L(M), L(K), L(ldx), g, block, fmt, codes, scales, delta, NULL)


def test_quantize_refusals(lib):
    assert quantize(lib, M=0) == fq.OK and quantize(lib, M=0, x=NULL, codes=NULL) == fq.OK
    for bad in (dict(M=-1), dict(K=0), dict(K=-32), dict(fmt=2), dict(fmt=-1), dict(xt=2), dict(x=NULL), dict(ldx=56), dict(codes=NULL), dict(scales=NULL),
                dict(delta=NULL)):
        assert quantize(lib, **bad) == fq.ERR_INVALID_ARG, bad
    for bad in (dict(K=48, ldx=48), dict(K=32800, ldx=32800), dict(block=3), dict(block=512, K=512, ldx=512), dict(block=0), dict(block=128), dict(M=(1 << 31) + 1)):
        assert quantize(lib, **bad) == fq.ERR_UNSUPPORTED, bad
    for bad in (dict(x=ODD), dict(ldx=68), dict(codes=ODD), dict(scales=ctypes.c_void_p(4104)), dict(delta=ODD), dict(g=ctypes.c_void_p(4104))):
        assert quantize(lib, **bad) == fq.ERR_ALIGNMENT, bad


def test_handle_refusals(lib):
    out = ctypes.c_void_p()

    def fold(W=ONE, wt=0, N=8, K=64, ld=64, smooth=NULL, bias=NULL, block=1, fmt=0, to=ctypes.byref(out)):
        return lib.fq_fold_weights_fp4(W, wt, L(N), L(K), L(ld), smooth, bias, block, fmt, NULL, to)

    def load(codes=ONE, scales=ONE, N=8, K=64, block=1, fmt=0, to=ctypes.byref(out), ws=NULL):
        return lib.fq_fp4_weights_import(codes, scales, ws, NULL, NULL, L(N), L(K), block, fmt, NULL, to)

    for call in (fold, load):
        for bad in (dict(N=-8), dict(K=0), dict(fmt=2), dict(to=NULL)):
            assert call(**bad) == fq.ERR_INVALID_ARG, bad
        for bad in (dict(N=12), dict(K=40), dict(K=65536), dict(block=5), dict(block=128)):
            assert call(**bad) == fq.ERR_UNSUPPORTED, bad
    for bad in (dict(W=NULL), dict(wt=3), dict(ld=32)):
        assert fold(**bad) == fq.ERR_INVALID_ARG, bad
    for bad in (dict(W=ODD), dict(ld=68), dict(smooth=ctypes.c_void_p(4104)), dict(bias=ODD)):
        assert fold(**bad) == fq.ERR_ALIGNMENT, bad
    assert load(codes=NULL) == fq.ERR_INVALID_ARG and load(scales=NULL) == fq.ERR_INVALID_ARG and load(ws=ODD) == fq.ERR_ALIGNMENT
    assert out.value is None
    n = ctypes.c_int64()
    assert lib.fq_fp4_weights_info(NULL, ctypes.byref(n), NULL, NULL, NULL) == fq.ERR_INVALID_ARG
    assert lib.fq_fp4_weights_export(NULL, NULL, NULL, NULL, NULL, NULL, NULL) == fq.ERR_INVALID_ARG
    assert lib.fq_fp4_weights_destroy(NULL) == fq.OK and not lib.fq_fp4_weights_multiplier(NULL)
    assert lib.fq_gemm_fp4(ONE, ONE, ONE, L(1), NULL, ONE, 0, L(8), NULL) == fq.ERR_INVALID_ARG
    assert lib.fq_linear_fp4(ONE, 0, L(1), L(64), NULL, ONE, 0, L(8), ONE, Z(1 << 20), NULL) == fq.ERR_INVALID_ARG


def norm(lib, x=ONE, r=ctypes.c_void_p(8192), xt=1, M=4, K=64, ldx=64, ldr=64, eps=1e-6, h=ctypes.c_void_p(16384), ldh=64, g=NULL, block=1, bits=8, clip=1.0,
         codes=ONE, delta=ONE):
    return lib.fq_rmsnorm_quantize_act(x, r, xt, L(M), L(K), L(ldx), L(ldr), F(eps), h, L(ldh), g, block, bits, F(clip), codes, delta, NULL)


def test_norm_refusals(lib):
    assert norm(lib, M=0) == fq.OK
    for bad in (dict(M=-1), dict(K=0), dict(bits=6), dict(clip=0.0), dict(clip=1.5), dict(clip=float("nan")), dict(eps=-1e-9), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(xt=5), dict(x=NULL), dict(r=NULL), dict(h=NULL), dict(ldx=32), dict(ldr=32), dict(ldh=32), dict(codes=NULL),
                dict(delta=NULL), dict(h=ONE, ldh=72), dict(h=ctypes.c_void_p(8192), ldr=72)):
        assert norm(lib, **bad) == fq.ERR_INVALID_ARG, bad
    for bad in (dict(K=40, ldx=40, ldr=40, ldh=40), dict(block=7), dict(block=128), dict(M=(1 << 31) + 1)):
        assert norm(lib, **bad) == fq.ERR_UNSUPPORTED, bad
    for bad in (dict(x=ODD), dict(ldx=68), dict(r=ODD), dict(ldr=68), dict(h=ODD), dict(ldh=68), dict(codes=ODD), dict(delta=ODD), dict(g=ODD)):
        assert norm(lib, **bad) == fq.ERR_ALIGNMENT, bad
    call = lambda fmt, scales: lib.fq_rmsnorm_quantize_act_fp4(ONE, NULL, 1, L(4), L(64), L(64), L(0), F(0.0), NULL, L(0), NULL, 1, fmt, ONE, scales, ONE, NULL)
    assert call(2, ONE) == fq.ERR_INVALID_ARG and call(1, NULL) == fq.ERR_INVALID_ARG and call(0, ODD) == fq.ERR_ALIGNMENT


class Rows:
    """What a handle is compared with: rows of a width, on a device."""
    def __init__(self, K, device):
        self.shape, self.device = (4, K), type("Device", (), {"index": device})


@pytest.mark.parametrize("cls", [fq.Weights, fq.Fp4Weights])
def test_multiplier_of_another_site_is_refused(cls, lib, monkeypatch):
    """A handle's multiplier carries its block's norm and lies on its device."""
    h = cls.__new__(cls)
    h.K, h.block, h.device, h.fold_after, h._h, h._addr = 128, 64, 0, False, None, None
    monkeypatch.setattr(cls, "handle", ctypes.c_void_p(0), raising=False)
    monkeypatch.setattr(cls, "multiplier_ptr", lambda self: 4096)
    assert fq._multiplier(h, Rows(128, 0), 64) == 4096
    for rows, block in ((Rows(96, 0), 64), (Rows(128, 0), 32), (Rows(128, 0), 1), (Rows(128, 1), 64), (Rows(128, None), 64)):
        with pytest.raises(ValueError):
            fq._multiplier(h, rows, block)


def test_multiplier_may_be_a_parameter():
    """A torch.nn.Parameter is a tensor like any other."""
    import torch
    for g in (None, torch.ones(128), torch.nn.Parameter(torch.ones(128)), torch.nn.Buffer(torch.ones(128))):
        assert fq._multiplier(g, Rows(128, 0), 64) is g
    for bad in (4096, 1.0, "g", [1.0]):
        with pytest.raises(TypeError):
            fq._multiplier(bad, Rows(128, 0), 64)
