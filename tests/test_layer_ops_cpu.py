"""Refusals of the operators between a layer's projections: argument checks run on the host, ahead of any device work."""
import ctypes

import pytest
import torch

from paper_2609_24433_b200 import build as fq_build
from paper_2609_24433_b200 import fq

NULL = ctypes.c_void_p(0)
ONE = ctypes.c_void_p(4096)             # an address that is never touched
I, L, F, Z = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


@pytest.fixture(scope="module")
def lib():
    fq_build.build()
    return fq.lib()


class Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("page", ctypes.c_int)]


def cache(pages=4, heads=2, head_dim=64, page=16, k=4096):
    return Cache(k, 4096, 4096, 4096, pages, heads, head_dim, page)


def rope(lib, M=4, ldx=512, hq=4, hk=2, D=64, x=ONE, positions=ONE, r=64, layout=0, q=ONE, ldq=256, k=ONE, ldk=128, xt=1, yt=1, eps=1e-6, gain=NULL):
    return lib.fq_qk_norm_rope(x, xt, L(M), L(ldx), hq, hk, D, gain, NULL, F(eps), positions, ONE, r, layout, F(1.0), q, L(ldq), k, L(ldk), yt, NULL)


def test_rope_refusals(lib):
    assert rope(lib, M=0) == fq.OK and rope(lib, hq=0, hk=0) == fq.OK
    for bad in (dict(M=-1), dict(hq=-1), dict(D=0), dict(r=63), dict(r=66), dict(r=-2), dict(layout=2), dict(xt=2), dict(yt=7),
                dict(ldx=376), dict(x=NULL), dict(positions=NULL), dict(q=NULL), dict(k=NULL), dict(ldq=248), dict(ldk=120),
                dict(eps=-1.0), dict(eps=float("nan"))):
        assert rope(lib, **bad) == fq.ERR_INVALID_ARG, bad
    for bad in (dict(D=60, r=60), dict(D=264, ldx=4096, ldq=4096, ldk=4096), dict(hq=40000)):
        assert rope(lib, **bad) == fq.ERR_UNSUPPORTED, bad
    for bad in (dict(ldx=513), dict(x=ctypes.c_void_p(4098)), dict(q=ctypes.c_void_p(4104)), dict(ldk=132), dict(gain=ctypes.c_void_p(4100))):
        assert rope(lib, **bad) == fq.ERR_ALIGNMENT, bad


def test_rope_frequency_refusals(lib):
    for args in ((7,), (-2,), (8, 0.0), (8, -1.0), (8, 1e4, 9), (8, 1e4, fq.ROPE_LINEAR, 0.5), (8, 1e4, fq.ROPE_LINEAR, float("nan")),
                 (8, 1e4, fq.ROPE_PARTS, 2.0, 0.0), (8, 1e4, fq.ROPE_PARTS, 2.0, 100.0, 4.0, 4.0), (2, 1e4, fq.ROPE_BASE, 2.0)):
        with pytest.raises(fq.FqError) as e:
            fq.rope_frequencies(*args, device="cpu")
        assert e.value.status == fq.ERR_INVALID_ARG, args


def append(lib, c, T=4, batch=2, k=ONE, ldk=128, table=ONE, ld=8, width=8, lens=ONE, offsets=NULL, xt=1, most=0):
    return lib.fq_kv8_append(k, ONE, xt, L(T), L(ldk), L(128), ctypes.byref(c) if c is not None else NULL, table, L(ld), L(width), batch, lens,
                             offsets, L(most), NULL)


def test_append_refusals(lib):
    assert append(lib, cache(), T=0) == fq.OK and append(lib, cache(), batch=0, T=0) == fq.OK and append(lib, cache(), width=0) == fq.OK
    assert append(lib, cache(pages=0, k=0)) == fq.OK
    assert append(lib, None) == fq.ERR_INVALID_ARG
    for c in (cache(pages=-1), cache(heads=0), cache(head_dim=0), cache(page=0), cache(k=0)):
        assert append(lib, c) == fq.ERR_INVALID_ARG
    for c in (cache(head_dim=40), cache(head_dim=272), cache(page=48), cache(page=256), cache(page=8), cache(heads=40000)):
        assert append(lib, c, ldk=1 << 24) == fq.ERR_UNSUPPORTED
    assert append(lib, cache(k=4100)) == fq.ERR_ALIGNMENT
    for bad in (dict(T=-1), dict(T=5), dict(batch=-1), dict(k=NULL), dict(ldk=120), dict(table=NULL), dict(ld=4), dict(width=-1), dict(lens=NULL),
                dict(xt=3), dict(most=-1)):
        assert append(lib, cache(), **bad) == fq.ERR_INVALID_ARG, bad
    for bad in (dict(k=ctypes.c_void_p(4097)), dict(ldk=130)):
        assert append(lib, cache(), **bad) == fq.ERR_ALIGNMENT, bad


def attend(lib, c, rows=4, hq=4, q=ONE, ldq=256, table=ONE, ld=8, width=8, batch=2, lens=ONE, offsets=NULL, max_q=0, max_kv=0, scale=1.0, y=ONE,
           ws=NULL, ws_bytes=0, dt=1):
    return lib.fq_attention_kv8(q, dt, L(rows), L(ldq), hq, ctypes.byref(c) if c is not None else NULL, table, L(ld), L(width), batch, lens, offsets,
                                L(max_q), L(max_kv), 1, F(scale), y, L(256), ws, Z(ws_bytes), NULL)


def test_attention_kv8_refusals(lib):
    assert attend(lib, cache(), rows=0) == fq.OK and attend(lib, cache(), rows=0, batch=0) == fq.OK
    for bad in (dict(rows=-1), dict(rows=5), dict(hq=0), dict(hq=3), dict(q=NULL), dict(ldq=248), dict(table=NULL), dict(ld=7), dict(lens=NULL),
                dict(max_q=-1), dict(max_kv=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(y=NULL), dict(dt=2)):
        assert attend(lib, cache(), **bad) == fq.ERR_INVALID_ARG, bad
    assert attend(lib, None) == fq.ERR_INVALID_ARG
    for c in (cache(head_dim=24), cache(head_dim=512), cache(page=100)):
        assert attend(lib, c, ldq=1 << 16) == fq.ERR_UNSUPPORTED
    assert attend(lib, cache(), ldq=260) == fq.ERR_ALIGNMENT and attend(lib, cache(), y=ctypes.c_void_p(4098)) == fq.ERR_ALIGNMENT


def test_attention_workspaces(lib):
    c = cache(pages=4096, heads=1, head_dim=128, page=64)
    need = lib.fq_attention_kv8_workspace_bytes(1, 1, 8, ctypes.byref(c), 1000, 1, 0, 0, 0)
    assert need > 0 and need % 256 == 0                 # one token over 64000 keys: chunks that meet
    assert lib.fq_attention_kv8_workspace_bytes(1, 1, 8, ctypes.byref(c), 1, 1, 0, 0, 0) == 0
    assert lib.fq_attention_kv8_workspace_bytes(1, 0, 8, ctypes.byref(c), 1000, 0, 0, 0, 0) == 0
    assert lib.fq_cross_attention_workspace_bytes(1, 1, 8, 100000, 8, 64, 1, 0, 0, 0, 0) > 0
    assert lib.fq_cross_attention_workspace_bytes(1, 1, 8, 100000, 8, 64, 1, 0, 0, 0, 64) == 0


def cross(lib, rows=4, hq=4, hk=2, D=64, batch=2, kv_rows=8, q=ONE, ldq=256, k=ONE, ldk=128, scale=1.0, y=ONE, dt=1, max_kv=0):
    return lib.fq_cross_attention(q, dt, L(rows), L(ldq), hq, k, ONE, L(kv_rows), L(ldk), L(128), hk, D, batch, NULL, NULL, NULL, NULL, L(0), L(max_kv),
                                  F(scale), y, L(256), NULL, Z(0), NULL)


def test_cross_attention_refusals(lib):
    assert cross(lib, rows=0) == fq.OK and cross(lib, rows=0, batch=0) == fq.OK
    for bad in (dict(rows=-2), dict(rows=5), dict(kv_rows=7), dict(kv_rows=-2), dict(hq=3), dict(hk=0), dict(D=0), dict(batch=-1), dict(q=NULL),
                dict(k=NULL), dict(ldq=200), dict(ldk=120), dict(scale=float("nan")), dict(y=NULL), dict(dt=5), dict(max_kv=-1)):
        assert cross(lib, **bad) == fq.ERR_INVALID_ARG, bad
    for bad in (dict(D=72, ldq=512, ldk=512), dict(D=512, ldq=4096, ldk=4096)):
        assert cross(lib, **bad) == fq.ERR_UNSUPPORTED, bad
    for bad in (dict(q=ctypes.c_void_p(4100)), dict(ldk=132), dict(k=ctypes.c_void_p(4104))):
        assert cross(lib, **bad) == fq.ERR_ALIGNMENT, bad


def test_tensors_that_are_not_on_the_device_are_refused():
    x, f = torch.zeros(2, 192), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="current CUDA device"):
        fq.qk_norm_rope(x, 1, 1, 64, torch.zeros(2, dtype=torch.int32), f)
    c = fq.KV8Cache.empty(2, 1, 64, 16, device="cpu")
    with pytest.raises(ValueError, match="current CUDA device"):
        fq.kv8_append(x[:, :64], x[:, :64], c, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="current CUDA device"):
        fq.attention_kv8(x[:, :64], 1, c, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="current CUDA device"):
        fq.cross_attention(x[:, :64], x[:, :64], x[:, :64], 1, 1, 1)


def test_a_cache_of_other_shapes_or_types_is_refused():
    k, v, s = torch.zeros(2, 3, 16, 64, dtype=torch.int8), torch.zeros(2, 3, 64, 16, dtype=torch.int8), torch.zeros(2, 3)
    c = fq.KV8Cache(k, v, s, s.clone())
    assert (c.pages, c.heads, c.page, c.head_dim) == (2, 3, 16, 64)
    for bad in ((k[0], v, s, s), (k, k, s, s), (k, v.float(), s, s), (k, v, s.double(), s), (k, v, s, s[:, :2]), (k, v.transpose(2, 3).contiguous().transpose(2, 3), s, s.t().contiguous().t())):
        with pytest.raises(ValueError):
            fq.KV8Cache(*bad)


def test_arrays_that_do_not_begin_on_an_element_are_refused(lib):
    for at in (4097, 4098, 4099):
        assert rope(lib, positions=ctypes.c_void_p(at)) == fq.ERR_ALIGNMENT
        assert append(lib, Cache(4096, 4096, at, 4096, 4, 2, 64, 16)) == append(lib, Cache(4096, 4096, 4096, at, 4, 2, 64, 16)) == fq.ERR_ALIGNMENT
        assert attend(lib, Cache(4096, 4096, 4096, at, 4, 2, 64, 16)) == fq.ERR_ALIGNMENT
    for at in (4098, 4100):
        assert lib.fq_qk_norm_rope(ONE, 1, L(4), L(512), 4, 2, 64, NULL, NULL, F(1e-6), ONE, ctypes.c_void_p(at), 64, 0, F(1.0), ONE, L(256), ONE, L(128),
                                   1, NULL) == fq.ERR_ALIGNMENT


def test_leading_dimensions_by_type(lib):
    for bad in (dict(ldx=518, xt=0), dict(ldq=258, yt=0), dict(ldk=130, yt=0), dict(ldq=260, xt=0), dict(ldk=132, xt=0)):
        assert rope(lib, **bad) == fq.ERR_ALIGNMENT, bad
    assert append(lib, cache(), ldk=130, xt=0) == append(lib, cache(), ldk=132) == fq.ERR_ALIGNMENT
    assert attend(lib, cache(), ldq=258, dt=0) == cross(lib, ldq=258, dt=0) == cross(lib, ldk=130, dt=0) == fq.ERR_ALIGNMENT


def test_pairs_of_sequence_and_head_by_route(lib):
    """Single tokens take as many as there are; the other kernels have a grid of them."""
    c = cache(heads=8, head_dim=16)
    assert lib.fq_attention_kv8_workspace_bytes(1, 70000, 8, ctypes.byref(c), 1000, 70000, 0, 0, 0) > 0
    assert attend(lib, c, rows=3 * 8200, batch=8200, hq=64, ldq=1024) == fq.ERR_UNSUPPORTED
    assert cross(lib, rows=8200, batch=8200, kv_rows=8200, hq=8, hk=8, D=16) == fq.ERR_UNSUPPORTED


@pytest.mark.parametrize("at", [4097, 4098, 4099])
def test_lengths_offsets_and_tables_that_do_not_begin_on_an_element_are_refused(lib, at):
    odd = ctypes.c_void_p(at)
    for which in ("table", "lens", "offsets"):
        assert append(lib, cache(), **{which: odd}) == attend(lib, cache(), **{which: odd}) == fq.ERR_ALIGNMENT, which
    for arrays in ((odd, NULL, NULL), (NULL, odd, NULL), (NULL, NULL, odd)):
        assert lib.fq_cross_attention(ONE, 1, L(4), L(256), 4, ONE, ONE, L(8), L(128), L(128), 2, 64, 2, *arrays, NULL, L(0), L(0), F(1.0), ONE, L(256),
                                      NULL, Z(0), NULL) == fq.ERR_ALIGNMENT
