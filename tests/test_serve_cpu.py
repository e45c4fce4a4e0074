"""The serving operators without a GPU: the tests' own plain forms, the sizes of workspaces, and what the C entry points
and the binding refuse before they touch a device."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

import serve_reference as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2410_07505_b200 import build, cq
    build.build()
    return cq.lib()


FAKE = C.c_void_p(0x10000)     # never dereferenced: every call below fails validation first
ODD = C.c_void_p(0x10001)
OK, NULL, SHAPE, DTYPE, BITS, ALPHA, ALIGN, WORKSPACE = range(8)


def test_e4m3_rounding_of_the_plain_form_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    values = codes[torch.isfinite(codes)].double().numpy()
    assert len(values) == 254 and values.max() == 448
    np.testing.assert_array_equal(ref.round_e4m3(values), values)
    v = np.sort(np.unique(values))
    mids = (v[1:] + v[:-1]) / 2                             # ties, and their neighbours on both sides
    probe = np.concatenate((mids, np.nextafter(mids.astype(np.float32), np.float32(1e9)), np.nextafter(mids.astype(np.float32), np.float32(-1e9))))
    probe = probe.astype(np.float32)
    np.testing.assert_array_equal(ref.round_e4m3(probe), torch.from_numpy(probe).to(torch.float8_e4m3fn).double().numpy())


def test_packing_of_the_plain_form_round_trips():
    c = np.random.default_rng(0).integers(-7, 8, (3, 2, 5, 64))
    np.testing.assert_array_equal(ref.unpack(ref.pack(c, 4), 4), c)
    assert int(ref.pack(np.array([[1, -2]]), 4)[0, 0]) == 0xE1       # element 0 low, element 1 high


def test_workspace_sizes(lib):
    from paper_2410_07505_b200 import cq
    assert lib.cq_fp8_linear_workspace_bytes(1, 128) >= 128 + 16
    assert lib.cq_fp8_linear_workspace_bytes(4096, 8192) >= 4096 * 8192 + 4 * 4096 * 64
    assert lib.cq_fp8_linear_workspace_bytes(-1, 128) == 0
    assert 0 < cq.kv_attention_workspace_bytes(64) < cq.kv_attention_workspace_bytes(128) < 64 << 20
    assert cq.kv_attention_workspace_bytes(0) == 0


def test_fp8_quantizers_refuse(lib):
    def act(X=FAKE, dt=1, T=4, K=256, ld=256, codes=FAKE, ldc=256, scale=FAKE, lds=4):
        return lib.cq_fp8_quantize_act(X, dt, T, K, ld, codes, ldc, scale, lds, None)
    assert act(X=None) == NULL and act(codes=None) == NULL and act(scale=None) == NULL
    assert act(T=-1) == SHAPE and act(ld=255) == SHAPE and act(ldc=255) == SHAPE and act(lds=3) == SHAPE
    assert act(dt=2) == DTYPE and act(X=ODD) == ALIGN and act(scale=C.c_void_p(0x10002)) == ALIGN
    assert act(T=0) == OK and act(K=0, ld=0, ldc=0) == OK

    def weight(W=FAKE, dt=1, N=4, K=256, ld=256, codes=FAKE, ldc=256, scale=FAKE):
        return lib.cq_fp8_quantize_weight(W, dt, N, K, ld, codes, ldc, scale, None)
    assert weight(W=None) == NULL and weight(codes=None) == NULL and weight(scale=None) == NULL
    assert weight(N=-1) == SHAPE and weight(ldc=100) == SHAPE and weight(dt=7) == DTYPE and weight(N=0) == OK


def test_fp8_product_refuses(lib):
    def mm(A=FAKE, lda=256, sa=FAKE, lds=8, W=FAKE, ldw=256, sw=FAKE, M=5, N=7, K=250, out=FAKE, dt=1, ldo=7):
        return lib.cq_fp8_matmul(A, lda, sa, lds, W, ldw, sw, M, N, K, out, dt, ldo, None)
    for name in ("A", "sa", "W", "sw", "out"):
        assert mm(**{name: None}) == NULL
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(lda=249), dict(ldw=249), dict(ldo=6), dict(lds=4)):
        assert mm(**bad) == SHAPE
    for bad in (dict(A=C.c_void_p(0x10008)), dict(W=C.c_void_p(0x10008)), dict(lda=264), dict(ldw=264), dict(lds=6),
                dict(sa=C.c_void_p(0x10004)), dict(sw=C.c_void_p(0x10002)), dict(out=ODD)):
        assert mm(**bad) == ALIGN, bad
    assert mm(dt=5) == DTYPE
    assert mm(M=0, lds=0) == OK and mm(N=0, ldo=0) == OK

    def linear(X=FAKE, dt=1, M=5, K=250, ldx=250, W=FAKE, ldw=256, sw=FAKE, N=7, out=FAKE, odt=1, ldo=7, ws=FAKE, n=1 << 20):
        return lib.cq_fp8_linear(X, dt, M, K, ldx, W, ldw, sw, N, out, odt, ldo, ws, n, None)
    assert linear(X=None) == NULL and linear(W=None) == NULL and linear(sw=None) == NULL and linear(out=None) == NULL
    assert linear(ldx=249) == SHAPE and linear(ldw=249) == SHAPE and linear(ldo=6) == SHAPE and linear(N=-1) == SHAPE
    assert linear(dt=2) == DTYPE and linear(odt=3) == DTYPE
    assert linear(ldw=260) == ALIGN and linear(out=ODD) == ALIGN
    assert linear(ws=None) == WORKSPACE and linear(ws=C.c_void_p(0x10010)) == WORKSPACE and linear(n=100) == WORKSPACE
    assert linear(M=0) == OK and linear(N=0, ldo=0) == OK


CACHE = dict(kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, kcol=None, vcol=None, bits=8, pages=4, page=16, H=2, D=64)
BAD_CACHES = [(dict(kc=None), NULL), (dict(vs=None), NULL), (dict(kcol=FAKE), NULL), (dict(bits=2), BITS), (dict(pages=-1), SHAPE),
              (dict(page=8), SHAPE), (dict(page=24), SHAPE), (dict(page=8192), SHAPE), (dict(H=0), SHAPE), (dict(D=80), SHAPE),
              (dict(D=256), SHAPE), (dict(pages=1 << 26, page=16, H=2), SHAPE), (dict(kc=C.c_void_p(0x10008)), ALIGN),
              (dict(ks=C.c_void_p(0x10004)), ALIGN), (dict(kcol=FAKE, vcol=C.c_void_p(0x10004)), ALIGN)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_cache_entry_points_refuse_a_bad_cache(lib, bad, status):
    c = list({**CACHE, **bad}.values())
    assert lib.cq_kv_write(FAKE, 128, 64, FAKE, 128, 64, 1, 3, FAKE, *c, None) == status
    assert lib.cq_kv_read(*c, 3, FAKE, FAKE, FAKE, 1, None) == status
    assert lib.cq_kv_attention(FAKE, 1, 128, 128, 64, 1, 1, 2, *c, FAKE, 4, 4, FAKE, 0.1, FAKE, None, FAKE, 1 << 30, None) == status


def test_cache_entry_points_refuse_bad_arguments(lib):
    c = list(CACHE.values())

    def write(K=FAKE, V=FAKE, dt=1, T=3, slots=FAKE):
        return lib.cq_kv_write(K, 128, 64, V, 128, 64, dt, T, slots, *c, None)
    assert write(K=None) == NULL and write(V=None) == NULL and write(slots=None) == NULL
    assert write(dt=2) == DTYPE and write(T=-1) == SHAPE and write(K=ODD) == ALIGN and write(slots=C.c_void_p(0x10004)) == ALIGN
    assert write(T=0) == OK

    def read(L=3, slots=FAKE, k=FAKE, v=FAKE, dt=1):
        return lib.cq_kv_read(*c, L, slots, k, v, dt, None)
    assert read(slots=None) == NULL and read(k=None) == NULL and read(v=None) == NULL
    assert read(L=-1) == SHAPE and read(dt=4) == DTYPE and read(k=C.c_void_p(0x10008)) == ALIGN and read(L=0) == OK

    def attend(Q=FAKE, dt=1, B=1, Lq=1, Hq=4, table=FAKE, width=4, stride=4, lens=FAKE, scale=0.1, out=FAKE, lse=None, ws=FAKE, n=1 << 30):
        return lib.cq_kv_attention(Q, dt, 256, 256, 64, B, Lq, Hq, *c, table, width, stride, lens, scale, out, lse, ws, n, None)
    assert attend(Q=None) == NULL and attend(out=None) == NULL and attend(lens=None) == NULL and attend(table=None) == NULL
    assert attend(dt=2) == DTYPE
    for bad in (dict(B=-1), dict(Lq=-1), dict(Hq=1), dict(Hq=3), dict(width=-1), dict(stride=3), dict(width=1 << 28, stride=1 << 28)):
        assert attend(**bad) == SHAPE, bad
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(scale=s) == ALPHA
    assert attend(Q=ODD) == ALIGN and attend(out=ODD) == ALIGN and attend(lse=C.c_void_p(0x10002)) == ALIGN and attend(lens=C.c_void_p(0x10002)) == ALIGN
    assert attend(ws=None) == WORKSPACE and attend(ws=C.c_void_p(0x10010)) == WORKSPACE and attend(n=1000) == WORKSPACE
    assert attend(B=0) == OK and attend(Lq=0) == OK
    assert lib.cq_serve_fault(None) == NULL


def test_binding_refuses_host_tensors_and_wrong_layouts(lib):
    from paper_2410_07505_b200 import cq
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    w = cq.Fp8Weight(torch.zeros(8, 256, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(1, 2))
    with pytest.raises(TypeError):
        cq.fp8_quantize_act(x)
    with pytest.raises(TypeError):
        cq.fp8_linear(x, w)
    with pytest.raises(TypeError):
        cq.fp8_matmul(cq.Fp8Act(w.codes, torch.zeros(2, 8)), w)
    codes, scale = torch.zeros(2, 1, 16, 64, dtype=torch.int8), torch.zeros(2, 1, 16)
    with pytest.raises(TypeError):
        cq.KVCache(codes, codes, scale, scale)
    with pytest.raises(ValueError):
        cq.KVCache(codes.to(torch.uint8), codes, scale, scale)
    with pytest.raises(ValueError):
        cq.KVCache(codes, codes, scale[:1], scale)
    with pytest.raises(ValueError):
        cq.KVCache(codes, codes, scale, scale, 8, torch.ones(1, 64))
    with pytest.raises(cq.CQError):
        cq.KVCache(codes, codes, scale, scale, 16)
