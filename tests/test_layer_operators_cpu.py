"""What the C entry points of the layer's operators (prompt attention, norms and rotation, adapters) refuse, without a GPU."""
from __future__ import annotations

import ctypes as C

import pytest

FAKE, ODD = C.c_void_p(0x10000), C.c_void_p(0x10001)            # never dereferenced: the calls fail validation, or have nothing to do
OK, NULL, SHAPE, DTYPE, ALPHA, ALIGN, WORKSPACE = 0, 1, 2, 3, 5, 6, 7


@pytest.fixture(scope="module")
def lib():
    from paper_2410_07505_b200 import build, cq
    build.build()
    return cq.lib()


def test_prompt_attention_refuses(lib):
    def call(Q=FAKE, qt=256, qh=64, K=FAKE, kt=128, kh=64, V=FAKE, vt=128, vh=64, dt=1, B=1, Tq=10, Tk=20, Hq=4, H=2, D=64, qs=FAKE, ks=FAKE, scale=0.1,
             out=FAKE, lse=None, ws=FAKE, n=1 << 40):
        return lib.cq_prompt_attention(Q, qt, qh, K, kt, kh, V, vt, vh, dt, B, Tq, Tk, Hq, H, D, qs, ks, scale, out, lse, ws, n, None)
    for name in ("Q", "K", "V", "out", "qs", "ks"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(B=-1), dict(Tq=-1), dict(Tk=-1), dict(H=0), dict(Hq=3), dict(Hq=1), dict(D=80), dict(D=256), dict(Tq=1 << 30), dict(Tk=1 << 30),
                dict(qt=0), dict(kh=0), dict(vt=-128), dict(kt=1 << 39), dict(Hq=1 << 17, H=1 << 17), dict(B=1 << 21)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(qt=257), dict(qh=68), dict(kt=4), dict(kh=60), dict(vt=129), dict(vh=65), dict(Q=ODD), dict(K=C.c_void_p(0x10008)), dict(V=C.c_void_p(0x10002)),
                dict(out=C.c_void_p(0x10008)), dict(lse=C.c_void_p(0x10002)), dict(qs=C.c_void_p(0x10002)), dict(ks=ODD)):
        assert call(**bad) == ALIGN, bad
    assert call(dt=2) == DTYPE and call(dt=-1) == DTYPE
    for s in (0.0, -1.0, float("nan"), float("inf"), 1e-40, 1e31):
        assert call(scale=s) == ALPHA
    assert call(B=0) == OK and call(Tq=0) == OK
    need = lib.cq_prompt_attention_workspace_bytes
    assert need(1, 10, 20, 4, 2, 64) == 0 and need(1, 10, 20, 4, 2, 80) == 0 and need(-1, 10, 20, 4, 2, 64) == 0


def test_norm_rotate_refuses(lib):
    def call(Q=FAKE, Hq=4, K=FAKE, H=2, dt=1, T=3, D=64, R=64, pos=FAKE, freq=FAKE, qw=None, kw=None, eps=1e-6, qo=FAKE, ko=FAKE):
        return lib.cq_norm_rotate(Q, 256, 64, Hq, K, 128, 64, H, dt, T, D, R, 0, pos, freq, qw, kw, eps, qo, 256, 64, ko, 128, 64, None)
    for name in ("Q", "K", "pos", "freq", "qo", "ko"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(T=-1), dict(Hq=-1), dict(H=-1), dict(Hq=1 << 17), dict(D=0), dict(D=513), dict(R=63), dict(R=66), dict(R=-2), dict(T=1 << 31)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(Q=ODD), dict(ko=ODD), dict(qw=ODD), dict(pos=C.c_void_p(0x10004)), dict(freq=C.c_void_p(0x10004))):
        assert call(**bad) == ALIGN, bad
    assert call(dt=2) == DTYPE
    assert call(eps=float("nan")) == ALPHA and call(eps=1e31) == ALPHA and call(eps=-1.0, qw=FAKE) == ALPHA and call(eps=-1.0, kw=FAKE) == ALPHA
    assert call(T=0) == OK and call(Hq=0, H=0) == OK


def test_adapter_add_refuses(lib):
    def call(X=FAKE, dt=1, T=5, K=64, ldx=64, A=FAKE, B=FAKE, scale=FAKE, n=3, R=16, N=72, index=FAKE, y=FAKE, ydt=1, ldy=72, out=FAKE, ldo=72, ws=FAKE, size=1 << 30):
        return lib.cq_adapter_add(X, dt, T, K, ldx, A, B, scale, n, R, N, index, y, ydt, ldy, out, ldo, ws, size, None)
    for name in ("X", "A", "B", "index", "y", "out"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(T=-1), dict(K=-1), dict(N=-1), dict(n=-1), dict(ldx=63), dict(ldy=71), dict(ldo=71), dict(R=0), dict(R=12), dict(R=136), dict(T=1 << 23)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(X=ODD), dict(A=ODD), dict(B=C.c_void_p(0x10008)), dict(scale=C.c_void_p(0x10002)), dict(index=C.c_void_p(0x10002)), dict(y=ODD), dict(out=ODD),
                dict(ydt=2, y=C.c_void_p(0x10002))):
        assert call(**bad) == ALIGN, bad
    assert call(dt=2) == DTYPE and call(ydt=3) == DTYPE
    assert call(ws=None) == WORKSPACE and call(ws=C.c_void_p(0x10010)) == WORKSPACE and call(size=100) == WORKSPACE
    assert call(T=0) == OK and call(N=0, ldy=0, ldo=0) == OK
    need = lib.cq_adapter_add_workspace_bytes
    assert need(5, 16) >= 5 * 16 * 4 + 20 and need(0, 16) >= 0 and need(-1, 16) == 0 and need(5, 0) == 0 and need(5, 129) == 0
