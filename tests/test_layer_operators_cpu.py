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
