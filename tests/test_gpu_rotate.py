"""Norms and position rotation of queries and keys on the GPU against the formula in 64 bits.

Tolerance of an element y = a cos - b sin (U half an ulp at 1 of the dtype): the mean of up to 512 squares, its root and the products
are fp32: a and b are off by less than (512 / 2 + 8) 2^-24 < 2^-15 of themselves (the sum's relative error halves in the root); an angle's
sine and cosine by 2^-24 for the fraction of a turn, times 2 pi, plus 2^-22: 2^-20 in all; together 2^-14 (|a| + |b|).  The angle f = position * freq itself is a 64-bit product: the definition's below is rounded once
(2^-53 |f|), the kernel's is turns = position * (freq * (1 / 2 pi)), a rounded constant and two rounded products (3 * 2^-53 |f|): 2^-51 |f| (|a| + |b|) more,
which is 2^-11 at 2^40 radians and nothing at 2^31.  The result is rounded once: U |y|, or half a subnormal step.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from guards import Arena
from test_gpu_serve import DT, TINY, UNIT, cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


def definition(x, w, positions, freq, eps, neighbours):
    """(y, its tolerance without the rounding) in float64."""
    x = x.cpu().double().numpy()
    T, _, D = x.shape
    R = 2 * len(freq)
    with np.errstate(invalid="ignore", divide="ignore"):
        if eps is not None:
            x = x / np.sqrt((x ** 2).mean(axis=-1, keepdims=True) + eps)
            if w is not None:
                x = x * w.cpu().double().numpy()
        f = positions.cpu().numpy().astype(np.float64)[:, None] * freq.cpu().numpy()[None]
        cos, sin = np.cos(f)[:, None], np.sin(f)[:, None]
        at = (np.s_[..., 0:R:2], np.s_[..., 1:R:2]) if neighbours else (np.s_[..., :R // 2], np.s_[..., R // 2:R])
        y, tol = x.copy(), 2.0 ** -14 * np.abs(x)
        a, b = x[at[0]], x[at[1]]
        y[at[0]], y[at[1]] = a * cos - b * sin, a * sin + b * cos
        tol[at[0]] = tol[at[1]] = (2.0 ** -14 + 2.0 ** -51 * np.abs(f)[:, None]) * (np.abs(a) + np.abs(b))
    return y, tol


def compare(got, x, w, positions, freq, eps, neighbours):
    y, tol = definition(x, w, positions, freq, eps, neighbours)
    tol = tol + UNIT[x.dtype] * np.abs(y) * 1.001 + TINY[x.dtype]
    g = got.cpu().double().numpy()
    bad = ~(np.abs(g - y) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], y[bad][:5])


def case(cq, T, Hq, H, D, R, dtype, *, norm=True, weights=True, neighbours=False, first=0, eps=1e-6, seed=0, skew=0, wide=0):  # noqa: F811
    """`skew`: bytes that every tensor is moved by; `wide`: elements between heads beyond D."""
    t = DT[dtype]
    ar = Arena()
    row = (Hq + H) * (D + wide)
    for name in ("x", "y"):
        ar.add(name, max(1, T * row), t, skew=skew)
    ar.build()
    x = ar["x"][:T * row].view(T, Hq + H, D + wide)[..., :D]
    y = ar["y"][:T * row].view(T, Hq + H, D + wide)[..., :D]
    x.copy_(normal((T, Hq + H, D), seed, t).cuda())
    ar["y"].fill_(3)
    q, k = x.split((Hq, H), dim=1)
    w = [torch.exp(0.3 * normal((D,), seed + i, torch.float32, False)).to(t).cuda() if norm and weights else None for i in (1, 2)]
    positions = torch.arange(T, device="cuda") + first
    freq = cq.rotation_freq(R, 500000.0)
    e = eps if norm else None
    out = cq.norm_rotate(q, k, positions, freq, *w, eps=e, neighbours=neighbours, out=tuple(y.split((Hq, H), dim=1)))
    ar.check("norm_rotate")
    for got, src, ww in zip(out, (q, k), w):
        compare(got, src, ww, positions, freq, e, neighbours)
    if wide:
        assert bool((ar["y"][:T * row].view(T, Hq + H, D + wide)[..., D:] == 3).all())
    fresh = cq.norm_rotate(q, k, positions, freq, *w, eps=e, neighbours=neighbours)
    assert all(torch.equal(a, b) for a, b in zip(fresh, out))
    inplace = cq.norm_rotate(q, k, positions, freq, *w, eps=e, neighbours=neighbours, out=(q, k))
    assert inplace[0] is q and all(torch.equal(a, b) for a, b in zip(inplace, fresh))


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("neighbours", (False, True))
@pytest.mark.parametrize("D,R", ((64, 64), (64, 16), (128, 128), (128, 32), (128, 0), (256, 256), (96, 96), (80, 32), (72, 16), (8, 0)))
def test_rows_in_vectors(cq, dtype, neighbours, D, R):  # noqa: F811
    for T, Hq, H in ((1, 4, 1), (5, 9, 3), (70, 2, 2)):
        case(cq, T, Hq, H, D, R, dtype, neighbours=neighbours, first=17, seed=D + R + T)


@pytest.mark.parametrize("neighbours", (False, True))
@pytest.mark.parametrize("D,R,skew,wide", ((64, 64, 2, 0), (64, 64, 0, 3), (128, 8, 0, 0), (66, 34, 0, 0), (5, 4, 0, 0), (1, 0, 0, 0), (512, 512, 0, 0), (300, 250, 2, 1)))
def test_rows_of_any_width_and_alignment(cq, neighbours, D, R, skew, wide):  # noqa: F811
    for T, Hq, H in ((1, 4, 1), (33, 9, 3)):
        case(cq, T, Hq, H, D, R, "bf16", neighbours=neighbours, first=1000, seed=D + R, skew=skew, wide=wide)


@pytest.mark.parametrize("T,Hq,H", ((3000, 8, 2), (1, 72, 8), (300, 1, 1), (2500, 40, 40)))
def test_many_tokens_and_heads(cq, T, Hq, H):  # noqa: F811
    case(cq, T, Hq, H, 64, 64, "f16", seed=T)
    case(cq, T, Hq, H, 64, 32, "bf16", norm=False, neighbours=True, seed=T)


@pytest.mark.parametrize("first", (0, 1000003, (1 << 31) + 5, -70000, 1 << 40))
def test_far_positions(cq, first):  # noqa: F811
    case(cq, 40, 4, 2, 128, 128, "f16", first=first, weights=False)
    case(cq, 40, 4, 2, 66, 66, "f16", first=first, weights=False)


@pytest.mark.parametrize("D", (128, 130))
@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_rows_whose_squares_fp32_cannot_hold(cq, D, dtype):  # noqa: F811
    t = DT[dtype]
    x = normal((6, 3, D), 3, t).cuda()
    x[0] = torch.finfo(t).max
    x[1] = x[1] * (1e-5 if dtype == "f16" else 1e-30)
    x[2] = 0
    x[3] = torch.finfo(t).tiny
    x[4, 1] = x[4, 1] * (100.0 if dtype == "f16" else 1e25)
    positions, freq = torch.arange(6, device="cuda"), cq.rotation_freq(D - D % 4)
    for eps in (1e-6, 1e-30, 1e10):
        got = cq.norm_rotate(x, x, positions, freq, eps=eps)
        for g in got:
            compare(g, x, None, positions, freq, eps, False)
    a = cq.norm_rotate(x, x, positions, freq)[0]
    y = x.clone()
    y[4, 0] = torch.finfo(t).max                                 # another head's values do not matter
    assert torch.equal(cq.norm_rotate(y, y, positions, freq)[0][4, 1:], a[4, 1:])
    zero = cq.norm_rotate(x[2:3], x[2:3], positions[:1], freq, eps=0.0)[0]
    assert bool(torch.isnan(zero).all())                        # 0 / 0


def test_infinities_and_nan_stay_in_their_rows(cq):  # noqa: F811
    for D in (64, 66):
        x = normal((4, 4, D), 4, torch.bfloat16).cuda()
        positions, freq = torch.arange(4, device="cuda"), cq.rotation_freq(D)
        want = cq.norm_rotate(x, x, positions, freq)[0]
        for bad in (math.inf, math.nan):
            y = x.clone()
            y[1, 2, 5] = bad
            got = cq.norm_rotate(y, y, positions, freq)[0]
            assert bool(torch.isnan(got[1, 2, 5])) and (bad == math.inf or bool(torch.isnan(got[1, 2]).all()))
            got[1, 2] = want[1, 2]
            assert torch.equal(got, want)
            plain = cq.norm_rotate(y, y, positions, freq, eps=None)[0]
            off = ~torch.isfinite(plain[1, 2])
            assert bool(off[5]) and bool(off[5 + D // 2]) and int(off.sum()) == 2


def test_empty_calls_streams_and_graphs(cq):  # noqa: F811
    freq = cq.rotation_freq(64)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    a, b = cq.norm_rotate(none, none[:, :2], torch.empty(0, dtype=torch.int64, device="cuda"), freq)
    assert a.shape == (0, 4, 64) and b.shape == (0, 2, 64)
    x = normal((50, 6, 64), 5, torch.bfloat16).cuda()
    q, k = x.split((4, 2), dim=1)
    positions = torch.arange(50, device="cuda")
    a, b = cq.norm_rotate(q, k[:, :0], positions, freq)
    want = cq.norm_rotate(q, k, positions, freq)
    assert b.shape == (50, 0, 64) and torch.equal(a, want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cq.norm_rotate(q, k, positions, freq)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(m, n) for m, n in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = cq.norm_rotate(q, k, positions, freq)
    for moved in (0, 100):                                       # positions are read at each replay
        positions += moved
        graph.replay()
        assert all(torch.equal(m, n) for m, n in zip(held, cq.norm_rotate(q, k, positions, freq)))
    del graph


def test_binding_refuses(cq):  # noqa: F811
    x = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    positions, freq, w = torch.arange(5, device="cuda"), cq.rotation_freq(64), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(k=x.half()), dict(k=x[:4]), dict(k=x[..., :32]), dict(positions=positions.int()), dict(positions=positions[:4]), dict(freq=freq.float()),
                dict(freq=freq[None]), dict(freq=freq.cpu()), dict(q_weight=w.float()), dict(k_weight=w[:32]), dict(q=x.transpose(1, 2)), dict(eps=-1.0),
                dict(eps=math.nan), dict(eps=None, q_weight=w), dict(out=(x, x.half())), dict(out=(x[:4], x))):
        a = {**dict(q=x, k=x, positions=positions, freq=freq), **bad}
        with pytest.raises(ValueError):
            cq.norm_rotate(**a)
    with pytest.raises(TypeError):
        cq.norm_rotate(x.float(), x, positions, freq)
    with pytest.raises(cq.CQError):
        cq.norm_rotate(x, x, positions, cq.rotation_freq(128))           # more channels than a head has
    with pytest.raises(cq.CQError):
        wide = torch.zeros(5, 1, 520, dtype=torch.bfloat16, device="cuda")
        cq.norm_rotate(wide, wide, positions, freq)
