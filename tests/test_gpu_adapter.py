"""Low-rank adapters on the GPU against the formula in 64 bits.

Tolerance (U half an ulp at 1 of y's dtype, inner_r = sum_k |A_rk x_k|, reach = |scale| sum_r |B_r| inner_r): the K <= 8192 products of a row are added
in fp32, in pieces of 16 by the tensor cores and at most 600 pieces and parts one after the other: 2^-12 inner_r bounds their roundings
(each at most 2^-23 of the sum of magnitudes); the two halves of h keep it to 2^-16 of itself and 2^-24 of the token's largest, at most
max_r inner_r; R <= 128 products more: 2^-16.  In all 2^-11 reach + 2^-23 |scale| sum_r |B_r| max_r inner_r.  The result is rounded once: U, or half a
subnormal step.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from guards import Arena
from test_gpu_serve import DT, TINY, UNIT, cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


def definition(y, x, A, B, scale, index):
    y, x, A, B = (t.cpu().double().numpy() for t in (y, x, A, B))
    scale = np.ones(len(A)) if scale is None else scale.cpu().double().numpy()
    out, tol = y.copy(), np.zeros(y.shape)
    for t, a in enumerate(index.tolist()):
        if 0 <= a < len(A):
            h, inner = A[a] @ x[t], np.abs(A[a]) @ np.abs(x[t])
            out[t] += scale[a] * (B[a] @ h)
            Ba = np.abs(B[a])
            tol[t] = abs(scale[a]) * (2.0 ** -11 * (Ba @ inner) + 2.0 ** -23 * Ba.sum(axis=1) * (inner.max() if inner.size else 0))
    return out, tol


def adapters(cq, n, K, N, R, dtype, seed, scaled=True):  # noqa: F811
    A = (normal((n, R, K), seed, torch.float32, False) / math.sqrt(max(K, 1))).to(DT[dtype]).cuda()
    B = (normal((n, N, R), seed + 1, torch.float32, False) / math.sqrt(R)).to(DT[dtype]).cuda()
    return cq.Adapters(A, B, (0.25 + torch.rand(n, generator=torch.Generator().manual_seed(seed))).cuda() if scaled else None)


def check(cq, y, x, ad, index, out=None):  # noqa: F811
    want, tol = definition(y, x, *ad, index)
    got = cq.adapter_add(y, x, ad, index, out=out)
    tol = tol + UNIT[y.dtype] * (np.abs(want) + tol) * 1.001 + TINY[y.dtype]
    off = np.abs(got.cpu().double().numpy() - want)
    assert (off <= tol).all(), (float((off / tol).max()), np.argwhere(off > tol)[:5])
    bare = [t for t, a in enumerate(index.tolist()) if not 0 <= a < len(ad.A)]
    assert torch.equal(got[bare], y[bare])
    return got


def tokens(T, K, N, dtype, seed, y_dtype=None):
    return normal((T, N), seed, torch.float32, False).to(y_dtype or DT[dtype]).cuda(), normal((T, K), seed + 1, DT[dtype]).cuda()


def some_index(T, n, seed, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "mixed":
        i = torch.randint(-1, n, (T,), generator=g)
    elif kind == "runs":
        i = torch.arange(T) * 5 // max(T, 1) % n
    elif kind == "one":
        i = torch.full((T,), n - 1)
    else:
        i = torch.arange(T) % n
    return i.to(torch.int32).cuda()


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("R", (8, 16, 24, 32, 40, 64, 96, 128))
def test_ranks(cq, dtype, R):  # noqa: F811
    for T, K, N in ((1, 512, 264), (70, 1032, 300), (200, 1032, 296)):
        y, x = tokens(T, K, N, dtype, R)
        check(cq, y, x, adapters(cq, 5, K, N, R, dtype, R + 1), some_index(T, 5, R, "mixed"))


@pytest.mark.parametrize("kind", ("mixed", "runs", "one", "turns"))
@pytest.mark.parametrize("T,n", ((1, 1), (2, 3), (31, 4), (33, 40), (63, 64), (64, 70), (65, 1), (129, 2), (333, 9), (1000, 100)))
def test_batches(cq, kind, T, n):  # noqa: F811
    K, N = 264, 136
    y, x = tokens(T, K, N, "bf16", T)
    check(cq, y, x, adapters(cq, n, K, N, 16, "bf16", n), some_index(T, n, T, kind))


@pytest.mark.parametrize("K,N", ((1, 1), (7, 9), (31, 33), (100, 257), (513, 255), (2060, 1003), (4100, 8), (0, 40)))
def test_odd_widths(cq, K, N):  # noqa: F811
    for dtype, T in (("f16", 5), ("bf16", 67)):
        y, x = tokens(T, K, N, dtype, K + N)
        check(cq, y, x, adapters(cq, 3, K, N, 16, dtype, K), some_index(T, 3, T, "mixed"))


@pytest.mark.parametrize("T,K,N,n", ((128, 64, 8, 3), (129, 72, 1000, 200), (257, 136, 128, 1), (640, 520, 2056, 130), (511, 2048, 520, 4), (1500, 72, 264, 60)))
@pytest.mark.parametrize("R", (8, 24, 64, 128))
def test_many_tokens(cq, T, K, N, n, R):  # noqa: F811
    """Tiles of 128 tokens with one adapter, a few, or one for each token."""
    y, x = tokens(T, K, N, "bf16", T + R)
    ad = adapters(cq, n, K, N, R, "bf16", n)
    check(cq, y, x, ad, some_index(T, n, R, "mixed"))
    check(cq, y.float(), x, ad, some_index(T, n, R, "runs"))


@pytest.mark.parametrize("T,n", ((128, 1), (128, 128), (300, 90), (1200, 33)))
def test_clusters_that_share_out_a_tiles_adapters(cq, T, n):  # noqa: F811
    for R in (8, 16, 64):
        y, x = tokens(T, 2056, 264, "f16", n + R)
        for kind in ("turns", "one"):
            check(cq, y, x, adapters(cq, n, 2056, 264, R, "f16", R), some_index(T, n, n, kind))


@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("N", (1, 127, 128, 129, 255, 258, 1003, 20011))
def test_many_tokens_whose_rows_begin_anywhere(cq, N, dtype):  # noqa: F811
    """Rows at every place of a word, ends inside tiles, in place, and results that begin elsewhere than y."""
    T, K, n = 300, 72, 5
    y, x = tokens(T, K, N, "bf16", N)
    y = y.to({"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype])
    ad, index = adapters(cq, n, K, N, 16, "bf16", N), some_index(T, n, N, "mixed")
    check(cq, y, x, ad, index)
    for first, pitch in ((0, N + 1), (1, N + 2), (3, N + 4)):
        room = torch.full((T, pitch + 3), 7.0, dtype=y.dtype, device="cuda")
        room[:, first:first + N] = y
        here = room[:, first:first + N]
        check(cq, here, x, ad, index, out=torch.empty(T, N, dtype=y.dtype, device="cuda"))
        check(cq, y, x, ad, index, out=here)
        room[:, first:first + N] = y
        want = cq.adapter_add(y, x, ad, index)
        cq.adapter_add(here, x, ad, index, out=here)
        assert torch.equal(here, want)
        assert bool((room[:, :first] == 7).all()) and bool((room[:, first + N:] == 7).all())


def test_long_contractions_and_wide_results(cq):  # noqa: F811
    for T, K, N, R in ((3, 8192, 6000, 16), (90, 8200, 2048, 64), (150, 8192, 2048, 128)):
        y, x = tokens(T, K, N, "bf16", T)
        check(cq, y, x, adapters(cq, 4, K, N, R, "bf16", T), some_index(T, 4, T, "runs"))


@pytest.mark.parametrize("T", (40, 300))
def test_results_of_other_types_strides_and_in_place(cq, T):  # noqa: F811
    K, N = 520, 264
    ad, index = adapters(cq, 3, K, N, 16, "f16", 1), some_index(T, 3, 2, "mixed")
    for y_dtype in (torch.float32, torch.bfloat16, torch.float16):
        for ld, skew in ((N, 0), (N + 8, 0), (N + 3, 0), (N, 2 if y_dtype != torch.float32 else 4)):
            y, x = tokens(T, K, N, "f16", 3, y_dtype)
            ar = Arena()
            ar.add("y", T * ld, y_dtype, skew=skew)
            pitch = K + (8 if ld % 8 == 0 else 5)
            ar.add("x", T * pitch, torch.float16, skew=skew & 2)
            ar.build()
            ar["y"].fill_(9)
            y2, x2 = ar["y"].view(T, ld)[:, :N], ar["x"].view(T, pitch)[:, :K]
            y2.copy_(y)
            x2.copy_(x)
            want = check(cq, y2, x2, ad, index)
            assert cq.adapter_add(y2, x2, ad, index, out=y2) is y2
            ar.check("adapter_add")
            assert torch.equal(y2, want) and bool((ar["y"].view(T, ld)[:, N:] == 9).all())


def test_no_factors_and_empty_calls(cq):  # noqa: F811
    y, x = tokens(20, 64, 72, "bf16", 4)
    check(cq, y, x, adapters(cq, 2, 64, 72, 8, "bf16", 5, scaled=False), some_index(20, 2, 1, "mixed"))
    none = cq.Adapters(torch.empty(0, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 72, 8, dtype=torch.bfloat16, device="cuda"))
    y[0, 0] = -0.0
    got = cq.adapter_add(y, x, none, torch.zeros(20, dtype=torch.int32, device="cuda"))
    assert torch.equal(got.view(torch.int16), y.view(torch.int16))
    assert cq.adapter_add(y[:0], x[:0], none, torch.zeros(0, dtype=torch.int32, device="cuda")).shape == (0, 72)


def test_a_token_depends_on_no_other(cq):  # noqa: F811
    """Other tokens' values, and infinities and NaN in theirs or in another adapter."""
    T, K, N = 130, 520, 264
    y, x = tokens(T, K, N, "bf16", 6)
    ad, index = adapters(cq, 3, K, N, 16, "bf16", 7), some_index(T, 3, 8, "mixed")
    want = cq.adapter_add(y, x, ad, index)
    for bad in (math.inf, math.nan):
        x2, A, B = x.clone(), ad.A.clone(), ad.B.clone()
        x2[50, 3] = bad
        mine = torch.arange(T, device="cuda") == 50
        got = cq.adapter_add(y, x2, ad, index)
        assert torch.equal(got[~mine], want[~mine])
        A[1, 2, 5] = bad
        B[1, 9, 3] = bad
        got = cq.adapter_add(y, x, cq.Adapters(A, B, ad.scale), index)
        other = index != 1
        assert torch.equal(got[other], want[other]) and not bool(torch.isfinite(got[~other]).any())
        B2 = ad.B.clone()
        B2[1, 9, 3] = bad                                        # one output channel of one adapter
        got = cq.adapter_add(y, x, cq.Adapters(ad.A, B2, ad.scale), index)
        assert not bool(torch.isfinite(got[~other][:, 9]).any())
        got[:, 9] = want[:, 9]
        assert torch.equal(got, want)


@pytest.mark.parametrize("T", (9, 140))
def test_inner_values_beyond_the_types_range(cq, T):  # noqa: F811
    """fp16: |A x| above 65504 and below 2^-24 for whole tokens."""
    K, N, R = 512, 64, 16
    y, x = tokens(T, K, N, "f16", 9)
    ad, index = adapters(cq, 2, K, N, R, "f16", 10), some_index(T, 2, 1, "turns")
    x = x * 0 + torch.randn(T, K, device="cuda").half()
    big = cq.Adapters((ad.A.float() * 20000).half(), (ad.B.float() * 1e-4).half(), ad.scale)
    x[3] *= 100
    y = y.float()
    assert float((big.A[1].float() @ x[3].float()).abs().max()) > 65504
    check(cq, y, x, big, index)
    small = cq.Adapters((ad.A.float() * 1e-4).half(), ad.B, ad.scale * 1e6)
    check(cq, y, (x.float() * 1e-4).half(), small, index)


@pytest.mark.parametrize("T", (100, 500))
def test_equal_calls_give_equal_bits_on_streams_and_from_graphs(cq, T):  # noqa: F811
    K, N = 1024, 520
    y, x = tokens(T, K, N, "bf16", 11)
    ad, index = adapters(cq, 6, K, N, 32, "bf16", 12), some_index(T, 6, 13, "mixed")
    want = cq.adapter_add(y, x, ad, index)
    order = torch.randperm(T, device="cuda")
    check(cq, y[order].contiguous(), x[order].contiguous(), ad, index[order].contiguous())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cq.adapter_add(y, x, ad, index)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    ws = torch.empty(cq.adapter_add_workspace_bytes(T, 32), dtype=torch.uint8, device="cuda")
    graphs, held = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append((cq.adapter_add(y, x, ad, index, workspace=ws), cq.adapter_add(x, y, cq.Adapters(ad.B.transpose(1, 2).contiguous(), ad.A.transpose(1, 2).contiguous()),
                                                                                       index, workspace=ws)))
        graphs.append(g)
    index += 1                                                   # read at each replay
    again = cq.adapter_add(y, x, ad, index)
    for g in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    for h in held:
        assert torch.equal(h[0], again)
    assert not torch.equal(again, want)
    del graphs, g


def test_adapters_whose_offsets_pass_32_bits(cq):  # noqa: F811
    """A and B of more than 2^31 elements each; only a few of them are used."""
    n, K, N, R = 17000, 1024, 1024, 128
    ad = cq.Adapters(torch.zeros(n, R, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, N, R, dtype=torch.bfloat16, device="cuda"))
    assert ad.A.numel() > 1 << 31
    small = adapters(cq, 2, K, N, R, "bf16", 14, scaled=False)
    ad.A[n - 2:], ad.B[n - 2:] = small.A, small.B
    y, x = tokens(7, K, N, "bf16", 15)
    index = some_index(7, 2, 16, "turns")
    assert torch.equal(cq.adapter_add(y, x, ad, index + (n - 2)), check(cq, y, x, small, index))


def test_binding_refuses(cq):  # noqa: F811
    y, x = tokens(6, 64, 72, "bf16", 17)
    ad, index = adapters(cq, 3, 64, 72, 16, "bf16", 18), some_index(6, 3, 1, "turns")
    for bad in (dict(A=ad.A.half()), dict(A=ad.A[:2]), dict(A=ad.A[:, :, :32]), dict(B=ad.B[:, :, :8]), dict(B=ad.B.transpose(1, 2)), dict(A=ad.A.cpu()),
                dict(scale=ad.scale[:2]), dict(scale=ad.scale.double()), dict(index=index.long()), dict(index=index[:5]), dict(y=y[:5]), dict(y=y[:, :64]),
                dict(y=y.t()), dict(out=y.float()), dict(out=y[:5])):
        a = {**dict(y=y, x=x, A=ad.A, B=ad.B, scale=ad.scale, index=index, out=None), **bad}
        with pytest.raises(ValueError):
            cq.adapter_add(a["y"], a["x"], cq.Adapters(a["A"], a["B"], a["scale"]), a["index"], out=a["out"])
    with pytest.raises(TypeError):
        cq.adapter_add(y.double(), x, ad, index)
    with pytest.raises(TypeError):
        cq.adapter_add(y, x.float(), ad, index)
    for R in (4, 12, 136):
        with pytest.raises(cq.CQError):
            cq.adapter_add(y, x, adapters(cq, 3, 64, 72, R, "bf16", 19), index)
    with pytest.raises(cq.CQError):
        cq.adapter_add(y, x, ad, index, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):                              # in place with another pitch
        wide = torch.zeros(8, 80, dtype=torch.bfloat16, device="cuda")
        cq.adapter_add(wide.view(-1)[:432].view(6, 72), x, ad, index, out=wide[:6, :72])
