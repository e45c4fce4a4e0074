"""Adapters: the second halves of A x, and that infinities and NaN beside a row, a token or an adapter stay where they are.

The first.  Every token has one element that is not 0 and every row of B two, so that A x is a product of two 16-bit numbers (exact in
fp32) and the second product has two terms, four with the halves; y is zeros in fp32.  Tolerance, relative to |scale| sum_r |B_r h_r|: the
halves keep h to U^2 of itself (U half an ulp at 1 of the dtype) and, in fp16, to 2^-24 of the token's largest |h|, times |scale| sum_r |B_r|;
three additions in fp32 at 2^-23, the factors' products and the result 2^-22.  Without the second halves a result is off by up to U.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from test_gpu_adapter import adapters, some_index, tokens
from test_gpu_serve import DT, UNIT, cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("R", (8, 16, 72, 128))
@pytest.mark.parametrize("T", (5, 70, 300))
@pytest.mark.parametrize("K,N", ((520, 264), (513, 261)))
def test_both_halves_of_the_inner_product_count(cq, dtype, R, T, K, N):  # noqa: F811
    n, g = 3, torch.Generator().manual_seed(T + R + K)
    ad = adapters(cq, n, K, N, R, dtype, R + T)
    B = torch.zeros(n, N, R)
    at = torch.arange(N)
    for shift in (0, 5):
        B[:, at, (at + shift) % R] = torch.randn(n, N, generator=g)
    ad = cq.Adapters(ad.A, B.to(DT[dtype]).cuda(), ad.scale)
    x = torch.zeros(T, K)
    x[torch.arange(T), torch.randint(0, K, (T,), generator=g)] = 1 + torch.rand(T, generator=g)
    x = x.to(DT[dtype]).cuda()
    y, U = torch.zeros(T, N, device="cuda"), UNIT[DT[dtype]]
    for kind in ("mixed", "one", "turns"):
        index = some_index(T, n, 3, kind)
        got = cq.adapter_add(y, x, ad, index).cpu().double().numpy()
        shows = False
        for t, a in enumerate(index.tolist()):
            if not 0 <= a < n:
                continue
            h = ad.A[a].cpu().double().numpy() @ x[t].cpu().double().numpy()
            Ba, s = ad.B[a].cpu().double().numpy(), float(ad.scale[a])
            want, size = s * (Ba @ h), abs(s) * (np.abs(Ba) @ np.abs(h))
            tol = (U * U + 3 * 2.0 ** -23 + 2.0 ** -22) * size + (2.0 ** -24 * abs(s) * np.abs(Ba).sum(axis=1) * np.abs(h).max() if dtype == "f16" else 0.0)
            off = np.abs(got[t] - want)
            assert (off <= tol).all(), (kind, t, float((off / np.maximum(tol, 1e-300)).max()))
            first = torch.from_numpy(h / 2.0 ** math.floor(math.log2(np.abs(h).max()))).to(DT[dtype]).double().numpy() * 2.0 ** math.floor(math.log2(np.abs(h).max()))
            shows = shows or bool((np.abs(s * (Ba @ first) - want) > 8 * tol).any())
        assert shows                                            # the first halves alone would have been seen


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("R", (16, 72))
@pytest.mark.parametrize("T", (5, 40, 100, 300))
@pytest.mark.parametrize("K,N", ((520, 264), (513, 255), (2060, 1003)))
def test_infinities_and_nan_stay_where_they_are(cq, dtype, R, T, K, N):  # noqa: F811
    """In the elements beside a row above all: rows that begin in the middle of words share one with the row before."""
    y, x = tokens(T, K, N, dtype, T + K)
    ad = adapters(cq, 3, K, N, R, dtype, R)
    t = T // 2
    for kind in ("mixed", "turns", "one"):
        index = some_index(T, 3, 8, kind)
        index[t - 1], index[t], index[t + 1] = 0, 1, 2
        if kind == "one":
            index[:] = 1
        want = cq.adapter_add(y, x, ad, index)
        mine = torch.zeros(T, dtype=torch.bool, device="cuda")
        mine[t - 1] = mine[t + 1] = True
        for bad in (math.inf, math.nan):
            x2, y2 = x.clone(), y.clone()
            x2[t - 1, K - 1] = x2[t + 1, 0] = bad
            got = cq.adapter_add(y, x2, ad, index)
            assert torch.equal(got[~mine], want[~mine]) and not bool(torch.isfinite(got[mine]).any())
            y2[t - 1, N - 1] = y2[t + 1, 0] = bad
            got = cq.adapter_add(y2, x, ad, index)
            assert not bool(torch.isfinite(got[t - 1, N - 1])) and not bool(torch.isfinite(got[t + 1, 0]))
            got[t - 1, N - 1], got[t + 1, 0] = want[t - 1, N - 1], want[t + 1, 0]
            assert torch.equal(got, want)
            own = index == 1
            A, B = ad.A.clone(), ad.B.clone()
            A[1, 0, 0] = A[1, R - 1, K - 1] = bad
            got = cq.adapter_add(y, x, cq.Adapters(A, ad.B, ad.scale), index)
            assert torch.equal(got[~own], want[~own]) and not bool(torch.isfinite(got[own]).any())
            B[1, 0, 0] = B[1, N - 1, R - 1] = bad
            got = cq.adapter_add(y, x, cq.Adapters(ad.A, B, ad.scale), index)
            assert not bool(torch.isfinite(got[own][:, 0]).any()) and not bool(torch.isfinite(got[own][:, N - 1]).any())
            got[:, 0], got[:, N - 1] = want[:, 0], want[:, N - 1]
            assert torch.equal(got, want)
