"""Attention over the cache with logits far from 0: where a logit's own rounding in fp32 is more than a probability can bear.

All channels of a query hold a power of two, all of a key one number b_j of 8 bits, whose codes are all the largest: a logit is one product of
the token's scale and factors.  Neighbouring b_j lie 2^-7 of them apart, at the sizes below 1000 or more between logits, so that a key
that is not the largest has no probability that fp32 holds, and those equal to the largest have equal ones.  The result is the mean of their
values, off by a probability's one rounding to fp16 (2^-11, and 2^-11 for its scale in the row's units), the sums' n 2^-22 + 2^-20, and one
rounding to the dtype.  The logarithm of the sum: its largest logit L, a product of six factors in fp32: 2^-21 |L|.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_serve import DT, TINY, UNIT, cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu

# the power of two in the queries and the least number in the keys
SIZES = {"f16": ((2.0 ** 6, 2.0 ** 12), (2.0 ** 12, 2.0 ** 13), (2.0 ** 15, 2.0 ** 14), (2.0 ** 15, 2.0 ** 15)),
         "bf16": ((2.0 ** 12, 2.0 ** 13), (2.0 ** 20, 2.0 ** 15), (2.0 ** 40, 2.0 ** 30))}


def numbers(kind, n):
    """n numbers from 1 to 2, with 7 bits behind the first."""
    at = torch.arange(n)
    if kind == "rising":
        r = at * 126 // max(n - 1, 1)
    elif kind == "falling":
        r = 126 - at * 126 // max(n - 1, 1)
    else:
        r = torch.randint(0, 127, (n,), generator=torch.Generator().manual_seed(n))
    return 1 + r.double() / 128


def attend(cq, dtype, D, bits, Hq, Lq, q, k, v, lens, page=64):  # noqa: F811
    """(out, lse, what the cache stands for); k, v [n, D] of one sequence after another, one key head; q a number or [B, Lq, Hq, D]."""
    n, pages = k.shape[0], [-(-m // page) for m in lens]
    cache = cq.KVCache.empty(sum(pages), page, 1, D, bits)
    table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
    slots, first = [], 0
    for b, m in enumerate(lens):
        table[b, :pages[b]] = torch.arange(first, first + pages[b])
        slots.append(torch.arange(m) + first * page)
        first += pages[b]
    slots = torch.cat(slots).cuda()
    cq.kv_write(cache, k[:, None].to(DT[dtype]).cuda(), v[:, None].to(DT[dtype]).cuda(), slots)
    kk, vv = cq.kv_read(cache, slots, torch.float32)
    if not torch.is_tensor(q):
        q = torch.full((len(lens), Lq, Hq, D), q, dtype=DT[dtype], device="cuda")
    lse = torch.empty(q.shape[:3], device="cuda")
    out = cq.kv_attention(q, cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), lse=lse)
    assert n == sum(lens)
    return out, lse, kk[:, 0].cpu().double().numpy(), vv[:, 0].cpu().double().numpy()


def check(cq, dtype, D, bits, Hq, Lq, a, b, lens):  # noqa: F811
    k = b[:, None].expand(-1, D)
    v = normal((len(b), D), 5, torch.float32, outliers=False)
    out, lse, kk, vv = attend(cq, dtype, D, bits, Hq, Lq, a, k, v, lens)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    first = 0
    for s, m in enumerate(lens):
        l = float(a) * kk[first:first + m].sum(axis=1) * D ** -0.5
        for i in range(Lq):
            sees = m - Lq + i + 1
            if sees <= 0:
                assert (out[s, i] == 0).all() and (lse[s, i] == -np.inf).all()
                continue
            top = l[:sees].max()
            best = l[:sees] >= top - 1e-6 * abs(top)             # (equal numbers are equal here up to the 64-bit sum)
            part = vv[first:first + sees][best]
            want, mag = part.mean(axis=0), np.abs(part).mean(axis=0)
            tol = (2.0 ** -10 + sees * 2.0 ** -22 + 2.0 ** -20) * mag
            tol = tol + UNIT[DT[dtype]] * (np.abs(want) + tol) * 1.001 + TINY[DT[dtype]]
            off = np.abs(out[s, i] - want[None])
            assert (off <= tol).all(), (s, i, float((off / tol).max()), np.argwhere(~(off <= tol))[:4])
            assert (np.abs(lse[s, i] - (top + np.log(best.sum()))) <= 2.0 ** -21 * abs(top) + sees * 2.0 ** -23 + 2.0 ** -20).all(), (s, i)
        first += m


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("kind", ("rising", "falling", "any"))
@pytest.mark.parametrize("dtype,size", [(d, s) for d in SIZES for s in SIZES[d]])
def test_the_largest_key_has_the_probability(cq, dtype, size, kind, bits):  # noqa: F811
    a, least = size
    for D, Hq, Lq, lens in ((128, 1, 1, [1]), (128, 4, 2, [300]), (64, 8, 3, [65, 2, 700]), (64, 6, 4, [200]), (64, 8, 4, [100]), (128, 2, 1, [6000])):
        for sign in (1, -1):
            check(cq, dtype, D, bits, Hq, Lq, sign * a, numbers(kind, sum(lens)) * least, lens)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("n", (150, 5000))
def test_a_row_beside_rows_of_large_logits_keeps_its_bits(cq, dtype, n, bits):  # noqa: F811
    k, v = normal((n, 128), 1, torch.float32, False) * 60, normal((n, 128), 2, torch.float32, False)
    q = normal((1, 2, 8, 128), 3, DT[dtype], False).cuda() / 16
    big = q.clone()
    big[0, 0, 3] *= 2.0 ** 16
    big[0, 1, 6] *= 2.0 ** 16
    want, got = (attend(cq, dtype, 128, bits, 8, 2, t, k, v, [n])[0] for t in (q, big))
    same = torch.ones(2, 8, dtype=torch.bool, device="cuda")
    same[0, 3] = same[1, 6] = False
    assert torch.equal(got[0][same], want[0][same]) and bool(torch.isfinite(got).all())


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
def test_value_scales_of_any_size_beside_large_logits(cq, dtype):  # noqa: F811
    """The row's units follow the probability times the value's scale, not the logit."""
    n, D = 200, 64
    b = numbers("rising", n) * 2.0 ** 14
    for size in (1e-4, 1.0, 1e4):
        v = normal((n, D), 7, torch.float32, False) * torch.logspace(0, -2, n)[:, None] * size
        k = b[:, None].expand(-1, D)
        out, _, kk, vv = attend(cq, dtype, D, 8, 4, 2, 2.0 ** 15, k, v, [n])
        for i in range(2):
            l = kk[:n - 1 + i].sum(axis=1)
            best = l >= l.max() * (1 - 1e-6)
            want, mag = vv[:n - 1 + i][best].mean(axis=0), np.abs(vv[:n - 1 + i][best]).mean(axis=0)
            tol = (2.0 ** -10 + n * 2.0 ** -22 + 2.0 ** -20) * mag
            tol = tol + UNIT[DT[dtype]] * (np.abs(want) + tol) * 1.001 + TINY[DT[dtype]]
            assert (np.abs(out[0, i].cpu().double().numpy() - want[None]) <= tol).all(), (size, i)
