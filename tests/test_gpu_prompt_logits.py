"""Prompt attention with logits far from 0: where a logit's own rounding in fp32 is more than a weight can bear.

All channels of a query hold a power of two, all of a key one number b_j of at most 11 bits, so that a product q . k_j = D a b_j is exact in fp32
whatever the order of its sum.  Neighbouring values of b_j lie 2^-7 (bf16) or 2^-10 (fp16) apart, which at the sizes below is a difference
of 250 or more between logits: a key that is not the largest has no weight that fp32 holds (e^-104 < 2^-150), and those equal to the largest have
equal weights.  So the result is the mean of v over the largest, off by
  the sums' n 2^-23 and 2^x's 2^-22 in numerator and denominator: (n 2^-22 + 2^-20) of the mean of |v|
  the weights' rounding to the dtype, which their sum has not: U of the mean of |v|.  (A weight of the largest is a power of two only where
  its exponent is 0 or a whole number.  Below 2^20 that is c L - ref in one rounding with ref = fl(c L), so up to half a step of c L: 2^(2^-5) at most.)
  one rounding to the dtype: U of itself, or half a subnormal step
and the logarithm of the sum is its largest logit L, rounded by the factor in base 2 (2^-24), the product with it, the sum, ln 2 (2^-24) and
its product: 2^-21 |L|, and the sum's n 2^-23 + 2^-20.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from test_gpu_prompt import starts
from test_gpu_serve import DT, TINY, UNIT, cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu

BITS = {"f16": 10, "bf16": 7}                                   # of a mantissa, its first one not counted


def numbers(kind, n, dtype, size):
    """n numbers of the dtype between `size` (a power of two) and twice that, for the keys."""
    steps = 1 << BITS[dtype]
    at = torch.arange(n)
    if kind == "rising":
        r = at * (steps - 1) // max(n - 1, 1)
    elif kind == "falling":
        r = (steps - 1) - at * (steps - 1) // max(n - 1, 1)
    elif kind == "one":
        r = torch.where(at == n // 3, steps - 3, 5)
    else:
        r = torch.randint(0, steps, (n,), generator=torch.Generator().manual_seed(n))
    return (size * (1 + r.double() / steps)).to(DT[dtype])


def expect(logits, v):
    """(out, lse, mean of |v|) of rows of logits [n, m] (-infinity: not seen) over v [m, D], in 64 bits."""
    top = logits.max(axis=1, keepdims=True)
    p = np.exp(logits - top)
    total = p.sum(axis=1, keepdims=True)
    return p @ v / total, (top + np.log(total))[:, 0], p @ np.abs(v) / total


def check(cq, dtype, D, a, b, q_lens, k_lens, heads=(2, 1), scale=None):  # noqa: F811
    Hq, H = heads
    scale = D ** -0.5 if scale is None else scale
    q = torch.full((sum(q_lens), Hq, D), float(a), dtype=DT[dtype], device="cuda")
    k = b.cuda()[:, None, None].expand(-1, H, D).contiguous()
    v = normal((sum(k_lens), H, D), 5, DT[dtype], outliers=False).cuda()
    lse = torch.empty(sum(q_lens), Hq, device="cuda")
    got = cq.prompt_attention(q, k, v, starts(q_lens), starts(k_lens), scale=scale, lse=lse).cpu().double().numpy()
    lse = lse.cpu().double().numpy()
    q0 = k0 = 0
    for n, m in zip(q_lens, k_lens):
        logits = np.repeat((scale * D * float(a) * b[k0:k0 + m].double().numpy())[None], n, axis=0)
        logits[np.arange(m)[None] > (m - n + np.arange(n))[:, None]] = -np.inf
        assert np.abs(logits[np.isfinite(logits)]).min() > 2.0 ** 17
        for h in range(Hq):
            out, ls, mag = expect(logits, v[k0:k0 + m, h * H // Hq].cpu().double().numpy())
            tol = (m * 2.0 ** -22 + 2.0 ** -20 + UNIT[DT[dtype]]) * mag
            tol = tol + UNIT[DT[dtype]] * (np.abs(out) + tol) * 1.001 + TINY[DT[dtype]]
            off = np.abs(got[q0:q0 + n, h] - out)
            assert (off <= tol).all(), (h, float((off / tol).max()), np.argwhere(~(off <= tol))[:5])
            off = np.abs(lse[q0:q0 + n, h] - ls)
            assert (off <= 2.0 ** -21 * np.abs(ls) + m * 2.0 ** -23 + 2.0 ** -20).all(), (h, np.argwhere(~(off <= 2.0 ** -21 * np.abs(ls)))[:5])
        q0, k0 = q0 + n, k0 + m


# q . k: the power of two in the queries and the least in the keys.  (D = 128 and the usual factor: logits between 1.8e5 and 1e10; D = 64 half of that.)
SIZES = {"f16": ((2.0 ** 3, 2.0 ** 12), (2.0 ** 6, 2.0 ** 12), (2.0 ** 9, 2.0 ** 13), (2.0 ** 12, 2.0 ** 13), (2.0 ** 15, 2.0 ** 14)),
         "bf16": ((2.0 ** 3, 2.0 ** 12), (2.0 ** 9, 2.0 ** 13), (2.0 ** 12, 2.0 ** 13), (2.0 ** 20, 2.0 ** 15), (2.0 ** 50, 2.0 ** 40))}


@pytest.mark.parametrize("sign", (1, -1))
@pytest.mark.parametrize("kind", ("rising", "falling", "one", "any"))
@pytest.mark.parametrize("dtype,size", [(d, s) for d in SIZES for s in SIZES[d]])
def test_the_largest_key_has_the_weight(cq, dtype, size, kind, sign):  # noqa: F811
    a, least = size
    for D, lens in ((128, [1]), (64, [300]), (128, [1, 200, 7])):
        check(cq, dtype, D, sign * a, numbers(kind, sum(lens), dtype, least), lens, lens)


@pytest.mark.parametrize("sign", (1, -1))
@pytest.mark.parametrize("kind", ("rising", "falling", "one", "any"))
@pytest.mark.parametrize("dtype,size", [(d, s) for d in SIZES for s in SIZES[d]])
def test_with_the_keys_split_over_several_ctas(cq, dtype, size, kind, sign):  # noqa: F811
    a, least = size
    assert cq.prompt_attention_workspace_bytes(1, 5, 6000, 2, 1, 128) > 0
    check(cq, dtype, 128, sign * a, numbers(kind, 6000, dtype, least), [5], [6000])


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
def test_equal_keys_share_the_weight(cq, dtype):  # noqa: F811
    for a, least in SIZES[dtype]:
        check(cq, dtype, 64, a, torch.full((333,), least * 1.5, dtype=DT[dtype]), [333], [333])


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("Tk", (150, 6000))
def test_a_row_beside_rows_of_large_logits_keeps_its_bits(cq, dtype, Tk):  # noqa: F811
    q, k, v = (normal((n, h, 128), 6 + h, DT[dtype], outliers=False).cuda() for n, h in ((20, 4), (Tk, 2), (Tk, 1)))
    v = v.expand(-1, 2, -1).contiguous()
    at = starts([20]), starts([Tk])
    want = cq.prompt_attention(q, k, v, *at, scale=8.0)
    big = q.clone()
    big[7, 2] *= 2.0 ** 13                                      # (largest logits of some 2e6; 8 times 2^13 is an fp16)
    big[11, 1] *= 2.0 ** 13
    got = cq.prompt_attention(big, k, v, *at, scale=8.0)
    same = torch.ones(20, 4, dtype=torch.bool, device="cuda")
    same[7, 2] = same[11, 1] = False
    assert torch.equal(got[same], want[same]) and bool(torch.isfinite(got).all())


@pytest.mark.parametrize("Tk", (260, 6000))
def test_a_logit_that_leaves_the_range_is_infinite(cq, Tk):  # noqa: F811
    """As a finite one, 2e37, it still decides; times 30 it makes the rows that see it NaN."""
    q = torch.full((3, 1, 64), 2.0 ** 60, dtype=torch.bfloat16, device="cuda")
    k = torch.ones(Tk, 1, 64, dtype=torch.bfloat16, device="cuda")
    v = normal((Tk, 1, 64), 9, torch.bfloat16, outliers=False).cuda()
    k[Tk - 2] = 2.0 ** 58                                       # seen by the last two
    at = starts([3]), starts([Tk])
    got = cq.prompt_attention(q, k, v, *at)
    assert torch.equal(got[1], v[Tk - 2]) and torch.equal(got[2], v[Tk - 2]) and bool(torch.isfinite(got[0]).all())
    got = cq.prompt_attention(q, k, v, *at, scale=30.0)
    assert bool(torch.isfinite(got[0]).all()) and bool(torch.isnan(got[1:]).all())
