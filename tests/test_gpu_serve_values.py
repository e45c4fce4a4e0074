"""Attention over the cache where tokens' scales differ by many powers of two or are not finite.

What a query does not see has no effect on it, bit for bit: such tests compare with a call on a cache that holds something
ordinary in the same place.  What it does see follows the formula.  Tolerance against 64 bits: the one of test_gpu_serve.py,
    (2 * 2^-11 * 1.1 * reach + 2^-10) * (probability-weighted |v|) + half an ulp of the result,
and, where value scales spread, what the fixed point of the 16-bit probabilities loses: probability times value scale is held in
steps of 2^-24 in units that put the row's largest above 2^4, so a token is off by at most 2^-25 / 2^4 = 2^-29 of the row's largest
(2^-28 with a factor of two for the rounding of references to whole powers of two), times its code.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import serve_reference as ref
from test_gpu_serve import DT, UNIT, build_sequences, cq, make_cache, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


def sequences(cq, lens, H, D, page, bits, col, seed):  # noqa: F811
    """(cache, its host codes, scales and factors, page table on the host)"""
    table, pages = build_sequences(None, lens, page, seed)
    cache, codes, scales, cols, _ = make_cache(cq, pages, page, H, D, bits, col, seed + 1)
    return cache, codes, scales, cols, table


def attend(cq, cache, q, table, lens, **more):  # noqa: F811
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    out = cq.kv_attention(q, cache, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), lse=lse, **more)
    return out, lse


def check_sequence(out, lse, q, table, n, codes, scales, cols, page, scale, dtype, spread=False, light=None):
    """One sequence of a call, out [Lq, Hq, D], against 64 bits.  `light`: a token of so small a probability (below e^-200) that an
    error of its logit does not show; it does not count for `reach`."""
    Lq, Hq, D = q.shape
    H = codes[0].shape[1]
    G = Hq // H
    at = table[:-(-n // page)]
    for h in range(H):
        kv, c_v, s_v = [], None, None
        for i in range(2):
            c = codes[i][at][:, h].reshape(-1, D)[:n].astype(np.float64)
            s = scales[i][at][:, h].reshape(-1)[:n].astype(np.float64)
            f = 1.0 if cols[i] is None else cols[i][h].astype(np.float64)
            kv.append(c * s[:, None] * f)
            if i == 1:
                c_v, s_v, f_v = c, s, f
        heads = np.s_[:, h * G:(h + 1) * G]
        want, want_lse, reach, mag = ref.attention(q[heads].double().cpu().numpy(), kv[0], kv[1], scale)
        if light is not None:
            k = np.delete(kv[0], light, axis=0)
            for i in range(Lq):
                reach[i] = (np.abs(q[i, h * G:(h + 1) * G].double().cpu().numpy()) @ np.abs(k[:n - Lq + i]).T * scale).max(axis=1)
        got = out[heads].double().cpu().numpy()
        bound = (2 * 2.0 ** -11 * 1.1 * reach[..., None] + 2.0 ** -10) * mag + UNIT[DT[dtype]] * np.abs(want) * 1.001 + 2.0 ** -24
        if spread:
            for i in range(Lq):
                m = n - Lq + i + 1
                if m <= 0:
                    continue
                p = np.exp(q[i, h * G:(h + 1) * G].double().cpu().numpy() @ kv[0][:m].T * scale - want_lse[i][:, None])
                bound[i] += 2.0 ** -28 * (p * s_v[:m]).max(axis=1)[:, None] * np.abs(c_v[:m]).sum(axis=0)[None] * f_v
        err = np.abs(got - want)
        assert np.isfinite(got).all() and (err <= bound).all(), f"head {h}: worst {np.nanmax(err / bound)} of the bound"
        fin = np.isfinite(want_lse)
        le = lse[heads].double().cpu().numpy()
        assert np.array_equal(np.isfinite(le), fin)
        assert (np.abs(le - np.where(fin, want_lse, 0))[fin] <= (2.0 ** -11 * 1.1 * reach + 2.0 ** -16 * (1 + np.abs(np.where(fin, want_lse, 0))))[fin]).all()


SHAPES = ((2, 4, 2, 64, 16, 8), (3, 8, 2, 128, 64, 4), (4, 4, 1, 128, 48, 8), (5, 16, 2, 64, 32, 4), (8, 8, 2, 64, 64, 8))


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("Lq,Hq,H,D,page,bits", SHAPES)
@pytest.mark.parametrize("bad", (math.inf, math.nan, 1e30, 3e38))
def test_a_value_that_a_query_does_not_see_has_no_effect(cq, dtype, Lq, Hq, H, D, page, bits, bad):  # noqa: F811
    lens = [Lq, 70, 333, Lq - 1]
    cache, _, _, _, table = sequences(cq, lens, H, D, page, bits, bits == 4, Lq)
    q = normal((len(lens), Lq, Hq, D), 5, DT[dtype], outliers=False).cuda()
    want, want_lse = attend(cq, cache, q, table, lens)
    for b, n in enumerate(lens):
        cache.v_scale[int(table[b, (n - 1) // page]), :, (n - 1) % page] = bad
    got, got_lse = attend(cq, cache, q, table, lens)
    assert torch.equal(got[:, :-1], want[:, :-1])                       # the last query alone sees the last token
    assert torch.equal(got_lse, want_lse)                               # and its probabilities are what they were
    if not math.isfinite(bad):
        assert not bool(torch.isfinite(got[:, -1]).any())


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("bits", (8, 4))
def test_a_small_value_beside_a_huge_one_that_is_not_seen(cq, dtype, bits):  # noqa: F811
    """Two tokens with values near 100 and near the type's largest; the first of two queries sees the first token alone."""
    big = 1e30 if dtype == "bf16" else 6e4
    cache = cq.KVCache.empty(1, 16, 1, 64, bits)
    x = normal((2, 2, 64), 1, torch.float32, outliers=False)
    x[0, 1], x[1, 1] = 100 + x[0, 1], big * (1 + 0.01 * x[1, 1].clamp(-3, 3))
    x = x.to(DT[dtype]).cuda()
    cq.kv_write(cache, x[:, :1], x[:, 1:], torch.arange(2, device="cuda"))
    q = normal((1, 2, 1, 64), 2, DT[dtype], outliers=False).cuda()
    out, _ = attend(cq, cache, q, np.zeros((1, 1), np.int32), [2])
    stored = cq.kv_read(cache, torch.zeros(1, dtype=torch.int64, device="cuda"), torch.float32)[1][0, 0]
    # one token: its probability is 1, and 1 times its scale is rounded to 11 bits
    assert bool(((out[0, 0, 0].float() - stored).abs() <= stored.abs() * (2.0 ** -11 + UNIT[DT[dtype]] * 1.01)).all())


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("Lq,Hq,H,D,page,bits", ((1, 4, 2, 64, 16, 8), (1, 8, 1, 128, 64, 4), (3, 4, 1, 128, 32, 8), (6, 4, 1, 64, 64, 4)))
def test_a_huge_value_of_next_to_no_probability(cq, dtype, Lq, Hq, H, D, page, bits):  # noqa: F811
    """A token with a value scale of 2^40 whose logits lie 300 below the others' leaves their result as it is."""
    n, at = 200, 37
    cache, codes, scales, cols, table = sequences(cq, [n], H, D, page, bits, False, 3)
    q = normal((1, Lq, Hq, D), 4, DT[dtype], outliers=False).abs().clamp(0.5, 2)         # all positive: a key can oppose all queries
    page_at, off = int(table[0, at // page]), at % page
    opposed = -(127 if bits == 8 else 7)
    codes[0][page_at, :, off] = opposed
    cache.k_codes[page_at, :, off] = ref.pack(codes[0][page_at, :, off], bits).cuda()
    # q . k is at most -0.5 D |code| scale, and the softmax's scale D^-1/2
    scales[0][page_at, :, off] = 300 / (0.5 * D * -opposed * D ** -0.5)
    scales[1][page_at, :, off] = 2.0 ** 40
    cache.k_scale[page_at, :, off], cache.v_scale[page_at, :, off] = float(scales[0][page_at, 0, off]), 2.0 ** 40
    out, lse = attend(cq, cache, q.cuda(), table, [n])
    check_sequence(out[0], lse[0], q[0], table[0], n, codes, scales, cols, page, D ** -0.5, dtype, light=at)


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("Lq,Hq,H,D,page,bits", ((1, 4, 2, 64, 16, 8), (4, 8, 2, 128, 64, 4), (2, 8, 1, 128, 48, 8), (7, 4, 1, 64, 64, 4)))
@pytest.mark.parametrize("order", ("up", "down", "mixed"))
def test_value_scales_over_many_powers_of_two(cq, dtype, Lq, Hq, H, D, page, bits, order):  # noqa: F811
    lens = [700, 65, 3]
    cache, codes, scales, cols, table = sequences(cq, lens, H, D, page, bits, True, 11)
    rng = np.random.default_rng(1)
    span = 40 if dtype == "bf16" else 12                                # results have to fit the type
    for b, n in enumerate(lens):
        e = rng.uniform(-span, 10, n)
        e = np.sort(e) if order == "up" else np.sort(e)[::-1] if order == "down" else e
        for j in range(n):
            scales[1][table[b, j // page], :, j % page] = 2.0 ** e[j] / 64
    cache.v_scale.copy_(torch.from_numpy(scales[1]))
    q = normal((len(lens), Lq, Hq, D), 6, DT[dtype], outliers=False)
    out, lse = attend(cq, cache, q.cuda(), table, lens)
    for b, n in enumerate(lens):
        check_sequence(out[b], lse[b], q[b], table[b], n, codes, scales, cols, page, D ** -0.5, dtype, spread=True)


def test_values_near_the_ends_of_the_type(cq):  # noqa: F811
    """One token each, value scales from 2^-118 to 2^120: the result is the value."""
    n = 120
    cache, codes, scales, cols, table = sequences(cq, [1] * n, 1, 64, 16, 8, False, 7)
    for b in range(n):
        scales[1][table[b, 0], 0, 0] = 2.0 ** (-118 + 2 * b)
    cache.v_scale.copy_(torch.from_numpy(scales[1]))
    q = normal((n, 1, 2, 64), 8, torch.bfloat16, outliers=False).cuda()
    out, _ = attend(cq, cache, q, table, [1] * n)
    for b in range(n):
        want = torch.from_numpy(codes[1][table[b, 0], 0, 0] * float(scales[1][table[b, 0], 0, 0])).float().to(torch.bfloat16)
        assert torch.equal(out[b, 0, 0].cpu(), want) and torch.equal(out[b, 0, 1].cpu(), want)


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("col", (False, True))
@pytest.mark.parametrize("Lq,Hq,H,D,page,bits", SHAPES + ((1, 8, 1, 128, 16, 8), (1, 8, 1, 64, 16, 4)))
@pytest.mark.parametrize("bad", (math.inf, -math.inf, math.nan))
def test_a_key_that_is_not_finite_makes_the_queries_that_see_it_nan(cq, dtype, col, Lq, Hq, H, D, page, bits, bad):  # noqa: F811
    """Written through kv_write: such a head has codes 0 and a scale that is not finite, and reads back as NaN."""
    lens = [Lq, 70, 333]
    cache, _, _, _, table = sequences(cq, lens, H, D, page, bits, col, 21)
    q = normal((len(lens), Lq, Hq, D), 22, DT[dtype], outliers=False).cuda()
    want, want_lse = attend(cq, cache, q, table, lens)
    for b, n in ((1, 70), (2, 333)):
        at = n - 1 if b == 1 else n - Lq                              # seen by the last query alone; by all of them
        x = normal((1, H, D), 23, DT[dtype], outliers=False)
        slot = torch.tensor([int(table[b, at // page]) * page + at % page], device="cuda")
        kept = cq.kv_read(cache, slot, torch.float32)[1].to(DT[dtype])
        x[:, 0, 5] = bad                                              # one head of the token
        cq.kv_write(cache, x.cuda(), kept, slot)
        assert bool(torch.isnan(cq.kv_read(cache, slot)[0][0, 0]).all())
    got, got_lse = attend(cq, cache, q, table, lens)
    G = Hq // H
    assert torch.equal(got[0], want[0]) and torch.equal(got_lse[0], want_lse[0])
    assert torch.equal(got[1, :-1], want[1, :-1]) and torch.equal(got_lse[1, :-1], want_lse[1, :-1])
    for rows, lse in ((got[1, -1:, :G], got_lse[1, -1:, :G]), (got[2, :, :G], got_lse[2, :, :G])):
        assert bool(torch.isnan(rows).all()) and bool(torch.isnan(lse).all())
    assert bool(torch.isfinite(got[1:, :, G:]).all())


@pytest.mark.parametrize("dtype,size,scale", (("bf16", 1e-28, 1e-30), ("bf16", 1.0, 1e-46), ("f16", 1.0, 1e-60), ("bf16", 1e-38, 0.1)))
def test_logits_that_vanish_give_the_mean_of_what_is_seen(cq, dtype, size, scale):  # noqa: F811
    """Queries and softmax scales so small that their product is no float: all that a query sees weighs the same."""
    lens, Lq, D, page = [100, 3], 3, 64, 16
    cache, codes, scales, cols, table = sequences(cq, lens, 2, D, page, 8, True, 31)
    q = normal((2, Lq, 4, D), 32, torch.float32, outliers=False).mul(size).to(DT[dtype])
    out, lse = attend(cq, cache, q.cuda(), table, lens, scale=scale)
    for b, n in enumerate(lens):
        check_sequence(out[b], lse[b], q[b], table[b], n, codes, scales, cols, page, scale, dtype)
