"""Prompt attention whose weights keep more than 16 bits (`fine`), and the layer's prompts, which attend so.

A result's own rounding hides what its weights lost, so the values here cancel.  Queries and keys hold -1, 0 and 1 (their products are exact), a
few pairs of keys have nearly all the weight, and the second key's value is minus the first one's times the ratio of their weights, rounded to the
dtype: what remains is U (half an ulp at 1) of the weighted mean of |v| (mag) or less, so that its rounding is U^2 mag.

Tolerance, for a row with n visible keys of which `heavy` have weights that fp16 holds, `far` the largest |logit| of those in base 2:
  a weight: two numbers of the dtype, U^2 of itself; fp16 keeps them, times 2^7, to 2^-25 below 2^-14: 2^-32 of the largest.  (The other
      keys, below 2^-32 of the largest each, may be off by all of that.)
  2^x 2^-22; its exponent carries the factor's 2^-24 and one rounding, of at most 2 far + 15: ln 2 (2^-24 far + 2^-24 (2 far + 15)) < 2^-22 (far + 4)
  sums of heavy (bf16: n) terms in fp32, each addition off by 2^-23 of their magnitudes, also where parts of the keys are joined (up to 16 more)
All but the weights' own in numerator and denominator both.
"""
from __future__ import annotations

import functools
import math
import types

import numpy as np
import pytest
import torch

import test_gpu_prompt as whole
import test_gpu_prompt_logits as logits
from test_gpu_prompt import qkv, starts
from test_gpu_serve import DT, TINY, UNIT, cq, normal  # noqa: F401  (cq: the fixture)
from test_gpu_serve_prompts import make

pytestmark = pytest.mark.gpu


def fine(cq):  # noqa: F811
    return types.SimpleNamespace(prompt_attention=functools.partial(cq.prompt_attention, fine=True),
                                 prompt_attention_workspace_bytes=cq.prompt_attention_workspace_bytes)


def pairs(n, D, dtype, seed, places):
    """(one query [D], keys [n, D], values [n, D], logits in 64 bits) with the weight on the pairs of `places`; the factor is 1 / 8."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(0, 2, (D,), generator=g).double() * 2 - 1
    k = -4 * q.repeat(n, 1)                                     # logits of -32 or -64: weights below 2^-50
    for i, at in enumerate(places):                             # logits from 3 to 4.25
        some = torch.randperm(D, generator=g)[:24 + 3 * i % 11]
        k[at] = 0
        k[at, some] = q[some]
    l = (k @ q) / 8
    v = torch.zeros(n, D, dtype=torch.float64)
    for a, b in zip(places[::2], places[1::2]):
        s = torch.randn(D, generator=g).to(DT[dtype]).double()
        v[a], v[b] = s, -(s * torch.exp(l[a] - l[b])).to(DT[dtype]).double()
    return q, k, v, l.numpy()


def expect(l, v, sees, dtype, parts=0):
    """(out, tolerance, what rounding each weight once would give) of a row that sees the first `sees` keys."""
    U, l, v = UNIT[DT[dtype]], l[:sees], v[:sees].numpy()
    p = np.exp(l - l.max())
    once = torch.from_numpy(p).to(DT[dtype]).double().numpy()
    out, mag, top = p @ v / p.sum(), p @ np.abs(v) / p.sum(), np.abs(v).max()
    some = p > 2.0 ** -32
    heavy = int(some.sum()) if dtype == "f16" else sees
    far = np.abs(l[some]).max() / math.log(2)
    tol = (U * U + 2 * (2.0 ** -22 * (far + 5) + (heavy + parts) * 2.0 ** -23)) * mag + sees * 2.0 ** -32 * top
    return out, tol + U * np.abs(out) * 1.001 + TINY[DT[dtype]], once @ v / p.sum()


CASES = ((6, (0, 1, 2, 3, 4, 5)), (130, (3, 64, 63, 100, 127, 128)), (300, (0, 299, 70, 200, 130, 190)), (257, (126, 127, 254, 255)))


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("n,places", CASES)
def test_weights_keep_what_16_bits_lose(cq, dtype, D, n, places):  # noqa: F811
    q, k, v, l = pairs(n, D, dtype, n + D, places)
    dt = DT[dtype]
    got = fine(cq).prompt_attention(q.to(dt).cuda().expand(n, 4, D).contiguous(), k[:, None].to(dt).cuda().expand(n, 2, D).contiguous(),
                                    v[:, None].to(dt).cuda().expand(n, 2, D).contiguous(), starts([n]), scale=0.125).cpu().double().numpy()
    seen = False
    for i in range(n):
        out, tol, once = expect(l, v, i + 1, dtype)
        assert (np.abs(got[i] - out) <= tol).all(), (i, float((np.abs(got[i] - out) / tol).max()))
        seen = seen or bool((np.abs(once - out) > 2 * tol).any())
    assert seen                                                 # one rounding would have shown


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_with_the_keys_split_over_several_ctas(cq, dtype):  # noqa: F811
    n, dt, places = 6000, DT[dtype], (5, 5990, 1000, 3003, 2222, 2223)
    assert cq.prompt_attention_workspace_bytes(1, 2, n, 4, 2, 64) > 0
    q, k, v, l = pairs(n, 64, dtype, 1, places)
    got = fine(cq).prompt_attention(q.to(dt).cuda().expand(2, 4, 64).contiguous(), k[:, None].to(dt).cuda().expand(n, 2, 64).contiguous(),
                                    v[:, None].to(dt).cuda().expand(n, 2, 64).contiguous(), starts([2]), starts([n]), scale=0.125).cpu().double().numpy()
    for i in range(2):
        out, tol, once = expect(l, v, n - 1 + i, dtype, 16)
        assert (np.abs(got[i] - out) <= tol).all(), (i, float((np.abs(got[i] - out) / tol).max()))
        assert dtype == "bf16" or (np.abs(once - out) > 2 * tol).any()          # (bf16: the sums of 6000 terms may be off by as much)


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_the_layers_prompts_attend_so(cq, dtype):  # noqa: F811
    n, dt = 130, DT[dtype]
    q, k, v, l = pairs(n, 64, dtype, 7, CASES[1][1])
    q, k, v = q.to(dt).cuda().expand(n, 4, 64).contiguous(), k[:, None].to(dt).cuda().expand(n, 2, 64).contiguous(), v[:, None].to(dt).cuda().expand(n, 2, 64).contiguous()
    got = make(cq, 1)._attend(q, k, v, [n]).cpu().double().numpy()
    for i in range(n):
        out, tol, _ = expect(l, v[:, 0].cpu().double(), i + 1, dtype)
        assert (np.abs(got[i] - out) <= tol).all(), (i, float((np.abs(got[i] - out) / tol).max()))
    assert torch.equal(make(cq, 1, fine_prompts=False)._attend(q, k, v, [n]), cq.prompt_attention(q, k, v, starts([n])))


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("D", (64, 128))
def test_lengths_and_heads(cq, dtype, D):  # noqa: F811
    for n in (1, 64, 65, 127, 128, 129, 300):
        whole.check(fine(cq), *qkv(n, (4, 2, 2), D, dtype, n), [n])
    whole.check(fine(cq), *qkv(600, (6, 2, 2), D, dtype, 2), [5, 0, 300, 1, 294])
    whole.check(fine(cq), *qkv(40, (8, 2, 2), D, dtype, 3, 5000), [33, 7], [4000, 1000])
    whole.check(fine(cq), *qkv(500, (16, 16, 16), D, dtype, 4), [37 * i % 101 for i in range(10)] + [500 - sum(37 * i % 101 for i in range(10))])


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_what_a_query_does_not_see_has_no_effect(cq, dtype):  # noqa: F811
    whole.test_what_a_query_does_not_see_has_no_effect(fine(cq), dtype, 64, [300, 77])


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_logits_far_from_0(cq, dtype):  # noqa: F811
    for a, least in logits.SIZES[dtype]:
        logits.check(fine(cq), dtype, 128, a, logits.numbers("any", 300, dtype, least), [300], [300])


def test_equal_calls_give_equal_bits_and_graphs_too(cq):  # noqa: F811
    q, k, v = qkv(333, (8, 2, 2), 128, "bf16", 19)
    at = starts([200, 133])
    want = cq.prompt_attention(q, k, v, at, fine=True)
    assert torch.equal(cq.prompt_attention(q, k, v, at, fine=True), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = cq.prompt_attention(q, k, v, at, fine=True)
    got.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    del graph


def test_refusals(cq):  # noqa: F811
    q, k, v = qkv(10, (4, 2, 2), 64, "bf16", 22)
    with pytest.raises(cq.CQError):
        cq.prompt_attention(q, k, v, starts([10]), scale=0.0, fine=True)
    with pytest.raises(ValueError):
        cq.prompt_attention(q, k[:9], v, starts([10]), fine=True)
