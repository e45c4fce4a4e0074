"""Prompt attention and values that are infinities or NaN: rows that see no weight, and keys split over several CTAs."""
from __future__ import annotations

import math

import pytest
import torch

from test_gpu_prompt import qkv, starts
from test_gpu_serve import cq  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fine", (False, True))
@pytest.mark.parametrize("dtype,D", (("bf16", 64), ("f16", 128)))
@pytest.mark.parametrize("n,m", ((1, 1), (100, 100), (300, 300), (4, 6000)))
def test_a_query_whose_logits_are_all_minus_infinity_gets_zeros(cq, dtype, D, n, m, fine):  # noqa: F811
    """Whatever its values are."""
    q, k, v = (t.contiguous() for t in qkv(n, (4, 2, 2), D, dtype, 3, m))
    q[..., 5] = 1
    k[..., 5] = -math.inf
    for bad in (0.0, math.inf, math.nan):
        for at in (0, m // 2, m - 1):
            v2 = v.clone()
            v2[at, :, 3::7] = bad
            lse = torch.empty(n, 4, device="cuda")
            out = cq.prompt_attention(q, k, v2, starts([n]), starts([m]), lse=lse, fine=fine)
            assert bool((out == 0).all()) and bool((lse == -math.inf).all()), (bad, at)


@pytest.mark.parametrize("fine", (False, True))
@pytest.mark.parametrize("dtype,D", (("bf16", 64), ("f16", 128), ("bf16", 128), ("f16", 64)))
@pytest.mark.parametrize("q_lens,k_lens", (([20], [6000]), ([10, 9], [3000, 3100])))
def test_keys_split_over_several_ctas(cq, dtype, D, q_lens, k_lens, fine):  # noqa: F811
    """What a query does not see leaves its bits alone; what it sees shows in its channel."""
    Tq, Tk = sum(q_lens), sum(k_lens)
    assert cq.prompt_attention_workspace_bytes(len(q_lens), Tq, Tk, 4, 2, D) > 0
    q, k, v = (t.contiguous() for t in qkv(Tq, (4, 2, 2), D, dtype, 4, Tk))
    at_q, at_k = starts(q_lens), starts(k_lens)
    want = cq.prompt_attention(q, k, v, at_q, at_k, fine=fine)
    sees = torch.zeros(Tq, Tk, dtype=torch.bool)
    q0 = k0 = 0
    for n, m in zip(q_lens, k_lens):
        for i in range(n):
            sees[q0 + i, k0:k0 + m - n + i + 1] = True
        q0, k0 = q0 + n, k0 + m
    channels = torch.zeros(D, dtype=torch.bool, device="cuda")
    channels[3::7] = True
    for at in sorted({0, 5, 700, 1535, 1536, 2990, 2995, 2999, 3000, Tk - 20, Tk - 12, Tk - 5, Tk - 1}):
        row = sees[:, at].cuda()
        for bad in (math.inf, -math.inf, math.nan):
            v2 = v.clone()
            v2[at, 1, 3::7] = bad
            got = cq.prompt_attention(q, k, v2, at_q, at_k, fine=fine)
            assert torch.equal(got[:, :2], want[:, :2]) and torch.equal(got[~row], want[~row]), (at, bad)
            assert torch.equal(got[row][:, 2:][..., ~channels], want[row][:, 2:][..., ~channels]), (at, bad)
            assert not bool(torch.isfinite(got[row][:, 2:][..., channels]).any()), (at, bad)
        k2 = k.clone()
        k2[at, 1, 3::7] = math.nan
        got = cq.prompt_attention(q, k2, v, at_q, at_k, fine=fine)
        assert torch.equal(got[:, :2], want[:, :2]) and torch.equal(got[~row], want[~row]) and bool(torch.isnan(got[row][:, 2:]).all()), at
