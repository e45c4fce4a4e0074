"""Host logic of serve.AttentionLayer on the CPU: what it refuses, which slots it writes, what it calibrates.

The operators are replaced by plain ones (no GPU); their numerics are tested in test_gpu_serve.py and test_gpu_serve_layer.py.
"""
from __future__ import annotations

import types

import pytest
import torch

from paper_2410_07505_b200 import serve

HIDDEN, HEADS, KV, D = 32, 4, 2, 8


class Plain:
    """Stands for the module cq."""

    def __init__(self):
        self.written, self.seen, self.caches = [], [], []
        self.KVCache = types.SimpleNamespace(empty=self.empty)

    def empty(self, pages, page_size, heads, head_dim, bits, *, k_col, v_col, device):
        self.caches.append((pages, page_size, k_col, v_col))
        return "cache"

    fp8_quantize_weight = staticmethod(lambda w: w)
    fp8_linear = staticmethod(lambda x, w: x @ w.t())
    absmax_cols = staticmethod(lambda x: x.abs().amax(0).float())

    def kv_write(self, cache, k, v, slots):
        assert cache == "cache"
        self.written.append(slots.tolist())

    def kv_read(self, cache, slots, dtype):
        return (torch.ones(len(slots), KV, D, dtype=dtype),) * 2

    def kv_attention(self, q, cache, table, lens):
        self.seen.append((table.clone(), lens.clone()))
        return torch.zeros_like(q)


@pytest.fixture
def plain(monkeypatch):
    p = Plain()
    monkeypatch.setattr(serve, "cq", p)
    return p


def layer(sequences=2, longest=10, page_size=4, **more):
    g = torch.Generator().manual_seed(0)
    return serve.AttentionLayer(torch.randn((HEADS + 2 * KV) * D, HIDDEN, generator=g), torch.randn(HIDDEN, HEADS * D, generator=g), HEADS, KV,
                                sequences=sequences, longest=longest, page_size=page_size, **more)


def tokens(n, seed=1):
    return torch.randn(n, HIDDEN, generator=torch.Generator().manual_seed(seed))


def test_slots_of_a_prompt_and_of_steps(plain):
    a = layer()                                                 # 3 pages of 4 tokens each: sequence 1 has slots 12..23
    a.prompt(tokens(5), 1)
    a.prompt(tokens(2), 0)
    assert plain.written == [[12, 13, 14, 15, 16], [0, 1]]
    for _ in range(3):
        assert a.step(tokens(2)).shape == (2, HIDDEN)
    assert plain.written[2:] == [[2, 17], [3, 18], [4, 19]]
    table, lens = plain.seen[-1]
    assert table.tolist() == [[0, 1, 2], [3, 4, 5]] and lens.tolist() == [5, 8]


def test_a_prompt_that_does_not_fit_is_refused(plain):
    a = layer()
    a.prompt(tokens(12), 0)                                     # whole pages
    before = a.lens.tolist()
    for bad in (13, 100):
        with pytest.raises(ValueError):
            a.prompt(tokens(bad), 0)
    with pytest.raises(ValueError):
        a.prompt(tokens(0), 1)
    for seq in (2, -3):
        with pytest.raises(IndexError):
            a.prompt(tokens(3), seq)
    assert len(plain.written) == 1 and a.lens.tolist() == before


def test_a_step_beyond_the_last_slot_is_refused(plain):
    a = layer()
    a.prompt(tokens(3), 0)
    a.prompt(tokens(11), 1)
    a.step(tokens(2))
    with pytest.raises(ValueError):
        a.step(tokens(2))                                       # sequence 1 is full
    assert len(plain.written) == 3 and a.lens.tolist() == [4, 12]
    a.prompt(tokens(2), 1)                                      # begins anew
    a.step(tokens(2))
    assert plain.written[-1] == [4, 14]


def test_a_step_before_any_prompt_or_of_another_batch_is_refused(plain):
    a = layer()
    with pytest.raises(ValueError):
        a.step(tokens(2))
    a.prompt(tokens(3), 0)
    for n in (1, 3):
        with pytest.raises(ValueError):
            a.step(tokens(n))
    assert len(plain.written) == 1 and a.lens.tolist() == [3, 0]


def test_positions_beyond_the_last_slot_name_no_slot(plain):
    """A step replayed from a CUDA graph passes the host's check once: on the device such tokens go nowhere."""
    a = layer()
    pos = torch.tensor([11, 12, 13, 16, 1000])
    got = a._slots(torch.ones(5, dtype=torch.long), pos).tolist()
    assert got[0] == 23 and all(s < 0 for s in got[1:])


@pytest.mark.parametrize("alpha", (0.15, 0.5, 1.0))
def test_channels_that_the_prompt_does_not_calibrate_have_factor_1(plain, alpha):
    """A factor of 0 would store 0 for whatever later tokens hold in the channel, an infinite one NaN."""
    a = layer(alpha=alpha)
    a.w_qkv = a.w_qkv.clone()
    key = HEADS * D
    a.w_qkv[key + 3] = 0                                        # channel 3 of key head 0: 0 in the prompt
    a.w_qkv[key + KV * D + D + 5] = float("inf")                # channel 5 of value head 1
    x = tokens(4).abs()
    a.prompt(x, 0)
    (_, _, k_col, v_col), = plain.caches
    assert k_col[0, 3] == 1 and v_col[1, 5] == 1
    want = (x @ a.w_qkv.t())[:, key:key + KV * D].abs().amax(0).pow(1 - alpha).view(KV, D)
    want[0, 3] = 1
    torch.testing.assert_close(k_col, want, rtol=1e-6, atol=0)
    assert bool(torch.isfinite(v_col).all()) and bool((v_col > 0).all())
