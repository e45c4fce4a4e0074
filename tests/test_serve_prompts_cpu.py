"""Host logic of serve.AttentionLayer's packed prompts, rotation and adapters, with plain operators in place of the kernels."""
from __future__ import annotations

import types

import pytest
import torch

from paper_2410_07505_b200 import serve
from test_serve_layer_cpu import D, HEADS, HIDDEN, KV, Plain, layer, tokens


class More(Plain):
    """Stands for the module cq; keeps what it was asked."""

    def __init__(self):
        super().__init__()
        self.turned, self.adapted = [], []

    def norm_rotate(self, q, k, pos, freq, q_weight, k_weight, *, eps, neighbours, out):
        self.turned.append((pos.tolist(), freq.shape[0], eps, neighbours))
        assert out[0].data_ptr() == q.data_ptr() and out[1].data_ptr() == k.data_ptr()
        return out

    def adapter_add(self, y, x, adapters, index, *, out):
        self.adapted.append((adapters, index.tolist()))
        return y


@pytest.fixture
def plain(monkeypatch):
    p = More()
    monkeypatch.setattr(serve, "cq", p)
    return p


def test_packed_prompts_are_the_prompts_one_by_one(plain):
    x = tokens(9)
    a, b = layer(sequences=3), layer(sequences=3)
    together = a.prompts(x, [2, 0], [5, 4])
    alone = torch.cat((b.prompt(x[:5], 2), b.prompt(x[5:], 0)))
    torch.testing.assert_close(together, alone)
    assert plain.written == [[24, 25, 26, 27, 28, 0, 1, 2, 3], [24, 25, 26, 27, 28], [0, 1, 2, 3]]
    assert a.lens.tolist() == [4, 0, 5] and a._filled == [4, 0, 5]


def test_packed_prompts_that_do_not_fit_are_refused(plain):
    a = layer()
    for seqs, lengths in (([0, 0], [2, 2]), ([0, 1], [2, 3]), ([0], [2, 2]), ([], []), ([0, 1], [4, 0]), ([0, 1], [13, -9])):
        with pytest.raises(ValueError):
            a.prompts(tokens(4), seqs, lengths)
    with pytest.raises(IndexError):
        a.prompts(tokens(4), [0, 5], [2, 2])
    with pytest.raises(ValueError):
        a.prompts(tokens(4), [0], [4], [1])                     # the layer has no adapters
    assert plain.written == [] and a.lens.tolist() == [0, 0]


def test_positions_reach_the_rotation(plain):
    a = layer(freq=torch.zeros(3, dtype=torch.float64), eps=1e-6, neighbours=True)
    a.prompts(tokens(5), [1, 0], [3, 2])
    a.step(tokens(2))
    assert plain.turned == [([0, 1, 2, 0, 1], 3, 1e-6, True), ([2, 3], 3, 1e-6, True)]
    b = layer(eps=1e-5)                                         # norms alone
    b.prompt(tokens(2), 0)
    assert plain.turned[-1] == ([0, 1], 0, 1e-5, False)
    with pytest.raises(ValueError):
        layer(q_weight=torch.ones(D))


def test_each_sequence_keeps_its_adapter(plain):
    a = layer(sequences=3, qkv_adapters="in", out_adapters="out")
    a.prompts(tokens(4), [2, 0], [3, 1], [5, -1])
    a.prompt(tokens(2), 1, 7)
    a.step(tokens(3))
    assert plain.adapted == [("in", [5, 5, 5, -1]), ("out", [5, 5, 5, -1]), ("in", [7, 7]), ("out", [7, 7]), ("in", [-1, 7, 5]), ("out", [-1, 7, 5])]
    a.prompt(tokens(2), 1)                                      # replaced, without an adapter
    a.step(tokens(3))
    assert plain.adapted[-1] == ("out", [-1, -1, 5])


def test_one_side_may_have_no_adapters(plain):
    a = layer(out_adapters="out")
    a.prompt(tokens(2), 0, 3)
    assert plain.adapted == [("out", [3, 3])]


def test_shapes(plain):
    assert layer().prompts(tokens(4), [0, 1], [1, 3]).shape == (4, HIDDEN) and HEADS % KV == 0 and isinstance(plain.KVCache, types.SimpleNamespace)
