"""The layer's operators together: rotation, adapters and packed prompts in an attention layer on quantized weights and cache."""
from __future__ import annotations

import pytest
import torch

from test_gpu_serve import cq, normal  # noqa: F401  (cq: the fixture)
from test_gpu_serve_layer import BOUND

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("rotate,rank", ((True, 0), (False, 16), (True, 8)))
def test_layer_with_rotation_and_adapters_against_the_unquantized_one(cq, bits, rotate, rank):  # noqa: F811
    """The bounds of the layer without them: the adapters' products are on 16 bits, which adds 2^-8 where those on 8 have 2^-4.  Norms of
    queries and keys leave relative errors as they are, a rotation too."""
    from paper_2410_07505_b200 import serve
    r = serve.demo(512, 8, 2, 70, 5, bits, sequences=3, rotate=rotate, adapter_rank=rank)
    assert r["relative_error_prompt"] < BOUND[bits] and r["relative_error_steps"] < BOUND[bits], r


def make(cq, sequences, **more):  # noqa: F811
    from paper_2410_07505_b200 import serve
    hidden, heads, kv_heads, D = 256, 4, 2, 64
    w_qkv = (normal(((heads + 2 * kv_heads) * D, hidden), 1, torch.bfloat16, outliers=False) * 0.06).cuda()
    w_out = (normal((hidden, heads * D), 2, torch.bfloat16, outliers=False) * 0.06).cuda()
    ad = [cq.Adapters((normal((3, 8, w.shape[1]), 3, torch.bfloat16, False) * 0.06).cuda(), normal((3, w.shape[0], 8), 4, torch.bfloat16, False).cuda())
          for w in (w_qkv, w_out)]
    return serve.AttentionLayer(w_qkv, w_out, heads, kv_heads, sequences=sequences, longest=200, page_size=16, freq=cq.rotation_freq(D), eps=1e-6,
                                qkv_adapters=ad[0], out_adapters=ad[1], **more)


def test_packed_prompts_and_steps_equal_those_one_by_one(cq):  # noqa: F811
    """Tokens of other sequences do not matter; what differs is where the product of 8-bit floats cuts its sums (fp32) and the
    calibration, which here is the same tensor's: both layers see the whole batch first."""
    x = normal((150, 256), 5, torch.bfloat16, outliers=False).cuda()
    a, b = make(cq, 3), make(cq, 3)
    lengths, adapters = [70, 1, 79], [2, -1, 0]
    first = a.prompts(x, [1, 0, 2], lengths, adapters)
    again = b.prompts(x, [1, 0, 2], lengths, adapters)
    assert torch.equal(first, again)                             # equal calls give equal bits
    one = [b.prompt(part, s, ad) for part, s, ad in zip(x.split(lengths), (1, 0, 2), adapters)]
    whole = torch.cat(one).double()
    # two layers of e4m3 roundings apart at most where fp32 sums differ in their last bits: a code may fall the other way, 2^-4 of one of 256 terms
    assert float((first.double() - whole).norm() / whole.norm()) < 0.02
    steps = [layer.step(x[:3]) for layer in (a, b)]
    assert float((steps[0].double() - steps[1].double()).norm() / steps[1].double().norm()) < 0.02


def test_a_prompt_and_steps_from_a_graph(cq):  # noqa: F811
    x = normal((60, 256), 6, torch.bfloat16, outliers=False).cuda()
    layer = make(cq, 1)
    layer.prompt(x, 0, 1)
    want = layer.prompt(x, 0, 1), layer.step(x[:1])
    layer.prompt(x, 0, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.prompt(x, 0, 1), layer.step(x[:1])
    for t in got:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del graph
