"""What the serving operators' binding allocates, accepts and refuses, on the GPU."""
from __future__ import annotations

import pytest
import torch

import serve_reference as ref
from test_gpu_serve import check_product, cq, normal, on_device, operands  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", (1, 2, 5, 63, 65, 131, 1501))
def test_scales_that_fp8_quantize_act_makes_have_whole_rows(cq, M):  # noqa: F811
    K, N = 300, 200
    a = cq.fp8_quantize_act(normal((M, K), 1, torch.bfloat16).cuda())
    nb, up = 3, -(-M // 4) * 4
    assert a.scale.shape == (nb, M) and a.scale.stride() == (up, 1)
    assert a.scale.untyped_storage().nbytes() >= 4 * nb * up
    w = cq.fp8_quantize_weight((normal((N, K), 2, torch.bfloat16, outliers=False) * 0.02).cuda())
    short = torch.empty_strided((nb, M), (up, 1), device="cuda")          # ends with its last element
    short.copy_(a.scale)
    assert torch.equal(cq.fp8_matmul(cq.Fp8Act(a.codes, short), w), cq.fp8_matmul(a, w))


@pytest.mark.parametrize("bits", (8, 4))
def test_a_full_layer_refuses_steps_and_goes_on(cq, bits):  # noqa: F811
    from paper_2410_07505_b200 import serve
    hidden, heads, kv_heads, D = 256, 4, 2, 64
    w_qkv = (normal(((heads + 2 * kv_heads) * D, hidden), 1, torch.bfloat16, outliers=False) * 0.06).cuda()
    w_out = (normal((hidden, heads * D), 2, torch.bfloat16, outliers=False) * 0.06).cuda()
    layer = serve.AttentionLayer(w_qkv, w_out, heads, kv_heads, sequences=2, longest=60, bits=bits, page_size=16)
    x = normal((70, hidden), 3, torch.bfloat16, outliers=False).cuda()
    with pytest.raises(ValueError):
        layer.step(x[:2])
    with pytest.raises(ValueError):
        layer.prompt(x, 0)
    layer.prompt(x[:62], 0)
    layer.prompt(x[:5], 1)
    first = layer.step(x[62:64])
    layer.step(x[64:66])
    held = layer.cache.k_codes.clone()
    with pytest.raises(ValueError):
        layer.step(x[66:68])
    slots = layer._slots(torch.zeros(3, dtype=torch.long, device="cuda"), torch.tensor([63, 64, 5000], device="cuda"))
    assert slots.tolist()[0] == 63 and max(slots.tolist()[1:]) < 0
    kv = normal((3, 2 * kv_heads, D), 4, torch.bfloat16).cuda()
    cq.kv_write(layer.cache, kv[:, :kv_heads], kv[:, kv_heads:], torch.where(slots == 63, -1, slots))      # all name nothing
    assert torch.equal(layer.cache.k_codes, held) and layer.lens.tolist() == [64, 7]
    layer.prompt(x[:62], 0)                                             # the sequence begins anew
    layer.prompt(x[:5], 1)
    assert torch.equal(layer.step(x[62:64]), first)
