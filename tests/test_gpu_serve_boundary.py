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
