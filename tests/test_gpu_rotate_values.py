"""Norms and rotation where a product of some of an element's factors leaves fp32's range and their whole product does not.
Tolerance: that of test_gpu_rotate."""
from __future__ import annotations

import pytest
import torch

from test_gpu_rotate import compare
from test_gpu_serve import cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("neighbours", (False, True))
@pytest.mark.parametrize("R", (0, 64, 128))
@pytest.mark.parametrize("x_size,w_size", ((1e16, 1e25), (1e16, 1e35), (1e-11, 1e-30), (1e-11, 1e-36), (1e-11, 1e35), (1e16, 1e-36), (1.0, 1e37), (1.0, 1e-37)))
def test_weights_far_from_1(cq, x_size, w_size, R, neighbours):  # noqa: F811
    """bfloat16 holds both; a normalised element is some 1 times its weight."""
    T, Hq, H, D = 40, 3, 2, 128
    x = (normal((T, Hq + H, D), 1, torch.float32, False).double() * x_size).bfloat16().cuda()
    w = [(torch.exp(0.3 * normal((D,), 2 + i, torch.float32, False)).double() * w_size).bfloat16().cuda() for i in range(2)]
    q, k = x.split((Hq, H), dim=1)
    positions, freq = torch.arange(T, device="cuda"), cq.rotation_freq(R)
    out = cq.norm_rotate(q, k, positions, freq, *w, eps=0.0, neighbours=neighbours)
    for got, src, ww in zip(out, (q, k), w):
        compare(got, src, ww, positions, freq, 0.0, neighbours)
