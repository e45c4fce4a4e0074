"""Norms and rotation where a product of some of an element's factors leaves fp32's range and their whole product does not, and a
stride that does not matter.  Tolerance: that of test_gpu_rotate."""
from __future__ import annotations

import pytest
import torch

from test_gpu_rotate import compare
from test_gpu_serve import DT, cq, normal  # noqa: F401  (cq: the fixture)

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


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_the_stride_of_an_axis_of_one_element_does_not_matter(cq, dtype):  # noqa: F811
    x = normal((5, 3, 40), 3, DT[dtype], False).cuda()
    one = x[:, :, 7:8]
    odd = torch.as_strided(x, (5, 3, 1), (120, 40, 9), 7)
    assert torch.equal(one, odd)
    positions, freq = torch.arange(5, device="cuda"), cq.rotation_freq(0)
    want = cq.norm_rotate(one.contiguous(), one.contiguous(), positions, freq)
    room = torch.zeros(5, 3, 12, dtype=DT[dtype], device="cuda")
    out = torch.as_strided(room, (5, 3, 1), (36, 12, 5))
    got = cq.norm_rotate(odd, odd, positions, freq, out=(out, torch.empty_like(one)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
