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


def test_workspaces_of_another_device_or_layout_are_refused(cq):  # noqa: F811
    x = normal((4, 256), 1, torch.bfloat16).cuda()
    w = cq.fp8_quantize_weight(x)
    need = int(cq.lib().cq_fp8_linear_workspace_bytes(4, 256))
    cache = cq.KVCache.empty(2, 16, 2, 64)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    more = cq.kv_attention_workspace_bytes(64)
    for n, call in ((need, lambda ws: cq.fp8_linear(x, w, workspace=ws)), (more, lambda ws: cq.kv_attention(q, cache, table, lens, workspace=ws))):
        for bad in (torch.empty(n, dtype=torch.uint8), torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2],
                    torch.empty(1, dtype=torch.uint8, device="cuda").expand(n)):
            with pytest.raises(ValueError):
                call(bad)
        with pytest.raises(cq.CQError):
            call(torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
        want = call(None)
        assert torch.equal(call(torch.empty(-(-n // 4), dtype=torch.float32, device="cuda")), want)      # sized in bytes, not elements


def test_one_row_of_an_odd_pitch_goes_through_the_product(cq):  # noqa: F811
    a, sa, w, sw = operands(1, 70, 100, 5)
    A, W = on_device(cq, a, sa, w, sw)
    wide = torch.zeros(3, 264, dtype=torch.uint8, device="cuda")
    wide[0, :100] = A.codes.view(torch.uint8)
    scale = torch.zeros(2, 9, device="cuda")
    scale[:1, :1] = A.scale
    odd = cq.Fp8Act(wide.view(torch.float8_e4m3fn)[:1, :100], scale[:1, :1])
    got = cq.fp8_matmul(odd, W, torch.float32)
    y, mag = ref.fp8_product(a, sa, w, sw)
    check_product(got, y, mag, torch.float32)
    row = cq.Fp8Weight(wide.view(torch.float8_e4m3fn)[:1, :100], torch.ones(1, 1, device="cuda"))       # one output channel
    y, mag = ref.fp8_product(a, sa, a, sw[:1] * 0 + 1)
    check_product(cq.fp8_matmul(odd, row, torch.float32), y, mag, torch.float32)


def test_the_demo_does_not_report_results_of_a_wait_that_gave_up(cq, monkeypatch):  # noqa: F811
    from paper_2410_07505_b200 import serve
    args = dict(hidden=256, heads=4, kv_heads=2, prompt=20, steps=2, bits=8)
    assert serve.demo(**args)["relative_error_steps"] < 0.2
    monkeypatch.setattr(cq, "serve_fault", lambda: 1)
    with pytest.raises(RuntimeError):
        serve.demo(**args)
