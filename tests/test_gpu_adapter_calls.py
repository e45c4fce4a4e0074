"""What calls of `adapter_add` ask the runtime besides their launches."""
from __future__ import annotations

import pytest
import torch

from test_gpu_adapter import adapters, some_index, tokens
from test_gpu_serve import cq  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ranks", ((8, 16), (64, 128), (8, 24, 64, 96)))
def test_ranks_in_turn_ask_for_occupancies_once(cq, ranks):  # noqa: F811
    """The projections of a layer may have adapters of different ranks: their calls take turns."""
    from torch.profiler import ProfilerActivity, profile
    T, K, N = 256, 520, 264
    y, x = tokens(T, K, N, "bf16", 1)
    ads, index = [adapters(cq, 2, K, N, R, "bf16", R) for R in ranks], some_index(T, 2, 1, "mixed")

    def calls():
        for ad in ads:
            cq.adapter_add(y, x, ad, index)
        torch.cuda.synchronize()

    calls()
    with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as seen:
        calls()
    names = {e.key: e.count for e in seen.key_averages()}
    launches = sum(n for k, n in names.items() if k.startswith("cudaLaunchKernel"))
    if launches == 0:
        pytest.skip("no calls are recorded here")
    assert launches >= 2 * len(ranks), names
    assert not [k for k in names if "Occupancy" in k or "FuncSetAttribute" in k], names
