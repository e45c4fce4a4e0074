"""The serving operators together: an attention layer on quantized weights and a quantized cache."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

# Relative errors of independent rounding: an e4m3 code keeps 4 bits, so a value is off by up to 2^-4 of itself, 0.026 in the
# root mean square over a binade; activations and weights both are: 0.037 for a product, and the layer has two in a row
# (0.053).  A cached row is off by a uniform half step of its largest element over 127 or 7; for normal rows of 64 or 128, whose
# largest is about 2.5 to 3.5 deviations, that is 0.29 * 3.5 / 127 = 0.008 or 0.29 * 3.5 / 7 = 0.15, for keys and values both
# (INT4: 0.21).  The bounds are twice the sums' roots.
BOUND = {8: 2 * 0.055, 4: 2 * 0.22}


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("hidden,heads,kv_heads,prompt,steps", ((512, 8, 2, 70, 5), (1024, 8, 8, 200, 3)))
def test_layer_against_the_unquantized_one(bits, hidden, heads, kv_heads, prompt, steps):
    from paper_2410_07505_b200 import build, cq, serve
    build.build()
    r = serve.demo(hidden, heads, kv_heads, prompt, steps, bits, sequences=3)
    assert r["relative_error_prompt"] < BOUND[bits] and r["relative_error_steps"] < BOUND[bits], r
    assert cq.serve_fault() == 0
