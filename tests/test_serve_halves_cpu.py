"""The bound of fp16 attention (tests/serve_halves.py) on a model of its roundings: met by two halves, missed by one."""
from __future__ import annotations

import numpy as np
import pytest

import serve_halves as sh

SHAPES = [(R, D, bits) for R in (1, 8, 12, 20, 28) for D in (64, 128) for bits in (8, 4)]


@pytest.mark.parametrize("R,D,bits", SHAPES)
def test_a_lost_second_half_misses_the_bound(R, D, bits):
    q, w = sh.query_case(R, D, bits, R + D), sh.weight_case(R, D, bits, R + D)
    for case in (q, w):
        out, lse = sh.worst(*sh.model(**case), case)
        assert out < 1 and lse < 1
    out, lse = sh.worst(*sh.model(**q, second_of_queries=False), q)
    assert out > 1 and lse > 1
    out, lse = sh.worst(*sh.model(**w, second_of_weights=False), w)
    assert out > 1


@pytest.mark.parametrize("bits", (8, 4))
def test_two_halves_meet_the_bound_on_ordinary_inputs(bits):
    r = np.random.default_rng(bits)
    qmax = 127 if bits == 8 else 7
    for D, n in ((64, 1), (128, 700)):
        case = dict(q=r.normal(0, 1.3, (9, D)).astype(np.float16).astype(np.float64), kf=np.exp(0.7 * r.normal(0, 1, D)).astype(np.float32),
                    vf=np.exp(0.7 * r.normal(0, 1, D)).astype(np.float32), kc=np.clip(np.round(r.normal(0, qmax / 3.5, (n, D))), -qmax, qmax),
                    ka=(3.5 / qmax * np.exp(0.4 * r.normal(0, 1, n))).astype(np.float32), vc=np.clip(np.round(r.normal(0, qmax / 3.5, (n, D))), -qmax, qmax),
                    va=(3.5 / qmax * np.exp(0.4 * r.normal(0, 1, n))).astype(np.float32), scale=D ** -0.5, bits=bits)
        out, lse = sh.worst(*sh.model(**case), case)
        assert out < 1 and lse < 1
