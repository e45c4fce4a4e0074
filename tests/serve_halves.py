"""fp16 attention over the cache: a bound of its own, inputs on which each second half shows, and a model to plant mistakes in.

For fp16 the kernel holds a query times its channel factors, z, and each probability times value scale, w, as two fp16 numbers each,
the second for what the first leaves.  With D channels, n tokens, `bias` = 128 (INT8) or 8 (INT4):

  logit     z = fl32(q f).  Two halves leave 2^-22 of an element and 2^-35 of the row's largest one.  A product with a block of 16
            channels is a sum of 17 terms that keep 24 bits below the largest one's exponent (codes are subnormal fp16 with the exponent
            of 2^-14, that is 2^10 of a code, and less than twice that), so each loses less than 2^-23 of the largest magnitude M: products
            stay below 2^11 max|z|, sums below 3 bias sum|z|.  There are 2 D / 16 such sums:  E = (D / 8) 17 2^-23 max(2^11 max|z|,
            3 bias sum|z|) code units.  With the other fp32 roundings and the halves a logit is off by at most
                d = scale ka E + 2^-21 reach,     reach = scale ka sum |z c|.
  weights   the result's numerator and denominator both carry the logits' errors: 2.2 d of the probability-weighted |v|.  ex2 and the
            sums of probabilities: 2^-18.  w: 2^-22 of itself, or 2^-25 of its row's unit, in which the row's largest is above 2^4.
  result    2 (n / 64 + 1) products of 16 tokens and the joins: 17 2^-23 of at most twice the sum's magnitude each.
Then half an ulp of the result.  A lost second half costs up to 2^-11 of z or w, which these bounds are to show: the two cases below
make it as large as it can be in all elements alike.
"""
from __future__ import annotations

import numpy as np

NEARLY_A_TIE = np.float32(1 + 0.9 * 2.0 ** -11)            # fp16 rounds it to 1; two halves hold it


def bound(q, kf, vf, kc, ka, vc, va, scale, bits):
    """(result in 64 bits, its bound, lse, its bound) of query rows q [R, D] that see all n tokens of one head."""
    R, D = q.shape
    n = kc.shape[0]
    bias = 128 if bits == 8 else 8
    z = (q.astype(np.float32) * kf.astype(np.float32)).astype(np.float64)
    ka, va = ka.astype(np.float64), va.astype(np.float64)
    logits = (q.astype(np.float64) * kf.astype(np.float64)) @ kc.T * ka * scale
    top = logits.max(axis=1, keepdims=True)
    p = np.exp(logits - top)
    total = p.sum(axis=1, keepdims=True)
    p /= total
    v = vc * va[:, None] * vf.astype(np.float64)
    want, mag, lse = p @ v, p @ np.abs(v), (top + np.log(total))[:, 0]
    E = D / 8 * 17 * 2.0 ** -23 * np.maximum(2.0 ** 11 * np.abs(z).max(axis=1), 3 * bias * np.abs(z).sum(axis=1))
    d = (scale * np.abs(ka)[None] * E[:, None] + 2.0 ** -21 * (np.abs(z) @ np.abs(kc).T * np.abs(ka) * scale)).max(axis=1)[:, None]
    off = (2.2 * d + 2.0 ** -18 + (2 * (n // 64 + 1) + 4) * 17 * 2.0 ** -22) * mag
    off += 2.0 ** -28 * (p * np.abs(va)).max(axis=1)[:, None] * (np.abs(vc).sum(axis=0) * vf)[None]
    half_ulp = np.spacing((np.abs(want) + off).astype(np.float16)).astype(np.float64) / 2
    return want, off + half_ulp * 1.001, lse, d[:, 0] + 2.0 ** -18 * (1 + np.abs(lse))


def worst(out, lse, case):
    """Largest errors as fractions of their bounds."""
    want, off, want_lse, off_lse = bound(**case)
    return float(np.max(np.abs(out.astype(np.float64) - want) / off)), float(np.max(np.abs(lse.astype(np.float64) - want_lse) / off_lse))


def query_case(R, D, bits, seed):
    """Logits of +-3 (and +-1.5) whose queries times factors are all nearly a tie: without their second halves all logits shrink by
    0.9 * 2^-11, and the unlikely tokens, which alone hold something in half of the channels, gain 2 * 3 times that."""
    r = np.random.default_rng(seed)
    n, qmax = 40, 127 if bits == 8 else 7
    sign = r.choice((-1.0, 1.0), D)
    q = sign[None] * np.where(np.arange(R) % 2 == 0, 1.0, 0.5)[:, None]
    likely = np.arange(n) % 2 == 0
    kc = np.where(likely, 1.0, -1.0)[:, None] * sign[None] * qmax
    vc = r.integers(1, qmax + 1, (n, D)).astype(np.float64)
    vc[likely, :D // 2] = 0
    scale = D ** -0.5
    return dict(q=q, kf=np.full(D, NEARLY_A_TIE), vf=np.ones(D, np.float32), kc=kc, ka=np.full(n, 3 / (scale * D * qmax), np.float32),
                vc=vc, va=np.full(n, 0.37, np.float32), scale=scale, bits=bits)


def weight_case(R, D, bits, seed):
    """All tokens weigh the same, and probability times value scale is nearly a tie: without second halves results shrink by 0.9 * 2^-11."""
    r = np.random.default_rng(seed)
    n, qmax = 40, 127 if bits == 8 else 7
    return dict(q=r.normal(0, 1, (R, D)).astype(np.float16).astype(np.float64), kf=np.ones(D, np.float32), vf=np.ones(D, np.float32),
                kc=np.round(r.uniform(-qmax, qmax, (n, D))), ka=np.full(n, 0.01, np.float32), vc=r.integers(1, qmax + 1, (n, D)).astype(np.float64),
                va=np.full(n, NEARLY_A_TIE / 4, np.float32), scale=1e-7, bits=bits)


# ----------------------------------------------------------------------------- the model
def halves(x, second):
    h = x.astype(np.float16).astype(np.float64)
    return h + (x - h).astype(np.float16).astype(np.float64) if second else h


def model(q, kf, vf, kc, ka, vc, va, scale, bits, second_of_queries=True, second_of_weights=True):
    """(out in fp16, lse): the kernel's roundings of z and w, everything else in 64 bits."""
    z = (q.astype(np.float32) * kf.astype(np.float32)).astype(np.float64)
    up = 2.0 ** (14 - np.floor(np.log2(np.abs(z).max(axis=1, keepdims=True))))
    logits = halves(z * up, second_of_queries) / up @ kc.T * ka.astype(np.float64) * scale
    ref = np.ceil(logits.max(axis=1, keepdims=True) / np.log(2))
    p = np.exp2(logits / np.log(2) - ref)
    w = p * va.astype(np.float64)
    unit = 2.0 ** (4 - np.floor(np.log2(np.abs(w).max(axis=1, keepdims=True))))
    total = p.sum(axis=1, keepdims=True)
    out = halves(w * unit, second_of_weights) / unit @ vc / total * vf
    return out.astype(np.float16), (ref * np.log(2) + np.log(total))[:, 0]
