"""Plain forms of the serving operators for the tests: what include/cq.h says, step by step.

Where the definition rounds to fp32 (fl32) the step is done in numpy's float32, everything else in 64 bits.  The
inputs are 16-bit tensors on the host.
"""
from __future__ import annotations

import math

import numpy as np
import torch

BLOCK = 128


def f32(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().float().numpy()


def round_e4m3(v: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value (ties to even, saturating at 448, NaN kept), in float64."""
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        _, e = np.frexp(v)
        step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
        r = np.round(v / step) * step
        return np.where(np.isnan(v), np.nan, np.clip(r, -448.0, 448.0))


def quotients(x: np.ndarray, s: np.ndarray) -> np.ndarray:
    """fl32(x / s), 0 where s is 0."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        q = np.divide(x.astype(np.float32), s.astype(np.float32), dtype=np.float32)
    return np.where(np.broadcast_to(s == 0, q.shape), np.float32(0), q)


def absmax(x: np.ndarray, axis) -> np.ndarray:
    return np.max(np.abs(x), axis=axis) if x.size else np.zeros([n for i, n in enumerate(x.shape) if i not in np.atleast_1d(axis)], np.float32)


def fp8_act(x: np.ndarray):
    """(code values [T, K] in float64, scales [blocks, T] in float32)"""
    T, K = x.shape
    nb = -(-K // BLOCK)
    scale = np.zeros((nb, T), np.float32)
    codes = np.zeros((T, K))
    for b in range(nb):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        scale[b] = absmax(part, 1) / np.float32(448)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = round_e4m3(quotients(part, scale[b][:, None]))
    return codes, scale


def fp8_weight(w: np.ndarray):
    N, K = w.shape
    scale = np.zeros((-(-N // BLOCK), -(-K // BLOCK)), np.float32)
    codes = np.zeros((N, K))
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = np.s_[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
            scale[i, j] = absmax(w[at], (0, 1)) / np.float32(448)
            codes[at] = round_e4m3(quotients(w[at], scale[i, j]))
    return codes, scale


def fp8_product(a: np.ndarray, sa: np.ndarray, w: np.ndarray, sw: np.ndarray):
    """(the product in 64 bits, the sum of its terms' magnitudes)"""
    M, K = a.shape
    N = w.shape[0]
    y, mag = np.zeros((M, N)), np.zeros((M, N))
    with np.errstate(invalid="ignore", over="ignore"):
        for b in range(-(-K // BLOCK)):
            at = np.s_[:, b * BLOCK:(b + 1) * BLOCK]
            f = sa[b].astype(np.float64)[:, None] * np.repeat(sw[:, b].astype(np.float64), BLOCK)[None, :N]
            y += (a[at] @ w[at].T) * f
            mag += (np.abs(a[at]) @ np.abs(w[at]).T) * f
    return y, mag


def kv_quantize(x: np.ndarray, col, bits: int):
    """(integer codes [T, H, D], scales [T, H]) of token rows x (float32)."""
    qmax = np.float32(127 if bits == 8 else 7)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        if col is not None:
            inv = np.where(col > 0, np.float32(1) / col, np.float32(0)).astype(np.float32)
            x = (x * inv).astype(np.float32)
        scale = (absmax(x, -1) / qmax).astype(np.float32)
        q = np.clip(np.round(quotients(x, scale[..., None])), -qmax, qmax)
    q = np.where(np.isfinite(scale)[..., None], q, 0.0)
    return q.astype(np.int64), scale


def kv_values(codes: np.ndarray, scale: np.ndarray, col) -> np.ndarray:
    """fl32(code * fl32(scale * factor)) of integer codes [..., H, D]."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale[..., None].astype(np.float32)
        if col is not None:
            s = (s * col).astype(np.float32)
        return (codes.astype(np.float32) * s).astype(np.float32)


def unpack(codes: torch.Tensor, bits: int) -> np.ndarray:
    c = codes.cpu().numpy()
    if bits == 8:
        return c.astype(np.int64)
    both = np.stack((c & 15, c >> 4), axis=-1).reshape(*c.shape[:-1], -1).astype(np.int64)
    return np.where(both > 7, both - 16, both)


def pack(codes: np.ndarray, bits: int) -> torch.Tensor:
    if bits == 8:
        return torch.from_numpy(codes.astype(np.int8))
    c = codes.astype(np.int64) & 15
    return torch.from_numpy((c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8))


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """One sequence and one key/value head in 64 bits: q [Lq, G, D], k, v [n, D] in float64.
    Returns (out, lse, largest sum of |q_d k_d| * scale, softmax-weighted |v|) for each query row."""
    Lq, G, D = q.shape
    n = k.shape[0]
    out, mag = np.zeros((Lq, G, D)), np.zeros((Lq, G, D))
    lse, reach = np.full((Lq, G), -math.inf), np.zeros((Lq, G))
    for i in range(Lq):
        m = n - Lq + i + 1
        if m <= 0:
            continue
        logits = q[i] @ k[:m].T * scale
        reach[i] = (np.abs(q[i]) @ np.abs(k[:m]).T * scale).max(axis=1)
        top = logits.max(axis=1, keepdims=True)
        p = np.exp(logits - top)
        total = p.sum(axis=1, keepdims=True)
        out[i] = p @ v[:m] / total
        mag[i] = p @ np.abs(v[:m]) / total
        lse[i] = (top + np.log(total))[:, 0]
    return out, lse, reach, mag
