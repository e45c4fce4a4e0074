"""Causal attention over packed prompts on the GPU against its definition in 64 bits (serve_reference.attention).

Tolerance, for a query with n visible keys, `reach` the largest sum of |q_d k_d| * scale over its keys, `mag` the weighted mean of |v|, U half
an ulp at 1 of the dtype, top the largest |v|:
  logits: D <= 128 products added in fp32 by the tensor cores, each addition off by at most 2^-23 of the sum of magnitudes: 2^-16 reach;
          the factor and the reference add 2^-22 reach.  Numerator and denominator both carry it: 2^-14 reach mag bounds both
  weights: rounded once to the dtype, U mag; 2^x is off by 2^-22; fp16 keeps them, times 2^7, to 2^-25 below 2^-14: 2^-32 of the
          largest each, n 2^-32 top in all
  sums: n additions each in numerator and denominator, the terms positive up to |v|: n 2^-23 mag, the references' renewals
          (at most 2^-24 each, fewer than 32 since each is by 2^8) 2^-18 mag
  result: U of itself, and a subnormal's half step
The logarithm of the sum: the logits' 2^-15 reach, the sum's n 2^-24 + 2^-19, and 2^-22 of itself.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import serve_reference as ref
from guards import Arena
from test_gpu_serve import DT, TINY, UNIT, cq, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu


def starts(lens):
    return torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device="cuda")


def definition(q, k, v, q_lens, k_lens, scale):
    """(out, lse, bound of out, bound of lse) in 64 bits; q [Tq, Hq, D], k, v [Tk, H, D] tensors."""
    Hq, H, dtype = q.shape[1], k.shape[1], q.dtype
    G, U = Hq // H, UNIT[dtype]
    q, k, v = (t.cpu().double().numpy() for t in (q, k, v))
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -math.inf)
    tol, lse_tol = np.zeros(q.shape), np.zeros(q.shape[:2])
    q0 = k0 = 0
    for n, m in zip(q_lens, k_lens):
        for h in range(H):
            at = np.s_[q0:q0 + n, h * G:(h + 1) * G]
            keys, values = k[k0:k0 + m, h], v[k0:k0 + m, h]
            o, ls, reach, mag = ref.attention(q[at], keys, values, scale)
            top = np.abs(values).max() if m else 0.0
            out[at], lse[at] = o, ls
            r = reach[..., None]
            tol[at] = (2.0 ** -14 * r + U + m * 2.0 ** -23 + 2.0 ** -18) * mag + m * 2.0 ** -32 * top + U * np.abs(o) * 1.001 + TINY[dtype]
            lse_tol[at] = 2.0 ** -15 * reach + m * 2.0 ** -24 + 2.0 ** -19 + 2.0 ** -22 * np.abs(np.where(np.isfinite(ls), ls, 0))
        q0, k0 = q0 + n, k0 + m
    return out, lse, tol, lse_tol


def check(cq, q, k, v, q_lens, k_lens=None, scale=None, **more):  # noqa: F811
    same = k_lens is None
    k_lens = q_lens if same else k_lens
    ar = Arena()
    ar.add("out", tuple(q.shape), q.dtype)
    ar.add("lse", tuple(q.shape[:2]), torch.float32)
    ar.build()
    got = cq.prompt_attention(q, k, v, starts(q_lens), None if same else starts(k_lens), scale=scale, out=ar["out"], lse=ar["lse"], **more)
    assert got is ar["out"]
    ar.check("prompt_attention")
    out, lse, tol, lse_tol = definition(q, k, v, q_lens, k_lens, q.shape[2] ** -0.5 if scale is None else scale)
    off = np.abs(got.cpu().double().numpy() - out)
    assert (off <= tol).all(), (float((off / np.maximum(tol, 1e-300)).max()), np.argwhere(off > tol)[:5])
    g = ar["lse"].cpu().double().numpy()
    assert ((g == -np.inf) == (lse == -np.inf)).all()
    with np.errstate(invalid="ignore"):
        assert ((np.abs(g - lse) <= lse_tol) | (lse == -np.inf)).all()
    return got


def qkv(T, heads, D, dtype, seed, Tk=None):
    """Slices of one projection, or keys and values of a length of their own."""
    x = normal((T, sum(heads), D), seed, DT[dtype], outliers=False).cuda()
    q, k, v = x.split(heads, dim=1)
    if Tk is not None:
        k, v = (normal((Tk, heads[1], D), seed + i, DT[dtype], outliers=False).cuda() for i in (1, 2))
    return q, k, v


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("n", (1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 700))
def test_one_prompt(cq, dtype, D, n):  # noqa: F811
    check(cq, *qkv(n, (4, 2, 2), D, dtype, n + D), [n])


@pytest.mark.parametrize("Hq,H", ((1, 1), (2, 1), (3, 1), (5, 5), (10, 2), (7, 1), (16, 1), (24, 2), (13, 1), (32, 1), (34, 2), (71, 1)))
def test_query_heads_that_share_a_key_head(cq, Hq, H):  # noqa: F811
    check(cq, *qkv(150, (Hq, H, H), 64, "bf16", Hq), [150])


@pytest.mark.parametrize("dtype,D", (("f16", 128), ("bf16", 64)))
@pytest.mark.parametrize("lens", ([0, 1, 0, 0, 127, 128, 129, 1, 300, 0], [1] * 70, [5, 600, 5], [0], [0, 0, 3]))
def test_packed_prompts(cq, dtype, D, lens):  # noqa: F811
    check(cq, *qkv(sum(lens), (8, 2, 2), D, dtype, len(lens)), lens)


def test_more_sequences_than_a_warp_looks_at_at_once(cq):  # noqa: F811
    lens = [(29 * i) % 41 for i in range(1500)]
    lens[700], lens[1499] = 400, 0
    check(cq, *qkv(sum(lens), (2, 1, 1), 64, "bf16", 8), lens)


def test_more_items_than_ctas(cq):  # noqa: F811
    lens = [(37 * i) % 301 for i in range(40)]
    check(cq, *qkv(sum(lens), (16, 16, 16), 64, "f16", 3), lens)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("q_lens,k_lens", (([1], [1000]), ([7, 130], [1000, 131]), ([3, 4, 0, 5], [2, 4, 9, 0]), ([300], [17]), ([129, 2], [128, 500]), ([4], [0]),
                                           ([200, 40], [0, 40])))
def test_queries_and_keys_of_different_lengths(cq, D, q_lens, k_lens):  # noqa: F811
    """Chunks behind a context, and queries before the first key: their rows are zeros."""
    check(cq, *qkv(sum(q_lens), (4, 2, 2), D, "bf16", 5, sum(k_lens)), q_lens, k_lens)


@pytest.mark.parametrize("q_lens,k_lens,Hq,H,D,dtype", (([1], [9000], 8, 2, 128, "bf16"), ([33], [5000], 4, 4, 64, "f16"), ([20, 3, 0], [3000, 4, 2900], 2, 1, 128, "f16"),
                                                        ([70], [600], 6, 2, 64, "bf16")))
def test_keys_split_over_several_ctas(cq, q_lens, k_lens, Hq, H, D, dtype):  # noqa: F811
    need = cq.prompt_attention_workspace_bytes(len(q_lens), sum(q_lens), sum(k_lens), Hq, H, D)
    assert (need > 0) == (sum(k_lens) > 1000)
    check(cq, *qkv(sum(q_lens), (Hq, H, H), D, dtype, 9, sum(k_lens)), q_lens, k_lens)


@pytest.mark.parametrize("scale", (1e-20, 0.01, 1.0, 30.0))
def test_scales(cq, scale):  # noqa: F811
    check(cq, *qkv(140, (4, 2, 2), 64, "f16", 11), [140], scale=scale)


def test_logits_that_grow_and_fall_along_the_keys(cq):  # noqa: F811
    """References are renewed many times in one order, never in the other."""
    for sign in (1, -1):
        q, k, v = qkv(900, (2, 2, 2), 64, "bf16", 12)
        ramp = torch.linspace(-12, 12, 900, device="cuda")[:, None, None] * sign
        q, k = q.clone(), k.clone()
        q[..., 0], k[..., 0:1] = 8, (ramp.expand(-1, 2, 1) * 1.0).to(k.dtype)
        check(cq, q, k, v, [900])


def test_orders_of_memory(cq):  # noqa: F811
    q, k, v = qkv(100, (4, 2, 2), 64, "bf16", 13)
    want = check(cq, q, k, v, [60, 40])
    heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    assert torch.equal(check(cq, *heads_first, [60, 40]), want)
    padded = []
    for t in (q, k, v):
        wide = torch.full((100, t.shape[1], 88), math.nan, dtype=t.dtype, device="cuda")
        wide[:, :, 8:72] = t
        padded.append(wide[:, :, 8:72])
    assert torch.equal(check(cq, *padded, [60, 40]), want)
    one = q[:1, :2], k[:1, :1], v[:1, :1]                        # strides of axes of one element do not matter
    odd = [torch.as_strided(t.contiguous(), t.shape, (3 if t.shape[0] == 1 else t.stride(0), 64 if t.shape[1] > 1 else 5, 1)) for t in one]
    assert torch.equal(check(cq, *odd, [1]), check(cq, *one, [1]))


def test_rows_outside_the_sequences_are_left_as_they_were(cq):  # noqa: F811
    for Tk in (50, 6000):                                       # whole, and with the keys split
        q, k, v = qkv(50, (4, 2, 2), 128, "bf16", 14, Tk)
        out, lse = torch.full_like(q, 7).contiguous(), torch.full((50, 4), 5.0, device="cuda")
        at_q = torch.tensor([3, 10, 10, 41], dtype=torch.int32, device="cuda")
        at_k = torch.tensor([2, 9, 9, Tk - 4], dtype=torch.int32, device="cuda")
        cq.prompt_attention(q, k, v, at_q, at_k, out=out, lse=lse)
        assert bool((out[:3] == 7).all()) and bool((out[41:] == 7).all()) and bool((lse[:3] == 5).all()) and bool((lse[41:] == 5).all())
        o, _, tol, _ = definition(q[3:41], k[2:Tk - 4], v[2:Tk - 4], [7, 0, 31], [7, 0, Tk - 13], 128 ** -0.5)
        assert (np.abs(out[3:41].cpu().double().numpy() - o) <= tol).all()


def test_starts_that_lie_outside_are_cut(cq):  # noqa: F811
    q, k, v = qkv(40, (2, 1, 1), 64, "bf16", 15)
    want = check(cq, q, k, v, [40])
    wild = torch.tensor([-5, 1000], dtype=torch.int32, device="cuda")
    assert torch.equal(cq.prompt_attention(q, k, v, wild), want)
    falling = torch.tensor([40, 3], dtype=torch.int32, device="cuda")
    out = torch.full_like(want, 3)
    cq.prompt_attention(q, k, v, falling, out=out)
    assert bool((out == 3).all())


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("lens", ([300, 77], [500]))
def test_what_a_query_does_not_see_has_no_effect(cq, dtype, D, lens):  # noqa: F811
    """Infinities and NaN in keys and values of later tokens and of other sequences."""
    T = sum(lens)
    q, k, v = (t.contiguous() for t in qkv(T, (4, 2, 2), D, dtype, 16))
    want = cq.prompt_attention(q, k, v, starts(lens))
    for bad in (math.inf, -math.inf, math.nan):
        for at in (0, 5, 130, 255, T - 1):
            for name in "kv":
                k2, v2 = k.clone(), v.clone()
                (k2 if name == "k" else v2)[at, 1, 3::7] = bad
                got = cq.prompt_attention(q, k2, v2, starts(lens))
                first = 0 if at < lens[0] else lens[0]
                last = lens[0] if at < lens[0] else T
                assert torch.equal(got[:, :2], want[:, :2])                      # heads of the other key head
                assert torch.equal(got[:at, 2:], want[:at, 2:]) and torch.equal(got[last:, 2:], want[last:, 2:]), (bad, at, name)
                assert first <= at < last
                seen = got[at:last, 2:].float()
                if name == "v":
                    channels = torch.zeros(D, dtype=torch.bool, device="cuda")
                    channels[3::7] = True
                    assert not bool(torch.isfinite(seen[..., channels]).any()), (bad, at)
                    assert torch.equal(got[at:last, 2:][..., ~channels], want[at:last, 2:][..., ~channels])


def test_a_key_of_nan_or_infinity_makes_rows_nan(cq):  # noqa: F811
    q, k, v = (t.contiguous() for t in qkv(200, (2, 1, 1), 64, "bf16", 17))
    want = cq.prompt_attention(q, k, v, starts([200]))
    k[100, 0, 0] = math.nan
    got = cq.prompt_attention(q, k, v, starts([200]))
    assert torch.equal(got[:100], want[:100]) and bool(torch.isnan(got[100:]).all())
    q, k, v = (t.contiguous() for t in qkv(200, (2, 1, 1), 64, "bf16", 17))
    q[..., 5] = 1
    k[100, 0, 5] = math.inf                                     # a logit of +infinity: infinity less infinity
    assert bool(torch.isnan(cq.prompt_attention(q, k, v, starts([200]))[100:]).all())
    want = definition(q, k, v, [200], [200], 0.125)
    k[100, 0, 5] = -math.inf                                    # of -infinity: no weight
    lse = torch.empty(200, 2, device="cuda")
    got = cq.prompt_attention(q, k, v, starts([200]), lse=lse)
    assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(lse).all())
    assert (np.abs(got[:100].cpu().double().numpy() - want[0][:100]) <= want[2][:100]).all()


def test_values_that_reach_the_types_limits(cq):  # noqa: F811
    for dtype in ("bf16", "f16"):
        big = torch.finfo(DT[dtype]).max
        q, k, v = (t.contiguous() for t in qkv(130, (2, 2, 2), 64, dtype, 18))
        v = torch.full_like(v, big)
        got = cq.prompt_attention(q, k, v, starts([130])).float()
        assert bool((got >= big * (1 - 2.0 ** -7)).all())        # (a rounding up may leave the type's range)


def test_empty_calls(cq):  # noqa: F811
    q, k, v = qkv(0, (4, 2, 2), 64, "bf16", 1)
    assert cq.prompt_attention(q, k, v, starts([])).shape == (0, 4, 64)
    assert cq.prompt_attention(q, k, v, starts([0, 0])).shape == (0, 4, 64)
    q = normal((5, 4, 64), 2, torch.bfloat16).cuda()
    lse = torch.empty(5, 4, device="cuda")
    out = cq.prompt_attention(q, k, v, starts([5]), starts([0]), lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    kept = torch.full_like(q, 2)
    cq.prompt_attention(q, q[:, :2], q[:, 2:], starts([]), out=kept)
    assert bool((kept == 2).all())


def test_equal_calls_give_equal_bits_on_streams_and_from_graphs(cq):  # noqa: F811
    q, k, v = qkv(333, (8, 2, 2), 128, "bf16", 19)
    at = starts([200, 133])
    long = [t.contiguous() for t in qkv(30, (4, 2, 2), 64, "f16", 20, 4000)]
    at_q, at_k = starts([30]), starts([4000])
    want = cq.prompt_attention(q, k, v, at), cq.prompt_attention(*long, at_q, at_k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cq.prompt_attention(q, k, v, at), cq.prompt_attention(*long, at_q, at_k)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.empty(cq.prompt_attention_workspace_bytes(1, 30, 4000, 4, 2, 64), dtype=torch.uint8, device="cuda")
    graphs, held = [], []
    for _ in range(2):                                          # two graphs with one workspace, replayed one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append((cq.prompt_attention(q, k, v, at), cq.prompt_attention(*long, at_q, at_k, workspace=ws)))
        graphs.append(g)
    for h in held:
        for t in h:
            t.zero_()
    for g in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    for h in held:
        assert all(torch.equal(a, b) for a, b in zip(h, want))
    del graphs, g


def test_offsets_that_pass_32_bits(cq):  # noqa: F811
    """Keys and values of 2.6 GB each: the last sequence's lie behind 2^31 bytes; queries and results too."""
    H, D, T = 8, 128, 1300000
    kv = torch.zeros(T, H, D, dtype=torch.bfloat16, device="cuda")
    assert kv.numel() * 2 > 1 << 31
    q, k, v = qkv(150, (H, H, H), D, "bf16", 21)
    kv[T - 150:] = k
    val = torch.zeros_like(kv)
    val[T - 150:] = v
    at = torch.tensor([T - 150, T], dtype=torch.int32, device="cuda")
    # (how the keys are split goes by the size of the whole tensors, so the bits need not be those of the small call)
    want, _, tol, _ = definition(q, k, v, [150], [150], D ** -0.5)
    got = cq.prompt_attention(q, kv, val, starts([150]), at)
    assert (np.abs(got.cpu().double().numpy() - want) <= tol).all()
    kv[T - 150:] = q                                            # now as queries
    out = torch.empty_like(kv)
    cq.prompt_attention(kv, k, v, at, starts([150]), out=out)
    assert (np.abs(out[T - 150:].cpu().double().numpy() - want) <= tol).all()


def test_binding_refuses(cq):  # noqa: F811
    q, k, v = qkv(10, (4, 2, 2), 64, "bf16", 22)
    at = starts([10])
    for bad in (dict(k=k.half()), dict(v=v[:9]), dict(k=k[:, :, :32]), dict(at=at.long()), dict(at=at[:0]), dict(at=at.cpu()),
                dict(q=q.transpose(1, 2)), dict(v=v.cpu())):
        a = {**dict(q=q, k=k, v=v, at=at), **bad}
        with pytest.raises(ValueError):
            cq.prompt_attention(a["q"], a["k"], a["v"], a["at"])
    for bad in (dict(k_starts=starts([5, 5])), dict(out=torch.empty(10, 4, 64, device="cuda")), dict(lse=torch.empty(4, 10, device="cuda")),
                dict(out=torch.empty(10, 4, 128, dtype=torch.bfloat16, device="cuda")[..., :64])):
        with pytest.raises(ValueError):
            cq.prompt_attention(q, k, v, at, **bad)
    with pytest.raises(TypeError):
        cq.prompt_attention(q.float(), k, v, at)
    for shape in ((10, 3, 64), (10, 4, 96)):                     # 3 heads over 2; a head width that is not served
        x = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(cq.CQError):
            cq.prompt_attention(x, x[:, :2], x[:, :2], at)
    flat = torch.zeros(10 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(cq.CQError):
        cq.prompt_attention(flat[1:2561].view(10, 4, 64), k, v, at)
    with pytest.raises(cq.CQError):
        cq.prompt_attention(torch.zeros(10, 4, 66, dtype=torch.bfloat16, device="cuda")[..., :64], k, v, at)
    with pytest.raises(cq.CQError):
        cq.prompt_attention(q, k[:, :1].expand(10, 2, 64), v, at)        # a head that stands for two
    long = [t.contiguous() for t in qkv(4, (4, 2, 2), 64, "bf16", 23, 4000)]
    with pytest.raises(cq.CQError):
        cq.prompt_attention(*long, starts([4]), starts([4000]), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    for scale in (0.0, -1.0, math.nan, 1e-40):
        with pytest.raises(cq.CQError):
            cq.prompt_attention(q, k, v, at, scale=scale)
