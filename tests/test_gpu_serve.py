"""The serving operators on the GPU against their plain forms (tests/serve_reference.py).

Quantizers and cache: every rounding is part of the definition, so codes, scales and read-back values are equal bit for bit.
Product: the terms of a block are added in tensor-core fp32 and the blocks by fp32 multiply-adds; 2^-12 of the sum of the terms'
magnitudes bounds both with room (a missing or doubled term of a block of 128 is 2^-7 of its sum), plus the output's rounding.
Attention: a query element is rounded to fp16 once (2^-12 of itself, with channel factors 2^-11), so a logit is off by at most
2^-11 of the sum of its terms' magnitudes (`reach`), a probability by that and 2^-12 of fp16; numerator and denominator both carry
the logits' error.  The result is within (2 * 2^-11 * reach * 1.1 + 2^-10) of the probability-weighted |v|, plus the output's rounding.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import serve_reference as ref
from guards import Arena

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}          # half an ulp at 1
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


@pytest.fixture(scope="module")
def cq():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2410_07505_b200 import build, cq as _cq
    build.build()
    _cq.lib()
    yield _cq
    assert _cq.serve_fault() == 0


def normal(shape, seed, dtype, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if outliers and shape[-1] > 8:
        x[..., 3::37] *= 25
    return x.to(dtype)


def eq_bits(got: torch.Tensor, want: np.ndarray, what: str):
    """Equal as numbers, NaN equal to NaN (a zero's sign is free)."""
    g = got.detach().cpu().double().numpy()
    np.testing.assert_array_equal(np.nan_to_num(g, nan=1e300), np.nan_to_num(np.asarray(want, np.float64), nan=1e300), err_msg=what)


# ------------------------------------------------------------------------------------------- block quantizers
def special(x: torch.Tensor) -> torch.Tensor:
    """Rows and runs of zeros, the type's extremes, subnormals, ties, infinities and NaN."""
    T, K = x.shape
    big = torch.finfo(x.dtype).max
    small = 6e-8 if x.dtype == torch.float16 else 1e-40
    for i, v in enumerate((0.0, big, -big, small, math.inf, -math.inf, math.nan)):
        if i + 1 < T:
            x[i + 1, (7 * i) % K] = v
    if T > 9:
        x[8] = 0
        x[9] = small
    if K > 130 and T > 0:
        x[0, 128:] = 0
    return x


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("T,K", ((1, 1), (1, 128), (3, 127), (5, 129), (9, 8), (17, 1000), (11, 2056), (33, 4093), (130, 1024), (8, 1032)))
def test_fp8_quantize_act(cq, dtype, T, K):
    for ld, skew in ((K, 0), (K + 8 - K % 8, 0), (K + 5, 2)):
        host = special(normal((T, K), T * K + ld, DT[dtype]))
        ar = Arena()
        ar.add("x", T * ld, DT[dtype], skew=skew)
        ar.add("codes", (T, K + (16 - K % 16)), torch.uint8)
        ar.add("scale", (-(-K // 128), T + (4 - T % 4)), torch.float32)
        ar.build()
        x = ar["x"].view(T, ld)[:, :K]
        x.copy_(host)
        ar["codes"].fill_(0x5A)
        ar["scale"].fill_(-3)
        out = cq.Fp8Act(ar["codes"].view(torch.float8_e4m3fn)[:, :K], ar["scale"][:, :T])
        assert cq.fp8_quantize_act(x, out=out) is out
        ar.check("fp8_quantize_act")
        codes, scale = ref.fp8_act(ref.f32(host))
        eq_bits(out.scale, scale, "scales")
        eq_bits(out.codes.float(), codes, "codes")
        assert bool((ar["codes"][:, K:] == 0x5A).all()) and bool((ar["scale"][:, T:] == -3).all())


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("N,K", ((1, 1), (128, 128), (127, 129), (130, 260), (300, 1000), (257, 77), (64, 1024)))
def test_fp8_quantize_weight(cq, dtype, N, K):
    for ld, skew in ((K, 0), (K + 8 - K % 8, 0), (K + 3, 2)):
        host = special(normal((N, K), N * K + ld, DT[dtype]))
        ar = Arena()
        ar.add("w", N * ld, DT[dtype], skew=skew)
        ar.add("codes", (N, K + (16 - K % 16)), torch.uint8)
        ar.add("scale", (-(-N // 128), -(-K // 128)), torch.float32)
        ar.build()
        w = ar["w"].view(N, ld)[:, :K]
        w.copy_(host)
        ar["codes"].fill_(0x5A)
        out = cq.Fp8Weight(ar["codes"].view(torch.float8_e4m3fn)[:, :K], ar["scale"])
        cq.fp8_quantize_weight(w, out=out)
        ar.check("fp8_quantize_weight")
        codes, scale = ref.fp8_weight(ref.f32(host))
        eq_bits(out.scale, scale, "scales")
        eq_bits(out.codes.float(), codes, "codes")
        assert bool((ar["codes"][:, K:] == 0x5A).all())


# ------------------------------------------------------------------------------------------- product
def operands(M, N, K, seed):
    """e4m3 operands with every kind of code, scales over several powers of two."""
    r = np.random.default_rng(seed)
    a, w = ref.round_e4m3(r.normal(0, 60, (M, K))), ref.round_e4m3(r.normal(0, 60, (N, K)))
    nb = -(-K // 128)
    sa = np.exp(r.normal(0, 2, (nb, M))).astype(np.float32)
    sw = np.exp(r.normal(-5, 2, (-(-N // 128), nb))).astype(np.float32)
    return a, sa, w, sw


def on_device(cq, a, sa, w, sw):
    (M, K), N = a.shape, w.shape[0]
    pitch = -(-K // 16) * 16
    codes = []
    for c, rows in ((a, M), (w, N)):
        full = torch.full((rows, pitch), 0x7F, dtype=torch.uint8, device="cuda")     # NaN behind the last column
        full[:, :K] = torch.from_numpy(c).float().to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        codes.append(full.view(torch.float8_e4m3fn)[:, :K])
    lds = -(-M // 4) * 4
    scale = torch.full((sa.shape[0], lds), math.nan, device="cuda")
    scale[:, :M] = torch.from_numpy(sa).cuda()
    return cq.Fp8Act(codes[0], scale[:, :M]), cq.Fp8Weight(codes[1], torch.from_numpy(sw).cuda())


def check_product(got, y, mag, dtype):
    err = np.abs(got.detach().cpu().double().numpy() - y)
    bound = 2.0 ** -12 * mag + UNIT[dtype] * np.abs(y) * 1.001 + TINY[dtype]
    assert np.isfinite(err).all() and (err <= bound).all(), f"worst {np.max(err / bound)} of the bound"


SMALL = [(M, N, K) for M in (1, 2, 16, 17, 33, 64, 65, 128, 129, 300) for N, K in ((1, 1), (127, 16), (128, 127), (129, 128), (300, 1000))]
# all lengths of the split along K, few and many tiles, several rounds of the persistent kernel, ragged last tiles and odd pitches
LARGE = [(7, 1000, 4096), (48, 512, 2049), (100, 200, 8192), (250, 130, 5000), (1300, 2000, 300), (2100, 3001, 260), (129, 20000, 128),
         (4500, 1100, 520), (700, 9000, 129)]


@pytest.mark.parametrize("M,N,K", SMALL + LARGE)
def test_fp8_matmul(cq, M, N, K):
    a, sa, w, sw = operands(M, N, K, M + N + K)
    A, W = on_device(cq, a, sa, w, sw)
    y, mag = ref.fp8_product(a, sa, w, sw)
    for dtype in (torch.bfloat16, torch.float32) if M * N < 10 ** 6 else (torch.bfloat16,):
        for ldo in (N, N + 7):
            ar = Arena()
            ar.add("out", (M, ldo), dtype)
            ar.build()
            ar["out"].fill_(7)
            out = ar["out"][:, :N]
            cq.fp8_matmul(A, W, dtype, out=out)
            ar.check("fp8_matmul")
            check_product(out, y, mag, dtype)
            assert bool((ar["out"][:, N:] == 7).all())


def test_fp8_matmul_half_outputs_and_repeats(cq):
    for M, N, K in ((5, 300, 700), (1500, 1800, 256)):
        a, sa, w, sw = operands(M, N, K, 1)
        sa, sw = sa * 0 + 0.01, sw * 0 + 0.02                           # keeps fp16 finite
        A, W = on_device(cq, a, sa, w, sw)
        y, mag = ref.fp8_product(a, sa, w, sw)
        got = cq.fp8_matmul(A, W, torch.float16)
        check_product(got, y, mag, torch.float16)
        for _ in range(3):
            assert torch.equal(got, cq.fp8_matmul(A, W, torch.float16))   # the same bits every time


# Few tiles and a long contraction of 16 blocks or more (an odd number, a partial last block, edges in both directions):
# two CTAs share a tile.  The tolerance is the one of every product.
@pytest.mark.parametrize("M,N,K", ((65, 4000, 2048), (130, 2000, 2100), (257, 1290, 2431), (500, 1999, 4000)))
def test_fp8_matmul_with_the_contraction_split(cq, M, N, K):
    a, sa, w, sw = operands(M, N, K, M + K)
    sa, sw = sa * 0 + 0.01, sw * 0 + 0.02
    A, W = on_device(cq, a, sa, w, sw)
    y, mag = ref.fp8_product(a, sa, w, sw)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        ar = Arena()
        ar.add("out", (M, N + 3), dtype)
        ar.build()
        ar["out"].fill_(7)
        out = ar["out"][:, :N]
        cq.fp8_matmul(A, W, dtype, out=out)
        ar.check("fp8_matmul")
        check_product(out, y, mag, dtype)
        assert bool((ar["out"][:, N:] == 7).all())
        assert torch.equal(out, cq.fp8_matmul(A, W, dtype))
    assert cq.serve_fault() == 0


def test_fp8_matmul_empty(cq):
    A, W = on_device(cq, *operands(5, 7, 64, 0))
    out = cq.fp8_matmul(cq.Fp8Act(A.codes[:0], A.scale[:, :0]), W)
    assert out.shape == (0, 7)
    out = torch.full((5, 7), 3.0, device="cuda", dtype=torch.bfloat16)
    empty = torch.empty((5, 16), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :0]
    empty_w = torch.empty((7, 16), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :0]
    cq.fp8_matmul(cq.Fp8Act(empty, torch.empty((0, 5), device="cuda")), cq.Fp8Weight(empty_w, torch.empty((1, 0), device="cuda")), out=out)
    assert bool((out == 0).all())


@pytest.mark.parametrize("M,N,K", ((1, 257, 385), (3, 130, 1001), (200, 300, 260), (1400, 2000, 130)))
@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_fp8_linear_is_quantize_then_product(cq, M, N, K, dtype):
    host = normal((M, K + 9), 5, DT[dtype])
    x = host.cuda()[:, 4:4 + K]                                         # a slice: odd start and pitch
    w = cq.fp8_quantize_weight((normal((N, K), 6, DT[dtype], outliers=False) * 0.02).cuda())
    ar = Arena()
    from paper_2410_07505_b200 import cq as raw
    ar.add("ws", int(raw.lib().cq_fp8_linear_workspace_bytes(M, K)), torch.uint8)
    ar.add("out", (M, N), DT[dtype])
    ar.build()
    got = cq.fp8_linear(x, w, out=ar["out"], workspace=ar["ws"])
    ar.check("fp8_linear")
    codes, scale = ref.fp8_act(ref.f32(host[:, 4:4 + K]))
    y, mag = ref.fp8_product(codes, scale, w.codes.float().cpu().double().numpy(), w.scale.cpu().numpy())
    check_product(got, y, mag, DT[dtype])
    assert torch.equal(got, cq.fp8_matmul(cq.fp8_quantize_act(x), w, DT[dtype]))


@pytest.mark.parametrize("M", (4, 200, 1500))
def test_a_block_that_is_not_finite_makes_its_rows_nan_and_no_others(cq, M):
    N, K = 1800, 300
    x = normal((M, K), 1, torch.bfloat16).cuda()
    x[1, 5], x[3, 290] = math.inf, math.nan
    w = cq.fp8_quantize_weight((normal((N, K), 2, torch.bfloat16, False) * 0.02).cuda())
    y = cq.fp8_linear(x, w)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    bad[1] = bad[3] = True
    assert bool(torch.isnan(y[bad]).all()) and bool(torch.isfinite(y[~bad]).all())


# ------------------------------------------------------------------------------------------- cache
def make_cache(cq, pages, page, H, D, bits, col, seed, poison=True):
    g = np.random.default_rng(seed)
    qmax = 127 if bits == 8 else 7
    codes = [np.clip(np.round(g.normal(0, qmax / 3.5, (pages, H, page, D))), -qmax, qmax).astype(np.int64) for _ in range(2)]
    scale = [(3.5 / qmax * np.exp(0.4 * g.normal(0, 1, (pages, H, page)))).astype(np.float32) for _ in range(2)]
    cols = [np.exp(0.7 * g.normal(0, 1, (H, D))).astype(np.float32) for _ in range(2)] if col else [None, None]
    ar = Arena()
    width, dt = (D, torch.int8) if bits == 8 else (D // 2, torch.uint8)
    for n in ("k", "v"):
        ar.add(n, (pages, H, page, width), dt)
        ar.add(n + "s", (pages, H, page), torch.float32)
    ar.build()
    for n, c, s in zip(("k", "v"), codes, scale):
        ar[n].copy_(ref.pack(c, bits))
        ar[n + "s"].copy_(torch.from_numpy(s))
    dev = [None if c is None else torch.from_numpy(c).cuda() for c in cols]
    cache = cq.KVCache(ar["k"], ar["v"], ar["ks"], ar["vs"], bits, *dev)
    return cache, codes, scale, cols, ar


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("col", (False, True))
@pytest.mark.parametrize("T,H,page,dtype", ((1, 1, 16, "bf16"), (3, 5, 48, "f16"), (130, 8, 64, "bf16"), (77, 3, 128, "f16")))
def test_kv_write_and_read(cq, bits, D, col, T, H, page, dtype):
    pages = -(-T // page) + 2
    cache, codes, scale, cols, ar = make_cache(cq, pages, page, H, D, bits, col, T)
    if col:
        for c, t in zip(cols, (cache.k_col, cache.v_col)):
            c[0, 1] = 0.0                                               # a channel that calibration never saw
            t[0, 1] = 0.0
    rng = np.random.default_rng(T)
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    skip = slots.copy()
    if T > 4:
        skip[1], skip[3], skip[4] = -1, pages * page, -(1 << 40)
    kv = []
    fused = normal((T, 3 * H, D), T + 1, DT[dtype])
    if T > 20:
        fused[5] = 0
        fused[6, :, 0] = math.inf
        fused[7, :, D - 1] = math.nan
        fused[8] *= 1e-7 if dtype == "f16" else 1e-38
        fused[9] = torch.finfo(fused.dtype).max
    for extra in (0, 1):                                                # 16-byte aligned rows, and rows that are not
        wide = torch.zeros(T, 3 * H * D + 8, dtype=DT[dtype], device="cuda")
        view = wide[:, extra:extra + 3 * H * D].view(T, 3 * H, D)
        view.copy_(fused)
        kv.append((view[:, H:2 * H], view[:, 2 * H:]))
    want = []
    for i, x in enumerate((fused[:, H:2 * H], fused[:, 2 * H:])):
        c, s = ref.kv_quantize(ref.f32(x), cols[i], bits)
        for t in range(T):
            if 0 <= skip[t] < pages * page:
                codes[i][skip[t] // page, :, skip[t] % page] = c[t]
                scale[i][skip[t] // page, :, skip[t] % page] = s[t]
        all_codes = codes[i].transpose(0, 2, 1, 3).reshape(-1, H, D)
        all_scale = scale[i].transpose(0, 2, 1).reshape(-1, H)
        want.append((codes[i], scale[i], ref.kv_values(all_codes, all_scale, cols[i])))
    for k, v in kv:
        cq.kv_write(cache, k, v, torch.from_numpy(skip).cuda())
        ar.check("kv_write")
        for (c, s, _), tc, ts in zip(want, (cache.k_codes, cache.v_codes), (cache.k_scale, cache.v_scale)):
            np.testing.assert_array_equal(ref.unpack(tc, bits), c)
            eq_bits(ts, s, "scales")
    # everything read back, in another order, with slots that name nothing
    order = np.concatenate((rng.permutation(pages * page), [-1, pages * page, 1 << 50, 0])).astype(np.int64)
    inside = (order >= 0) & (order < pages * page)
    for out in (torch.float32, torch.bfloat16, torch.float16):
        oa = Arena()
        for n in ("k", "v"):
            oa.add(n, (len(order), H, D), out)
        oa.build()
        cq.kv_read(cache, torch.from_numpy(order).cuda(), out, out=(oa["k"], oa["v"]))
        oa.check("kv_read")
        for (_, _, x), n in zip(want, ("k", "v")):
            x = np.where(inside[:, None, None], x[np.where(inside, order, 0)], 0)
            eq_bits(oa[n], torch.from_numpy(x.astype(np.float32)).to(out).double().numpy(), "values")


def test_kv_empty_calls(cq):
    cache = cq.KVCache.empty(2, 16, 2, 64, 4)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    x = torch.empty(0, 2, 64, dtype=torch.float16, device="cuda")
    cq.kv_write(cache, x, x, none)
    assert cq.kv_read(cache, none)[0].shape == (0, 2, 64)


# ------------------------------------------------------------------------------------------- attention
def build_sequences(cache_args, lens, page, seed):
    """Pages of every sequence in random order, pages behind its end unnamed (-1) or outside the cache."""
    need = [max(0, -(-n // page)) for n in lens]
    width = max(1, max(need, default=1))
    order = np.random.default_rng(seed).permutation(sum(need) + 2)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        table[b, n:] = (-7, 1 << 30, -1)[b % 3]
        at += n
    return table, sum(need) + 2


def attend_case(cq, lens, Lq, Hq, H, D, page, bits, col, dtype, seed=0, scale=None, q_pad=0, with_lse=True):
    table, pages = build_sequences(None, lens, page, seed)
    cache, codes, scales, cols, ar = make_cache(cq, pages, page, H, D, bits, col, seed + 1)
    for b, n in enumerate(lens):                                        # behind the end: NaN, infinities, the largest float
        if n > 0 and n % page:
            for s, bad in zip((cache.k_scale, cache.v_scale), (math.nan, math.inf)):
                s[int(table[b, n // page]), :, n % page:] = bad
    B = len(lens)
    q = (normal((B, Lq, Hq, D), seed + 2, DT[dtype], outliers=False) * 1.3).to(DT[dtype])
    wide = torch.zeros(B, Lq, Hq, D + q_pad, dtype=DT[dtype], device="cuda")
    dev_q = wide[..., q_pad:]
    dev_q.copy_(q)
    oa = Arena()
    oa.add("out", (B, Lq, Hq, D), DT[dtype])
    oa.add("lse", (B, Lq, Hq), torch.float32)
    oa.add("ws", cq.kv_attention_workspace_bytes(D), torch.uint8)
    oa.build()
    oa["ws"].fill_(0xFF)                                                # NaN wherever something unwritten is read
    cq.kv_attention(dev_q, cache, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                    scale=scale, out=oa["out"], lse=oa["lse"] if with_lse else None, workspace=oa["ws"])
    oa.check("kv_attention")
    ar.check("kv_attention (cache)")
    sc = D ** -0.5 if scale is None else scale
    got, got_lse = oa["out"].cpu().double().numpy(), oa["lse"].cpu().double().numpy()
    G = Hq // H
    for b, n in enumerate(lens):
        n = max(n, 0)
        at = table[b, :-(-n // page)]
        for h in range(H):
            kv = []
            for c, s, f in zip(codes, scales, cols):
                x = c[at][:, h].reshape(-1, D)[:n].astype(np.float64) * s[at][:, h].reshape(-1, 1)[:n]
                kv.append(x if f is None else x * f[h].astype(np.float64))
            heads = np.s_[b, :, h * G:(h + 1) * G]
            out, lse, reach, mag = ref.attention(q[heads].double().numpy(), kv[0], kv[1], sc)
            reach = reach[..., None]
            bound = (2 * 2.0 ** -11 * 1.1 * reach + 2.0 ** -10) * mag + UNIT[DT[dtype]] * np.abs(out) * 1.001 + 2.0 ** -24
            err = np.abs(got[heads] - out)
            assert np.isfinite(got[heads]).all()
            assert (err <= bound).all(), f"sequence {b} head {h}: worst {np.max(err / bound)} of the bound"
            if with_lse:
                le = got_lse[heads]
                assert np.array_equal(np.isneginf(le), np.isneginf(lse))
                fin = np.isfinite(lse)
                assert (np.abs(le - np.where(fin, lse, 0))[fin] <= (2.0 ** -11 * 1.1 * reach[..., 0] + 2.0 ** -16 * (1 + np.abs(np.where(fin, lse, 0))))[fin]).all()
    return oa["out"].clone(), (dev_q, cache, torch.from_numpy(table).cuda())


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("Lq,Hq,H", ((1, 1, 1), (1, 8, 1), (1, 12, 4), (3, 10, 2), (4, 8, 1), (5, 16, 2), (9, 16, 2)))
def test_attention_at_the_edges_of_tiles(cq, bits, D, Lq, Hq, H):
    lens = [1, 0, 15, 16, 17, 63, 64, 65, 2, 127, 129, 3]
    attend_case(cq, lens, Lq, Hq, H, D, 16, bits, bits == 4, "bf16", seed=Lq)


@pytest.mark.parametrize("page", (16, 48, 64, 128, 1024))
@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_attention_over_pages(cq, page, bits, dtype):
    attend_case(cq, [700, 33, 1100, 0, 1], 2, 6, 2, 128, page, bits, True, dtype, seed=page)
    attend_case(cq, [350, 1025], 1, 4, 4, 64, page, bits, False, dtype, seed=page + 1)


@pytest.mark.parametrize("lens,Lq,Hq,H,D,bits", (([20001], 1, 2, 1, 128, 8), ([20001], 1, 1, 1, 64, 4), ([9000, 7, 0, 12000], 4, 8, 1, 128, 4),
                                                 ([3000] * 3, 1, 40, 40, 128, 8), (list(range(0, 900, 9)), 1, 6, 2, 64, 8),
                                                 ([5000, 300], 40, 4, 2, 64, 8), ([1500] * 2, 70, 2, 1, 128, 4)))
def test_attention_cut_over_many_ctas(cq, lens, Lq, Hq, H, D, bits):
    attend_case(cq, lens, Lq, Hq, H, D, 64, bits, True, "bf16", seed=3)


def test_attention_large_and_small_scales(cq):
    attend_case(cq, [500, 77], 2, 4, 2, 128, 16, 8, True, "f16", seed=9, scale=4.0)      # one token takes it all
    attend_case(cq, [500, 77], 2, 4, 2, 128, 16, 8, True, "bf16", seed=9, scale=1e-6)    # a plain mean


def test_attention_strided_queries_and_no_lse(cq):
    for pad in (1, 4, 8):
        attend_case(cq, [100, 300], 3, 6, 3, 64, 32, 8, False, "bf16", seed=pad, q_pad=pad, with_lse=False)


def test_attention_more_sequences_than_lanes(cq):
    attend_case(cq, [int(n) for n in np.random.default_rng(1).integers(0, 200, 150)], 1, 2, 1, 64, 16, 8, False, "f16", seed=4)


def test_attention_repeats_bit_for_bit_and_ignores_other_sequences(cq):
    out, (q, cache, table) = attend_case(cq, [3000, 500, 40, 0, 999], 1, 8, 2, 128, 16, 8, True, "bf16", seed=8)
    lens = torch.tensor([3000, 500, 40, 0, 999], dtype=torch.int32, device="cuda")
    for _ in range(3):
        assert torch.equal(out, cq.kv_attention(q, cache, table, lens))
    cache.k_scale[table[1, 3].long()] = math.nan                         # a broken token in sequence 1 stays there
    got = cq.kv_attention(q, cache, table, lens)
    assert bool(torch.isnan(got[1]).all()) and torch.equal(got[[0, 2, 3, 4]], out[[0, 2, 3, 4]])


def test_attention_cuts_lens_and_leaves_out_pages_outside_the_cache(cq):
    out, (q, cache, table) = attend_case(cq, [64, 128], 1, 4, 2, 64, 64, 8, False, "bf16", seed=2)
    table = table.clone()
    table[0, 1] = 1 << 30
    lens = torch.tensor([10 ** 9, 128], dtype=torch.int32, device="cuda")   # cut to 128; the second page names nothing
    got = cq.kv_attention(q, cache, table, lens)
    torch.testing.assert_close(got[0].float(), out[0].float(), rtol=2.0 ** -7, atol=1e-6)
    assert torch.equal(got[1], out[1])
    gone = cq.kv_attention(q, cache, torch.full_like(table, -1), lens)
    assert bool((gone == 0).all())
    minus = cq.kv_attention(q, cache, table, torch.full_like(lens, -5))
    assert bool((minus == 0).all())
    empty = cq.kv_attention(q, cache, table[:, :0], lens)
    assert bool((empty == 0).all())


def test_attention_with_infinite_and_huge_queries(cq):
    out, (q, cache, table) = attend_case(cq, [200, 200], 1, 4, 2, 64, 64, 8, False, "bf16", seed=6)
    lens = torch.tensor([200, 200], dtype=torch.int32, device="cuda")
    q = q.clone()
    q[0, 0, 1, 3] = math.inf
    q[1, 0, 2] = 0
    got = cq.kv_attention(q, cache, table, lens)
    assert bool(torch.isnan(got[0, 0, 1]).all()) and torch.equal(got[0, 0, [0, 2, 3]], out[0, 0, [0, 2, 3]])
    assert torch.equal(got[1, 0, [0, 1, 3]], out[1, 0, [0, 1, 3]])
    v = ref.unpack(cache.v_codes[table[1, :4].long()], 8).transpose(1, 0, 2, 3).reshape(2, -1, 64)[1, :200]
    s = cache.v_scale[table[1, :4].long()].cpu().double().numpy().transpose(1, 0, 2).reshape(2, -1)[1, :200]
    mean = (v * s[:, None]).mean(axis=0)                                 # a query of zeros: the mean of the values
    weight = (np.abs(v) * s[:, None]).mean(axis=0)
    assert (np.abs(got[1, 0, 2].cpu().double().numpy() - mean) <= 2.0 ** -10 * weight + UNIT[torch.bfloat16] * np.abs(mean) * 1.001).all()


def test_cache_whose_offsets_pass_32_bits(cq):
    """2.4 GB of codes each for keys and values: the last pages lie behind 2^31 bytes."""
    page, H, D = 128, 8, 128
    pages = (2400 << 20) // (page * H * D)
    cache = cq.KVCache.empty(pages, page, H, D, 8)
    assert cache.k_codes.numel() > 1 << 31
    n = 200
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page] * page + at % page
    x = normal((n, 2 * H, D), 3, torch.bfloat16).cuda()
    cq.kv_write(cache, x[:, :H], x[:, H:], slots)
    k, v = cq.kv_read(cache, slots, torch.float32)
    for got, src in ((k, x[:, :H]), (v, x[:, H:])):
        c, s = ref.kv_quantize(ref.f32(src), None, 8)
        eq_bits(got, ref.kv_values(c, s, None), "values")
    q = normal((1, 1, H, D), 4, torch.bfloat16, False).cuda()
    got = cq.kv_attention(q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    for h in range(H):
        out, _, reach, mag = ref.attention(q[0, :, h:h + 1].cpu().double().numpy(), k[:, h].cpu().double().numpy(), v[:, h].cpu().double().numpy(), D ** -0.5)
        bound = (2 * 2.0 ** -11 * 1.1 * reach[..., None] + 2.0 ** -10) * mag + UNIT[torch.bfloat16] * np.abs(out) * 1.001 + 2.0 ** -24
        assert (np.abs(got[0, :, h:h + 1].cpu().double().numpy() - out) <= bound).all()


# ------------------------------------------------------------------------------------------- as they are used
def test_operators_on_another_stream_and_from_a_graph(cq):
    M, N, K, H, D = 6, 1000, 768, 4, 64
    x = normal((M, K), 1, torch.bfloat16).cuda()
    w = cq.fp8_quantize_weight((normal((N, K), 2, torch.bfloat16, False) * 0.02).cuda())
    cache = cq.KVCache.empty(8, 32, H, D, 4)
    kv = normal((M, 2 * H, D), 3, torch.bfloat16).cuda()
    q = normal((1, 2, H, D), 4, torch.bfloat16, False).cuda()
    slots = torch.tensor([32, 33, 34, 35, 36, 37], device="cuda")
    table, lens = torch.tensor([[1, 2]], dtype=torch.int32, device="cuda"), torch.tensor([M], dtype=torch.int32, device="cuda")

    def step():
        cq.kv_write(cache, kv[:, :H], kv[:, H:], slots)
        return cq.fp8_linear(x, w), *cq.kv_read(cache, slots), cq.kv_attention(q, cache, table, lens)
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for t in held:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(held, want):
        assert torch.equal(a, b)
    del graph


def test_binding_refuses_what_the_kernels_could_not_check(cq):
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    w = cq.fp8_quantize_weight(x)
    with pytest.raises(ValueError):
        cq.fp8_linear(x[:, :128], w)
    with pytest.raises(ValueError):
        cq.fp8_linear(x, cq.Fp8Weight(w.codes, w.scale[:, :1]))
    with pytest.raises(ValueError):
        cq.fp8_linear(x, w, out=torch.empty(4, 5, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        cq.fp8_linear(x.t(), w)
    with pytest.raises(cq.CQError):
        cq.fp8_linear(x, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(cq.CQError):                                      # a row pitch that is no multiple of 16
        odd = torch.empty(4, 264, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :256]
        cq.fp8_linear(x, cq.Fp8Weight(odd, w.scale))
    cache = cq.KVCache.empty(2, 16, 2, 64)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        cq.kv_write(cache, k, k[:2], slots)
    with pytest.raises(ValueError):
        cq.kv_write(cache, k, k.half(), slots)
    with pytest.raises(ValueError):
        cq.kv_write(cache, k, k, slots.int())
    with pytest.raises(ValueError):
        cq.kv_read(cache, slots, out=(k, k.float()))
    with pytest.raises(cq.CQError):
        cq.KVCache.empty(2, 16, 2, 80) and cq.kv_read(cq.KVCache.empty(2, 16, 2, 80), slots)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    for bad in (dict(q=q[:, :, :, :32]), dict(table=table.long()), dict(lens=lens.long()), dict(table=table[:0]), dict(lens=lens[:0])):
        a = {**dict(q=q, table=table, lens=lens), **bad}
        with pytest.raises(ValueError):
            cq.kv_attention(a["q"], cache, a["table"], a["lens"])
    with pytest.raises(cq.CQError):
        cq.kv_attention(q[:, :, :3], cache, table, lens)                 # 3 query heads over 2
