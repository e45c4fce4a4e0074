// The quantized key/value cache: tokens quantized as they are written, and read back.
//
// Write (keys and values in one launch; one head of one token = one row x_1..x_D under one scale, Eq. 1 on the row):
//   u = fl32(x * fl32(1 / factor)) (u = x without factors),  a = fl32(max |u| / qmax),  code = rint(fl32(u / a))
// The row's scale is fitted to the token as it arrives, so no code is ever clipped whatever the channel factors are;
// a factor of 0 gives codes 0.  A row with an infinity or NaN gets a scale that is one and codes 0: it reads back as NaN.
// Read:
//   xhat = fl32(code * fl32(a * factor)), rounded once more to 16 bits
//
// Both are bound by HBM (write: 2 bytes in, 1 or 1/2 out; read: the reverse).  A thread keeps one place in the row and
// walks over the tokens, so that channel factors are loaded (and inverted) once, and loads for its next tokens before it
// works on these.
#include "cq_kv.cuh"

#include <type_traits>

namespace cq {

// Tokens of one thread.  Of each it takes eight elements in either half of the row, so that a warp's 16-byte accesses lie side
// by side: 16 neighbouring elements would touch every 32-byte sector twice (read of 4096 tokens of 40 heads: 43 against 31 us).
// All blocks are resident at once, so that none runs a second, partial round (write: 30.6 us with two blocks an SM and 104 registers,
// 37 with three and 80, 38 with three in two rounds; read, 20011 tokens of 32 INT4 heads: 37.5 us with four blocks, 43 with three).
constexpr int kWriteTokens = 2, kWriteBlocks = 2;
constexpr int kReadTokens = 4, kReadBlocks = 4;

// Slots, rows and threads all stay below 2^31, so that divisions are 32-bit (the 64-bit ones took most of the write's time:
// 64 us for 4096 tokens of 40 heads, against 127 MB); a page size that is a power of two needs none.
struct PageMap {
    int size, shift;                // shift < 0: not a power of two
    __device__ __forceinline__ uint32_t row(uint32_t slot, int H, int h) const {
        const uint32_t page = shift >= 0 ? slot >> shift : slot / static_cast<uint32_t>(size);
        return (page * H + h) * size + (slot - page * size);
    }
};

struct WriteArgs {
    const uint16_t* x[2];            // keys, values [T][H][D]
    int64_t ts[2], hs[2];            // strides of tokens and heads, in elements
    uint8_t* codes[2];
    float* scale[2];
    const float* col[2];
    const int64_t* slots;
    int64_t T, nslots;
    PageMap pages;
    int H, parts, rounds;            // tokens are dealt out in groups to `parts` walkers, in so many rounds
};

// (a parameter indexed by a run-time number would be copied to local memory first)
template <typename P>
__device__ __forceinline__ P pick(const P (&two)[2], int kv) { return kv != 0 ? two[1] : two[0]; }

__device__ __forceinline__ float max_nan(float a, float b) {          // NaN if either is (a positive one: its pattern is above all)
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// eight elements in the order of memory, as floats would need them, from any 2-byte aligned place
template <bool VEC>
__device__ __forceinline__ uint4 load_row8(const uint16_t* p) {
    if constexpr (VEC) {
        return ld_stream(reinterpret_cast<const uint4*>(p));
    } else {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = p[e];
        return make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
    }
}

// Codes (as kMagic + q) of eight floats u under the scale a.  The candidate rint(u * fl32(1 / a)) is off the quotient by
// less than 2 * 2^-24 * 127.0001, so it stands unless the product lies within 2^-14 of a rounding boundary.
template <int BITS>
__device__ __forceinline__ void codes_of_floats(const float2 (&u)[4], float a, float ra, float2 (&y)[4]) {
    constexpr float qmaxf = static_cast<float>((1 << (BITS - 1)) - 1);
    const float2 ra2 = make_float2(ra, ra), m2 = make_float2(kMagic, kMagic), nm2 = make_float2(-kMagic, -kMagic);
    const float2 neg1 = make_float2(-1.0f, -1.0f);
    float worst = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 v = __fmul2_rn(u[k], ra2);
        y[k] = __fadd2_rn(v, m2);
        const float2 f = __ffma2_rn(__fadd2_rn(y[k], nm2), neg1, v);
        worst = fmaxf(fmaxf(worst, fabsf(f.x)), fabsf(f.y));
    }
    if (!(ra == ra && worst < kAcceptBelow)) {                // only what is undecided is settled by a division
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 v = __fmul2_rn(u[k], ra2);
            const float2 f = __ffma2_rn(__fadd2_rn(y[k], nm2), neg1, v);
            if (!(ra == ra && fabsf(f.x) < kAcceptBelow)) y[k].x = quant_exact(u[k].x, a, qmaxf);
            if (!(ra == ra && fabsf(f.y) < kAcceptBelow)) y[k].y = quant_exact(u[k].y, a, qmaxf);
        }
    }
}

template <int D, int DT, int BITS, bool VEC, bool COL>
__global__ void __launch_bounds__(kThreads, kWriteBlocks)
k14_kv_write(const WriteArgs p) {
    constexpr float qmaxf = static_cast<float>((1 << (BITS - 1)) - 1);
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int kv = blockIdx.y;
    constexpr uint32_t lanes = D / 16;                         // threads of a row: 4 or 8, an aligned part of a warp
    const uint32_t hv = p.H * lanes;
    const uint32_t gid = blockIdx.x * kThreads + threadIdx.x;
    const int part = gid / hv, at = gid - part * hv;
    const int64_t T = part < p.parts ? p.T : 0;               // the last block may reach beyond the last part
    const int h = at / lanes, v = at % lanes;
    const uint16_t* src = pick(p.x, kv) + h * pick(p.hs, kv) + v * 8;
    const int64_t ts = pick(p.ts, kv);
    uint4 w[kWriteTokens][2], w_next[kWriteTokens][2];
    int64_t slot[kWriteTokens], slot_next[kWriteTokens];
    auto load = [&](int64_t group) {
#pragma unroll
        for (int i = 0; i < kWriteTokens; ++i) {
            const int64_t t = group * kWriteTokens + i;
            w_next[i][0] = w_next[i][1] = make_uint4(0, 0, 0, 0);
            slot_next[i] = -1;
            if (t < T) {
                slot_next[i] = p.slots[t];
                w_next[i][0] = load_row8<VEC>(src + t * ts);
                w_next[i][1] = load_row8<VEC>(src + t * ts + D / 2);
            }
        }
    };
    load(part);
    float2 r[8];
    if constexpr (COL) {
        const float4* c = reinterpret_cast<const float4*>(pick(p.col, kv) + h * D + v * 8);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 f = c[(k >> 1) * (D / 8) + (k & 1)];
            r[2 * k] = make_float2(f.x > 0.0f ? __frcp_rn(f.x) : 0.0f, f.y > 0.0f ? __frcp_rn(f.y) : 0.0f);
            r[2 * k + 1] = make_float2(f.z > 0.0f ? __frcp_rn(f.z) : 0.0f, f.w > 0.0f ? __frcp_rn(f.w) : 0.0f);
        }
    }
    for (int it = 0; it < p.rounds; ++it) {                   // as many for all threads: lanes of a warp may be of two parts
#pragma unroll
    for (int i = 0; i < kWriteTokens; ++i) {
        w[i][0] = w_next[i][0];
        w[i][1] = w_next[i][1];
        slot[i] = slot_next[i];
    }
    if (it + 1 < p.rounds) load(part + static_cast<int64_t>(it + 1) * p.parts);
#pragma unroll
    for (int i = 0; i < kWriteTokens; ++i) {
        float2 u[2][4], y[2][4];
        float a;
        uint32_t m = 0;                                       // as a bit pattern: NaN is largest
        if constexpr (COL) {
            float top = 0.0f;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t words[4] = {w[i][q].x, w[i][q].y, w[i][q].z, w[i][q].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    u[q][k] = __fmul2_rn(unpack16x2<DT>(words[k]), r[4 * q + k]);
                    top = max_nan(max_nan(top, fabsf(u[q][k].x)), fabsf(u[q][k].y));
                }
            }
            m = __float_as_uint(top);
        } else {
            uint32_t mm = 0;
#pragma unroll
            for (int q = 0; q < 2; ++q)
                mm = max_u16x2(mm, max_u16x2(max_u16x2(w[i][q].x & 0x7FFF7FFFu, w[i][q].y & 0x7FFF7FFFu),
                                             max_u16x2(w[i][q].z & 0x7FFF7FFFu, w[i][q].w & 0x7FFF7FFFu)));
            m = max(mm & 0xFFFFu, mm >> 16);
        }
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        if constexpr (lanes == 8) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
        a = __fdiv_rn(COL ? __uint_as_float(m) : cvt16<DT>(static_cast<uint16_t>(m)), qmaxf);
        const float ra = guarded_rcp(a);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (!(a <= 3.402823466e38f)) {
#pragma unroll
                for (int k = 0; k < 4; ++k) y[q][k] = make_float2(kMagic, kMagic);
            } else if constexpr (COL) {
                codes_of_floats<BITS>(u[q], a, ra, y[q]);
            } else if (ra == ra) {
                exact_codes_uniform_row8<DT>(w[i][q], a, ra, y[q]);
            } else {
                exact_codes_uniform_slow<DT, BITS>(w[i][q], a, y[q]);
            }
        }
        if (slot[i] < 0 || slot[i] >= p.nslots) continue;
        const uint64_t row = p.pages.row(static_cast<uint32_t>(slot[i]), p.H, h);
        if (v == 0) pick(p.scale, kv)[row] = a;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if constexpr (BITS == 8)
                *reinterpret_cast<uint2*>(pick(p.codes, kv) + row * D + q * (D / 2) + v * 8) =
                    make_uint2(pack_int8x4(y[q][0].x, y[q][0].y, y[q][1].x, y[q][1].y), pack_int8x4(y[q][2].x, y[q][2].y, y[q][3].x, y[q][3].y));
            else
                *reinterpret_cast<uint32_t*>(pick(p.codes, kv) + row * (D / 2) + q * (D / 4) + v * 4) = pack_int4x8(y[q]);
        }
    }
    }
}

struct ReadArgs {
    KvCache c;
    void* out[2];                    // [L][H][D], dense
    const int64_t* slots;
    int64_t L, nslots;
    PageMap pages;
    int parts, rounds;
};

// four int8 codes / eight nibbles of a word as floats: the biased code in the low bits of 2^23, minus 2^23 and the bias
__device__ __forceinline__ void codes_to_float2(uint32_t w, float2 (&f)[2]) {
    const uint32_t b = w ^ 0x80808080u;
    const float2 off = make_float2(-8388736.0f, -8388736.0f);
#pragma unroll
    for (int e = 0; e < 2; ++e)
        f[e] = __fadd2_rn(make_float2(__uint_as_float(__byte_perm(b, 0x4B000000u, 0x7440u + 2 * e)),
                                      __uint_as_float(__byte_perm(b, 0x4B000000u, 0x7441u + 2 * e))), off);
}
__device__ __forceinline__ float nibble_float(uint32_t w, int shift) {          // ((w >> shift) & 15) ^ 8 in the low bits of 2^23
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(r) : "r"(w >> shift), "r"(0xFu), "r"(0x4B000008u));      // (a & b) ^ c
    return __uint_as_float(r);
}
__device__ __forceinline__ void nibbles_to_float2(uint32_t w, float2 (&f)[4]) {
    const float2 off = make_float2(-8388616.0f, -8388616.0f);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __fadd2_rn(make_float2(nibble_float(w, 8 * e), nibble_float(w, 8 * e + 4)), off);
}

template <int D, int OUT, int BITS, bool COL>
__global__ void __launch_bounds__(kThreads, kReadBlocks)
k15_kv_read(const ReadArgs p) {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int kv = blockIdx.y;
    constexpr uint32_t lanes = D / 16;
    const uint32_t hv = p.c.H * lanes;
    const uint32_t gid = blockIdx.x * kThreads + threadIdx.x;
    const int part = gid / hv, at = gid - part * hv;
    const int64_t L = part < p.parts ? p.L : 0;               // the last block may reach beyond the last part
    const int h = at / lanes, v = at % lanes;
    int64_t slot_next[kReadTokens];
    auto name = [&](int64_t t0) {
#pragma unroll
        for (int i = 0; i < kReadTokens; ++i) slot_next[i] = t0 + i < L ? p.slots[t0 + i] : -1;
    };
    name(static_cast<int64_t>(part) * kReadTokens);
    float2 col[8];
    if constexpr (COL) {
        const float4* c = reinterpret_cast<const float4*>(pick(p.c.col, kv) + h * D + v * 8);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 f = c[(k >> 1) * (D / 8) + (k & 1)];
            col[2 * k] = make_float2(f.x, f.y);
            col[2 * k + 1] = make_float2(f.z, f.w);
        }
    }
    for (int it = 0; it < p.rounds; ++it) {
    const int64_t t0 = (part + static_cast<int64_t>(it) * p.parts) * kReadTokens;
    const int64_t o0 = (t0 * p.c.H + h) * D + v * 8;
    int64_t slot[kReadTokens];
#pragma unroll
    for (int i = 0; i < kReadTokens; ++i) slot[i] = slot_next[i];
    if (it + 1 < p.rounds) name(t0 + static_cast<int64_t>(p.parts) * kReadTokens);
    uint4 w[kReadTokens];
    float a[kReadTokens];
#pragma unroll
    for (int i = 0; i < kReadTokens; ++i) {
        w[i] = make_uint4(0, 0, 0, 0);
        a[i] = 0.0f;
        if (slot[i] >= 0 && slot[i] < p.nslots) {
            const uint64_t row = p.pages.row(static_cast<uint32_t>(slot[i]), p.c.H, h);
            a[i] = pick(p.c.scale, kv)[row];
            if constexpr (BITS == 8) {
                const uint2* src = reinterpret_cast<const uint2*>(pick(p.c.codes, kv) + row * D + v * 8);
                const uint2 lo = __ldcs(src), hi = __ldcs(src + D / 16);
                w[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
            } else {
                const uint32_t* src = reinterpret_cast<const uint32_t*>(pick(p.c.codes, kv) + row * (D / 2) + v * 4);
                w[i].x = __ldcs(src);
                w[i].y = __ldcs(src + D / 16);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kReadTokens; ++i) {
        if (t0 + i >= L) break;
        float2 x[8];
        if constexpr (BITS == 8) {
            const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float2 f[2];
                codes_to_float2(words[k], f);
                x[2 * k] = f[0]; x[2 * k + 1] = f[1];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float2 f[4];
                nibbles_to_float2(k == 0 ? w[i].x : w[i].y, f);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * k + e] = f[e];
            }
        }
        const float2 a2 = make_float2(a[i], a[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __fmul2_rn(x[e], COL ? __fmul2_rn(a2, col[e]) : a2);
        const int64_t o = o0 + static_cast<int64_t>(i) * p.c.H * D;
        if constexpr (OUT == CQ_F32) {
            float4* out = reinterpret_cast<float4*>(static_cast<float*>(pick(p.out, kv)) + o);
#pragma unroll
            for (int k = 0; k < 4; ++k) st_stream(out + (k >> 1) * (D / 8) + (k & 1), make_float4(x[2 * k].x, x[2 * k].y, x[2 * k + 1].x, x[2 * k + 1].y));
        } else {
            uint4* out = reinterpret_cast<uint4*>(static_cast<uint16_t*>(pick(p.out, kv)) + o);
#pragma unroll
            for (int k = 0; k < 2; ++k)
                st_stream(out + k * (D / 16), make_uint4(pack16x2<OUT>(x[4 * k].x, x[4 * k].y), pack16x2<OUT>(x[4 * k + 1].x, x[4 * k + 1].y),
                                              pack16x2<OUT>(x[4 * k + 2].x, x[4 * k + 2].y), pack16x2<OUT>(x[4 * k + 3].x, x[4 * k + 3].y)));
        }
    }
    }
}

int check_cache(const void* k_codes, const void* v_codes, const void* k_scale, const void* v_scale, const void* k_col,
                const void* v_col, int bits, int64_t pages, int64_t page_size, int64_t H, int64_t D) {
    if (bits != 4 && bits != 8) return CQ_ERR_BITS;
    if (pages < 0 || H < 1 || H > 4096 || page_size < 16 || page_size > 4096 || page_size % 16 != 0 || (D != 64 && D != 128))
        return CQ_ERR_SHAPE;
    if (pages * H * page_size > (int64_t(1) << 31) - 4096 || pages > (int64_t(1) << 31) / 16) return CQ_ERR_SHAPE;   // rows a tensor map can count
    if ((k_col == nullptr) != (v_col == nullptr)) return CQ_ERR_NULL;
    if (pages > 0 && (k_codes == nullptr || v_codes == nullptr || k_scale == nullptr || v_scale == nullptr)) return CQ_ERR_NULL;
    if (!ptr_aligned(k_codes, 16) || !ptr_aligned(v_codes, 16) || !ptr_aligned(k_scale, 16) || !ptr_aligned(v_scale, 16) ||
        !ptr_aligned(k_col, 16) || !ptr_aligned(v_col, 16)) return CQ_ERR_ALIGN;
    return CQ_OK;
}

// How many walkers of `width` threads share the groups of tokens (about so many blocks an SM for keys and values
// together, one round where there is less), and the blocks that they fill.
static int64_t deal(int64_t tokens, int64_t per_group, int64_t width, int blocks_per_sm, int& parts, int& rounds) {
    const int64_t groups = (tokens + per_group - 1) / per_group;
    int64_t n = int64_t(sm_count()) * blocks_per_sm * kThreads / 2 / width;
    n = n < 1 ? 1 : n > groups ? groups : n;
    rounds = static_cast<int>((groups + n - 1) / n);
    n = (groups + rounds - 1) / rounds;                       // no part without work in the last round where it can be helped
    parts = static_cast<int>(n);
    return (n * width + kThreads - 1) / kThreads;
}

static PageMap page_map(int64_t page_size) {
    int shift = 0;
    while ((int64_t(1) << shift) < page_size) ++shift;
    return {static_cast<int>(page_size), (int64_t(1) << shift) == page_size ? shift : -1};
}

template <int D, int DT, int BITS>
static int launch_write(const WriteArgs& p, bool vec, dim3 grid, cudaStream_t st) {
    if (p.col[0] != nullptr) {
        if (vec) return launch_ex(k14_kv_write<D, DT, BITS, true, true>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
        else return launch_ex(k14_kv_write<D, DT, BITS, false, true>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
    } else {
        if (vec) return launch_ex(k14_kv_write<D, DT, BITS, true, false>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
        else return launch_ex(k14_kv_write<D, DT, BITS, false, false>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
    }
}

template <int D, int OUT>
static int launch_read(const ReadArgs& p, int bits, dim3 grid, cudaStream_t st) {
    const bool col = p.c.col[0] != nullptr;
    if (bits == 8) {
        if (col) return launch_ex(k15_kv_read<D, OUT, 8, true>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
        else return launch_ex(k15_kv_read<D, OUT, 8, false>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
    } else {
        if (col) return launch_ex(k15_kv_read<D, OUT, 4, true>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
        else return launch_ex(k15_kv_read<D, OUT, 4, false>, grid, kThreads, 0, st, 1, !tuning_no_pdl(), p);
    }
}

}  // namespace cq

extern "C" {

int cq_kv_write(const void* K, int64_t k_token_stride, int64_t k_head_stride, const void* V, int64_t v_token_stride,
                int64_t v_head_stride, int dtype, int64_t T, const int64_t* slots, void* k_codes, void* v_codes,
                float* k_scale, float* v_scale, const float* k_col, const float* v_col, int bits, int64_t pages,
                int64_t page_size, int64_t H, int64_t D, void* stream) {
    using namespace cq;
    const int rc = check_cache(k_codes, v_codes, k_scale, v_scale, k_col, v_col, bits, pages, page_size, H, D);
    if (rc != CQ_OK) return rc;
    if (dtype != CQ_F16 && dtype != CQ_BF16) return CQ_ERR_DTYPE;
    if (T < 0 || T > (int64_t(1) << 31) - 1024) return CQ_ERR_SHAPE;
    if (T == 0 || pages == 0) return CQ_OK;
    if (K == nullptr || V == nullptr || slots == nullptr) return CQ_ERR_NULL;
    if (!ptr_aligned(K, 2) || !ptr_aligned(V, 2) || !ptr_aligned(slots, 8)) return CQ_ERR_ALIGN;
    WriteArgs p;
    p.x[0] = static_cast<const uint16_t*>(K); p.x[1] = static_cast<const uint16_t*>(V);
    p.ts[0] = k_token_stride; p.ts[1] = v_token_stride; p.hs[0] = k_head_stride; p.hs[1] = v_head_stride;
    p.codes[0] = static_cast<uint8_t*>(k_codes); p.codes[1] = static_cast<uint8_t*>(v_codes);
    p.scale[0] = k_scale; p.scale[1] = v_scale; p.col[0] = k_col; p.col[1] = v_col;
    p.slots = slots; p.T = T; p.nslots = pages * page_size;
    p.pages = page_map(page_size); p.H = static_cast<int>(H);
    const int64_t blocks = deal(T, kWriteTokens, H * (D / 16), kWriteBlocks, p.parts, p.rounds);
    const bool vec = ptr_aligned(K, 16) && ptr_aligned(V, 16) &&
                     ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7) == 0;
    const dim3 grid(static_cast<unsigned>(blocks), 2);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto d, auto dt) {
        return bits == 8 ? launch_write<d.value, dt.value, 8>(p, vec, grid, st) : launch_write<d.value, dt.value, 4>(p, vec, grid, st);
    };
    using std::integral_constant;
    if (D == 128) return dtype == CQ_F16 ? go(integral_constant<int, 128>{}, integral_constant<int, CQ_F16>{}) : go(integral_constant<int, 128>{}, integral_constant<int, CQ_BF16>{});
    return dtype == CQ_F16 ? go(integral_constant<int, 64>{}, integral_constant<int, CQ_F16>{}) : go(integral_constant<int, 64>{}, integral_constant<int, CQ_BF16>{});
}

int cq_kv_read(const void* k_codes, const void* v_codes, const float* k_scale, const float* v_scale, const float* k_col,
               const float* v_col, int bits, int64_t pages, int64_t page_size, int64_t H, int64_t D, int64_t L,
               const int64_t* slots, void* k_out, void* v_out, int out_dtype, void* stream) {
    using namespace cq;
    const int rc = check_cache(k_codes, v_codes, k_scale, v_scale, k_col, v_col, bits, pages, page_size, H, D);
    if (rc != CQ_OK) return rc;
    if (out_dtype != CQ_F16 && out_dtype != CQ_BF16 && out_dtype != CQ_F32) return CQ_ERR_DTYPE;
    if (L < 0 || L > (int64_t(1) << 31) - 1024) return CQ_ERR_SHAPE;
    if (L == 0) return CQ_OK;
    if (slots == nullptr || k_out == nullptr || v_out == nullptr) return CQ_ERR_NULL;
    if (!ptr_aligned(slots, 8) || !ptr_aligned(k_out, 16) || !ptr_aligned(v_out, 16)) return CQ_ERR_ALIGN;
    ReadArgs p;
    p.c = KvCache{{static_cast<const int8_t*>(k_codes), static_cast<const int8_t*>(v_codes)}, {k_scale, v_scale}, {k_col, v_col},
                  pages, static_cast<int>(page_size), static_cast<int>(H), static_cast<int>(D)};
    p.out[0] = k_out; p.out[1] = v_out; p.slots = slots; p.L = L; p.nslots = pages * page_size;
    p.pages = page_map(page_size);
    const int64_t blocks = deal(L, kReadTokens, H * (D / 16), kReadBlocks, p.parts, p.rounds);
    const dim3 grid(static_cast<unsigned>(blocks), 2);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (D == 128) return out_dtype == CQ_F32 ? launch_read<128, CQ_F32>(p, bits, grid, st)
                       : out_dtype == CQ_F16 ? launch_read<128, CQ_F16>(p, bits, grid, st) : launch_read<128, CQ_BF16>(p, bits, grid, st);
    return out_dtype == CQ_F32 ? launch_read<64, CQ_F32>(p, bits, grid, st)
         : out_dtype == CQ_F16 ? launch_read<64, CQ_F16>(p, bits, grid, st) : launch_read<64, CQ_BF16>(p, bits, grid, st);
}

}  // extern "C"
