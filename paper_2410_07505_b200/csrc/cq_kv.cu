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
// takes several tokens, so that channel factors are loaded (and inverted) once and all loads are issued first.
#include "cq_kv.cuh"

#include <type_traits>

namespace cq {

constexpr int kWriteTokens = 2;     // tokens of one thread: write (16 elements of each)
constexpr int kReadTokens = 4;      // and read (8 elements of each, so that neighbours' stores are neighbours)

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
    int H;
};

// (a parameter indexed by a run-time number would be copied to local memory first)
template <typename P>
__device__ __forceinline__ P pick(const P (&two)[2], int kv) { return kv != 0 ? two[1] : two[0]; }

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
    if (!(ra == ra && worst < kAcceptBelow)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float y0 = quant_exact(u[k].x, a, qmaxf), y1 = quant_exact(u[k].y, a, qmaxf);
            y[k] = make_float2(y0, y1);
        }
    }
}

template <int D, int DT, int BITS, bool VEC, bool COL>
__global__ void __launch_bounds__(kThreads)
k14_kv_write(const WriteArgs p) {
    constexpr float qmaxf = static_cast<float>((1 << (BITS - 1)) - 1);
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int kv = blockIdx.y;
    constexpr uint32_t lanes = D / 16;                         // threads of a row: 4 or 8, an aligned part of a warp
    const uint32_t hv = p.H * lanes;
    const uint32_t gid = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t group = gid / hv, at = gid - group * hv;
    const int h = at / lanes, v = at % lanes;
    const uint16_t* src = pick(p.x, kv) + h * pick(p.hs, kv) + v * 16;
    uint4 w[kWriteTokens][2];
    int64_t slot[kWriteTokens];
#pragma unroll
    for (int i = 0; i < kWriteTokens; ++i) {
        const int64_t t = static_cast<int64_t>(group) * kWriteTokens + i;
        w[i][0] = w[i][1] = make_uint4(0, 0, 0, 0);
        slot[i] = -1;
        if (t < p.T) {
            slot[i] = __ldg(p.slots + t);
            w[i][0] = load_row8<VEC>(src + t * pick(p.ts, kv));
            w[i][1] = load_row8<VEC>(src + t * pick(p.ts, kv) + 8);
        }
    }
    float2 r[8];
    if constexpr (COL) {
        const float4* c = reinterpret_cast<const float4*>(pick(p.col, kv) + h * D + v * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 f = __ldg(c + k);
            r[2 * k] = make_float2(f.x > 0.0f ? __frcp_rn(f.x) : 0.0f, f.y > 0.0f ? __frcp_rn(f.y) : 0.0f);
            r[2 * k + 1] = make_float2(f.z > 0.0f ? __frcp_rn(f.z) : 0.0f, f.w > 0.0f ? __frcp_rn(f.w) : 0.0f);
        }
    }
#pragma unroll
    for (int i = 0; i < kWriteTokens; ++i) {
        float2 u[2][4], y[2][4];
        float a;
        uint32_t m = 0;                                       // over bit patterns: NaN is largest
        if constexpr (COL) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t words[4] = {w[i][q].x, w[i][q].y, w[i][q].z, w[i][q].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    u[q][k] = __fmul2_rn(unpack16x2<DT>(words[k]), r[4 * q + k]);
                    m = max(m, max(__float_as_uint(u[q][k].x) & 0x7FFFFFFFu, __float_as_uint(u[q][k].y) & 0x7FFFFFFFu));
                }
            }
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
        if constexpr (BITS == 8)
            *reinterpret_cast<uint4*>(pick(p.codes, kv) + row * D + v * 16) =
                make_uint4(pack_int8x4(y[0][0].x, y[0][0].y, y[0][1].x, y[0][1].y), pack_int8x4(y[0][2].x, y[0][2].y, y[0][3].x, y[0][3].y),
                           pack_int8x4(y[1][0].x, y[1][0].y, y[1][1].x, y[1][1].y), pack_int8x4(y[1][2].x, y[1][2].y, y[1][3].x, y[1][3].y));
        else
            *reinterpret_cast<uint2*>(pick(p.codes, kv) + row * (D / 2) + v * 8) = make_uint2(pack_int4x8(y[0]), pack_int4x8(y[1]));
    }
}

struct ReadArgs {
    KvCache c;
    void* out[2];                    // [L][H][D], dense
    const int64_t* slots;
    int64_t L, nslots;
    PageMap pages;
};

// four int8 codes / eight nibbles of a word as floats: the biased code in the low bits of 2^23, minus 2^23 and the bias
__device__ __forceinline__ void codes_to_float4(uint32_t w, float (&f)[4]) {
    const uint32_t b = w ^ 0x80808080u;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __fadd_rn(__uint_as_float(__byte_perm(b, 0x4B000000u, 0x7440u + e)), -8388736.0f);
}
__device__ __forceinline__ void nibbles_to_float8(uint32_t w, float (&f)[8]) {
    const uint32_t b = w ^ 0x88888888u;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __fadd_rn(__uint_as_float(((b >> (4 * e)) & 0xFu) | 0x4B000000u), -8388616.0f);
}

template <int D, int OUT, int BITS, bool COL>
__global__ void __launch_bounds__(kThreads)
k15_kv_read(const ReadArgs p) {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int kv = blockIdx.y;
    constexpr uint32_t lanes = D / 8;
    const uint32_t hv = p.c.H * lanes;
    const uint32_t gid = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t group = gid / hv, at = gid - group * hv;
    const int h = at / lanes, v = at % lanes;
    const int64_t t0 = static_cast<int64_t>(group) * kReadTokens;
    if (t0 >= p.L) return;
    const int64_t o0 = (t0 * p.c.H + h) * D + v * 8;
    uint2 w[kReadTokens];
    float a[kReadTokens];
    int64_t slot[kReadTokens];
#pragma unroll
    for (int i = 0; i < kReadTokens; ++i) slot[i] = t0 + i < p.L ? __ldg(p.slots + t0 + i) : -1;
#pragma unroll
    for (int i = 0; i < kReadTokens; ++i) {
        w[i] = make_uint2(0, 0);
        a[i] = 0.0f;
        if (slot[i] >= 0 && slot[i] < p.nslots) {
            const uint64_t row = p.pages.row(static_cast<uint32_t>(slot[i]), p.c.H, h);
            a[i] = __ldg(pick(p.c.scale, kv) + row);
            if constexpr (BITS == 8) w[i] = __ldcs(reinterpret_cast<const uint2*>(pick(p.c.codes, kv) + row * D + v * 8));
            else w[i].x = __ldcs(reinterpret_cast<const uint32_t*>(pick(p.c.codes, kv) + row * (D / 2) + v * 4));
        }
    }
    float col[8];
    if constexpr (COL) {
        const float4* c = reinterpret_cast<const float4*>(pick(p.c.col, kv) + h * D + v * 8);
        const float4 f0 = __ldg(c), f1 = __ldg(c + 1);
        col[0] = f0.x; col[1] = f0.y; col[2] = f0.z; col[3] = f0.w;
        col[4] = f1.x; col[5] = f1.y; col[6] = f1.z; col[7] = f1.w;
    }
#pragma unroll
    for (int i = 0; i < kReadTokens; ++i) {
        const int64_t t = t0 + i;
        if (t >= p.L) break;
        float x[8];
        if constexpr (BITS == 8) {
            float f[4];
            codes_to_float4(w[i].x, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = f[e];
            codes_to_float4(w[i].y, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 + e] = f[e];
        } else {
            nibbles_to_float8(w[i].x, x);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float s = a[i];
            if constexpr (COL) s = __fmul_rn(s, col[e]);
            x[e] = __fmul_rn(x[e], s);
        }
        const int64_t o = o0 + static_cast<int64_t>(i) * p.c.H * D;
        if constexpr (OUT == CQ_F32) {
            float4* out = reinterpret_cast<float4*>(static_cast<float*>(pick(p.out, kv)) + o);
            st_stream(out, make_float4(x[0], x[1], x[2], x[3]));
            st_stream(out + 1, make_float4(x[4], x[5], x[6], x[7]));
        } else {
            st_stream(reinterpret_cast<uint4*>(static_cast<uint16_t*>(pick(p.out, kv)) + o),
                      make_uint4(pack16x2<OUT>(x[0], x[1]), pack16x2<OUT>(x[2], x[3]), pack16x2<OUT>(x[4], x[5]), pack16x2<OUT>(x[6], x[7])));
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
    const int64_t threads = ((T + kWriteTokens - 1) / kWriteTokens) * H * (D / 16);
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    if (blocks * kThreads > 0x7FFFFFFF) return CQ_ERR_SHAPE;
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
    const int64_t threads = ((L + kReadTokens - 1) / kReadTokens) * H * (D / 8);
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    if (blocks * kThreads > 0x7FFFFFFF) return CQ_ERR_SHAPE;
    const dim3 grid(static_cast<unsigned>(blocks), 2);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (D == 128) return out_dtype == CQ_F32 ? launch_read<128, CQ_F32>(p, bits, grid, st)
                       : out_dtype == CQ_F16 ? launch_read<128, CQ_F16>(p, bits, grid, st) : launch_read<128, CQ_BF16>(p, bits, grid, st);
    return out_dtype == CQ_F32 ? launch_read<64, CQ_F32>(p, bits, grid, st)
         : out_dtype == CQ_F16 ? launch_read<64, CQ_F16>(p, bits, grid, st) : launch_read<64, CQ_BF16>(p, bits, grid, st);
}

}  // extern "C"
