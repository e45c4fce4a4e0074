// Block quantization to 8-bit floats (e4m3): activations with one scale for each run of 128 elements of a row,
// weights with one scale for each 128 x 128 block.
//
//   s = fl32(max |x| / 448),  code = e4m3(fl32(x / s)),  s == 0 -> code 0
//
// 448 is e4m3's largest value.  448 = 7 * 2^6, so s has the mantissa of the INT4 scales fl32(max / 7), and the
// division-free exact quotient that the integer weight quantizers use for 16-bit elements holds here as it stands.
// A block with an infinity or NaN gets a scale that is one (the maximum is taken over the bit patterns, where NaN is
// largest), so that everything computed from the block is NaN rather than a wrong number.
//
// Both are bound by HBM: 2 bytes read and 1 byte written for an element, the block's maximum found in registers.
// Measured, tensors larger than L2: weights 28672 x 8192 109 us (6.5 TB/s, 99 % of a copy's rate; up to 127 us behind work that
// has lowered the clocks); 1003 x 2060, 7 to 9 us, is latency.  Activations 4096 x 8192 19.9 us (5.1 TB/s), 1 x 8192 2.3 us.
#include "cq_serve.cuh"

namespace cq {

constexpr float kE4m3Max = 448.0f;
constexpr int kBlk = 128;

// (Plain loads, here and in the other kernels that start before the one in front of them has ended, not the read-only
// path: that is for memory that nobody writes while the kernel exists.)
// Eight neighbouring elements from any 2-byte aligned place, of which the first n are inside the row (the others read as
// zeros): whole words as far as the address allows, never a byte outside the row.
__device__ __forceinline__ uint4 load8_any(const uint16_t* p, int64_t n) {
    if (n >= 8) {
        const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p));
        if ((at & 15u) == 0u) return ld_stream(reinterpret_cast<const uint4*>(p));
        if ((at & 3u) == 0u) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p + 1);
        const uint32_t a = p[0], b = w[0], c = w[1], d = w[2], e = p[7];
        return make_uint4(a | (b << 16), __funnelshift_l(b, c, 16), __funnelshift_l(c, d, 16), (d >> 16) | (e << 16));
    }
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = e < n ? p[e] : 0u;
    return make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
}
// The first n of eight codes to any place.
__device__ __forceinline__ void store8_any(uint8_t* p, uint2 c, int64_t n) {
    if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 7u) == 0u) {
        *reinterpret_cast<uint2*>(p) = c;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = static_cast<uint8_t>((e < 4 ? c.x : c.y) >> (8 * (e & 3)));
}

__device__ __forceinline__ uint32_t absmax8(const uint4& w) {
    const uint32_t m = max_u16x2(max_u16x2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), max_u16x2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu));
    return max(m & 0xFFFFu, m >> 16);
}

__device__ __forceinline__ float e4m3_quotient_slow(float x, float s) {
    if (s == 0.0f) return 0.0f;
    const float u = __fdiv_rn(x, s);
    return u > kE4m3Max ? kE4m3Max : (u < -kE4m3Max ? -kE4m3Max : u);      // NaN stays NaN
}

// Eight elements under one scale -> eight codes.  rs = guarded_rcp(s): NaN where the short form does not hold.
template <int DT>
__device__ __forceinline__ uint2 e4m3_row8(const uint4& w, float s, float rs) {
    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
    uint32_t h[4];
    if (rs == rs) {
        const float2 rs2 = make_float2(rs, rs), ns2 = make_float2(-s, -s);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 x = unpack16x2<DT>(words[k]);
            const float2 q0 = __fmul2_rn(x, rs2);
            const float2 u = __ffma2_rn(__ffma2_rn(q0, ns2, x), rs2, q0);
            h[k] = pack_e4m3x2(u.x, u.y);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 x = unpack16x2<DT>(words[k]);
            h[k] = pack_e4m3x2(e4m3_quotient_slow(x.x, s), e4m3_quotient_slow(x.y, s));
        }
    }
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

// ---- activations --------------------------------------------------------------------------------
// A warp takes one row x 1024 columns (four 16-byte loads a lane, all issued first; 16 lanes hold a block), a CTA
// eight consecutive rows, whose scales leave as whole 32-byte sectors of the block-major scale matrix.
constexpr int kActVec = 4;
constexpr int kActRows = 8;
constexpr int kActCols = 256 * kActVec;

// VEC: all rows and codes are aligned and K is a multiple of 8; otherwise each warp goes by its row's address.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kThreads)
k10_fp8_act(const uint16_t* X, int64_t T, int64_t K, int64_t ld, uint8_t* codes, int64_t ldc,
            float* scale, int64_t lds, unsigned col_chunks) {
    __shared__ float s_scale[2 * kActVec][kActRows];
    // Launched while the kernel before it may still run: everything waits for that one's end.  Only then may the product
    // be launched, which loads weights ahead of its own wait: whatever wrote them is done by then.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned chunk = blockIdx.x % col_chunks;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x / col_chunks) * kActRows;
    const int64_t row = row0 + warp;
    const int64_t col0 = static_cast<int64_t>(chunk) * kActCols + lane * 8;
    uint4 w[kActVec];
#pragma unroll
    for (int k = 0; k < kActVec; ++k) {
        const int64_t col = col0 + 256 * k;
        w[k] = make_uint4(0, 0, 0, 0);
        if (row < T && col < K) {
            if constexpr (VEC) w[k] = ld_stream(reinterpret_cast<const uint4*>(X + row * ld + col));
            else w[k] = load8_any(X + row * ld + col, K - col);
        }
    }
#pragma unroll
    for (int k = 0; k < kActVec; ++k) {
        uint32_t m = absmax8(w[k]);
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
        const float s = __fdiv_rn(cvt16<DT>(static_cast<uint16_t>(m)), kE4m3Max);
        const uint2 c = e4m3_row8<DT>(w[k], s, guarded_rcp(s));
        const int64_t col = col0 + 256 * k;
        if (row < T && col < K) {
            if constexpr (VEC) *reinterpret_cast<uint2*>(codes + row * ldc + col) = c;
            else store8_any(codes + row * ldc + col, c, K - col);
        }
        if ((lane & 15) == 0) s_scale[2 * k + (lane >> 4)][warp] = s;
    }
    __syncthreads();
    if (threadIdx.x < 2 * kActVec * kActRows) {
        const int b = threadIdx.x / kActRows, r = threadIdx.x % kActRows;
        const int64_t blk = static_cast<int64_t>(chunk) * (2 * kActVec) + b;
        if (blk * kBlk < K && row0 + r < T) scale[blk * lds + row0 + r] = s_scale[b][r];
    }
}

// ---- weights --------------------------------------------------------------------------------------
// One CTA per 128 x 128 block, held in registers between the maximum and the codes (eight 16-byte loads a thread).
// (64 registers, four CTAs an SM: enough loads in flight.  Five spill, 144 us; CTAs that walk over blocks with the next one's
// loads ahead of this one's codes: 129 us with two an SM, 125 with three.)
template <int DT, bool VEC>
__global__ void __launch_bounds__(kThreads)
k11_fp8_weight(const uint16_t* __restrict__ W, int64_t N, int64_t K, int64_t ld, uint8_t* __restrict__ codes, int64_t ldc,
               float* __restrict__ scale, int64_t kblocks) {
    __shared__ uint32_t s_max[kThreads / 32];
    const int64_t nb = blockIdx.x / kblocks, kb = blockIdx.x % kblocks;
    const int64_t col = kb * kBlk + (threadIdx.x & 15) * 8;
    const int64_t row0 = nb * kBlk + (threadIdx.x >> 4);
    uint4 w[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + 16 * i;
        w[i] = make_uint4(0, 0, 0, 0);
        if constexpr (VEC) {
            if (row < N && col < K) w[i] = ld_stream(reinterpret_cast<const uint4*>(W + row * ld + col));
        } else {
            if (row < N && col < K) w[i] = load8_any(W + row * ld + col, K - col);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, absmax8(w[i]));
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) m = max(m, s_max[i]);
    const float s = __fdiv_rn(cvt16<DT>(static_cast<uint16_t>(m)), kE4m3Max);
    const float rs = guarded_rcp(s);
    if (threadIdx.x == 0) scale[nb * kblocks + kb] = s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + 16 * i;
        if (row >= N || col >= K) continue;
        const uint2 c = e4m3_row8<DT>(w[i], s, rs);
        if constexpr (VEC) st_stream(reinterpret_cast<uint2*>(codes + row * ldc + col), c);
        else store8_any(codes + row * ldc + col, c, K - col);
    }
}

static int check_codes(const void* codes, int64_t rows, int64_t K, int64_t ldc, const float* scale) {
    if (ldc < K) return CQ_ERR_SHAPE;
    if (rows > 0 && K > 0) {
        if (codes == nullptr || scale == nullptr) return CQ_ERR_NULL;
        if (!ptr_aligned(scale, 4)) return CQ_ERR_ALIGN;
    }
    return CQ_OK;
}

int fp8_quantize_act_impl(const void* X, int dtype, int64_t T, int64_t K, int64_t ld, void* codes, int64_t ldc,
                          float* scale, int64_t lds, cudaStream_t st) {
    int rc = check_matrix(X, dtype, T, K, ld);
    if (rc == CQ_OK) rc = check_codes(codes, T, K, ldc, scale);
    if (rc != CQ_OK) return rc;
    if (lds < T) return CQ_ERR_SHAPE;
    if (T == 0 || K == 0) return CQ_OK;
    const bool vec = K % 8 == 0 && ld % 8 == 0 && ldc % 8 == 0 && ptr_aligned(X, 16) && ptr_aligned(codes, 8);
    const int64_t chunks = (K + kActCols - 1) / kActCols;
    const int64_t blocks = chunks * ((T + kActRows - 1) / kActRows);
    if (blocks > 0x7FFFFFFF) return CQ_ERR_SHAPE;
    auto kern = dtype == CQ_F16 ? (vec ? k10_fp8_act<CQ_F16, true> : k10_fp8_act<CQ_F16, false>)
                                : (vec ? k10_fp8_act<CQ_BF16, true> : k10_fp8_act<CQ_BF16, false>);
    return launch_ex(kern, dim3(static_cast<unsigned>(blocks)), kThreads, 0, st, 1, !tuning_no_pdl(), static_cast<const uint16_t*>(X), T, K, ld,
                     static_cast<uint8_t*>(codes), ldc, scale, lds, static_cast<unsigned>(chunks));
}

}  // namespace cq

extern "C" {

int cq_fp8_quantize_act(const void* X, int dtype, int64_t T, int64_t K, int64_t ld, void* codes, int64_t ldc,
                        float* scale, int64_t lds, void* stream) {
    return cq::fp8_quantize_act_impl(X, dtype, T, K, ld, codes, ldc, scale, lds, static_cast<cudaStream_t>(stream));
}

int cq_fp8_quantize_weight(const void* W, int dtype, int64_t N, int64_t K, int64_t ld, void* codes, int64_t ldc,
                           float* scale, void* stream) {
    using namespace cq;
    int rc = check_matrix(W, dtype, N, K, ld);
    if (rc == CQ_OK) rc = check_codes(codes, N, K, ldc, scale);
    if (rc != CQ_OK) return rc;
    if (N == 0 || K == 0) return CQ_OK;
    const int64_t kblocks = (K + kBlk - 1) / kBlk, blocks = kblocks * ((N + kBlk - 1) / kBlk);
    if (blocks > 0x7FFFFFFF) return CQ_ERR_SHAPE;
    const bool vec = K % 8 == 0 && ld % 8 == 0 && ldc % 8 == 0 && ptr_aligned(W, 16) && ptr_aligned(codes, 8);
    auto kern = dtype == CQ_F16 ? (vec ? k11_fp8_weight<CQ_F16, true> : k11_fp8_weight<CQ_F16, false>)
                                : (vec ? k11_fp8_weight<CQ_BF16, true> : k11_fp8_weight<CQ_BF16, false>);
    kern<<<static_cast<unsigned>(blocks), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
        static_cast<const uint16_t*>(W), N, K, ld, static_cast<uint8_t*>(codes), ldc, scale, kblocks);
    return launch_status();
}

}  // extern "C"
