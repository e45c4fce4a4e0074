// Norms of queries and keys for each head, and the rotation by position, in one pass.
//
//   y_d = w_d x_d / sqrt(mean_d x_d^2 + eps)   (y = x without norms),   then for each pair (a, b) of the first R channels
//   (a, b) -> (a cos f - b sin f, a sin f + b cos f),   f = position * freq[pair]
//
// Bound by HBM (2 bytes in, 2 out).  A row's channels lie eight to a lane, so that its mean is a few shuffles and a pair is either in
// one lane (neighbours) or one shuffle away (halves).  The angles of a token are the same for all of its heads: a block forms those of
// a few tokens at a time, as a fraction of a turn in 64 bits (position * freq passes 2^24 radians, where 32 bits hold no angle), and
// each lane keeps its token's, times the weights: an element then costs a product, a multiply-add and the row's factor.
#include "cq_serve.cuh"

#include <algorithm>

namespace cq {

constexpr int kRotateThreads = 256;
constexpr int kMaxHeadDim = 512, kMaxRotated = 512;

struct RotateSide {                           // queries or keys
    const uint16_t* x; int64_t xt, xh;        // strides of tokens and heads
    uint16_t* y; int64_t yt, yh;
    const uint16_t* w;                        // null: ones
    int heads;
};
struct RotateArgs {
    RotateSide side[2];
    const int64_t* positions; const double* freq;
    int64_t T;
    int D, R;
    bool norm, neighbours;
    double eps;
    int slices;                               // blocks that share a token's heads
    int group;                                // tokens that a block takes at a time
};

// cos and sin of position * freq[i] for `group` tokens from t0 on: [token][R / 2]
__device__ __forceinline__ void angles(const RotateArgs& p, int64_t t0, float* s_cos, float* s_sin) {
    const int half = p.R / 2;
    for (int at = threadIdx.x; at < p.group * half; at += kRotateThreads) {
        const int token = at / half, i = at - token * half;
        if (t0 + token >= p.T) break;
        const double turns = static_cast<double>(p.positions[t0 + token]) * (p.freq[i] * 0.15915494309189535);
        sincospif(2.0f * static_cast<float>(turns - rint(turns)), s_sin + at, s_cos + at);
    }
}

// the sum of a row's squares in 64 bits, on all W lanes
template <int W, int DT>
__device__ __noinline__ double row_squares(uint4 x) {
    double sum = 0.0;
    const uint32_t r[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 e = unpack16x2<DT>(r[i]);
        sum += static_cast<double>(e.x) * e.x + static_cast<double>(e.y) * e.y;
    }
#pragma unroll
    for (int off = W / 2; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off, W);
    return sum;
}
// 1 / sqrt(mean + eps)
__device__ __noinline__ double wide_factor(double sum, int D, double eps) { return 1.0 / sqrt(sum / D + eps); }

template <int DT>
__device__ __forceinline__ void unpack8(const uint4& w, float (&v)[8]) {
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack16x2<DT>(r[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// W lanes for a row, eight channels each; rows in 16-byte accesses, R a multiple of 16.  The block's rows are `group` tokens x
// kRows / group heads at a time.
constexpr int kMaxGroup = 8;
constexpr int kFastDim = 256;

template <int W, int DT, bool NORM, bool NEAR>                 // NEAR: neighbours are pairs
__global__ void __launch_bounds__(kRotateThreads, 3)
k24_norm_rotate(const RotateArgs p) {
    constexpr int kRows = kRotateThreads / W;
    constexpr int kAhead = 4;                                   // rows whose loads are issued together
    __shared__ float s_cos[2][kMaxGroup * kFastDim / 2], s_sin[2][kMaxGroup * kFastDim / 2];
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x % W, row = threadIdx.x / W;
    const int token = row % p.group, first = row / p.group, step = kRows / p.group;
    const int d0 = lane * 8;
    const bool have = d0 < p.D;
    const int half = p.R / 2;
    const bool rotated = d0 < p.R, second = d0 >= half;
    // the lane with the other channels of this one's pairs (halves), and the first of its angles
    const int partner = NEAR || !rotated ? lane : second ? lane - half / 8 : lane + half / 8;
    const int angle0 = NEAR ? d0 / 2 : second ? d0 - half : d0;
    const int slice = blockIdx.x % p.slices;
    const int64_t stride = static_cast<int64_t>(gridDim.x / p.slices) * p.group;
    int buffer = 0;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x / p.slices) * p.group; t0 < p.T; t0 += stride, buffer ^= 1) {
        const int64_t t = t0 + token;
        bool ready = false;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const RotateSide& a = p.side[kv];
            const int h0 = static_cast<int>(static_cast<int64_t>(a.heads) * slice / p.slices), h1 = static_cast<int>(static_cast<int64_t>(a.heads) * (slice + 1) / p.slices);
            // this lane's heads: h0 + first, every `step`-th, `rows` of them; `most` of any lane of the block
            const bool live = have && t < p.T;
            const int rows = live && h1 - h0 > first ? (h1 - h0 - first + step - 1) / step : 0, most = (h1 - h0 + step - 1) / step;
            const uint16_t* x_at = a.x + t * a.xt + (h0 + first) * a.xh + d0;
            uint16_t* y_at = a.y + t * a.yt + (h0 + first) * a.yh + d0;
            const int64_t x_step = step * a.xh, y_step = step * a.yh;
            float c[8], s[8];                                   // y = (x c + partner s) factor
            for (int done = 0; done < most || (kv == 0 && !ready); done += kAhead) {
                uint4 x[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    x[u] = make_uint4(0, 0, 0, 0);
                    if (done + u < rows) x[u] = __ldcs(reinterpret_cast<const uint4*>(x_at));
                    x_at += x_step;
                }
                if (done == 0) {                                // (behind the first loads)
                    if (!ready) {
                        angles(p, t0, s_cos[buffer], s_sin[buffer]);
                        __syncthreads();
                        ready = true;
                    }
                    float w[8], wp[8];
                    if (NORM && a.w != nullptr && have) {
                        unpack8<DT>(*reinterpret_cast<const uint4*>(a.w + d0), w);
                        unpack8<DT>(*reinterpret_cast<const uint4*>(a.w + partner * 8), wp);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = wp[i] = 1.0f;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = token * half + angle0 + (NEAR ? i / 2 : i);
                        const bool later = NEAR ? (i & 1) != 0 : second;
                        const float other = NEAR ? w[i ^ 1] : wp[i];
                        c[i] = rotated ? s_cos[buffer][at] * w[i] : w[i];
                        s[i] = rotated ? (later ? s_sin[buffer][at] : -s_sin[buffer][at]) * other : 0.0f;
                    }
                }
                float f[kAhead];
                uint32_t moved = 0;                             // bits u, u + 4: row u is moved by 2^64, by 2^-64
                if constexpr (NORM) {
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        float v[8];
                        unpack8<DT>(x[u], v);
                        f[u] = 0.0f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[u] = __fmaf_rn(v[i], v[i], f[u]);
                    }
#pragma unroll
                    for (int off = W / 2; off > 0; off >>= 1)
#pragma unroll
                        for (int u = 0; u < kAhead; ++u) f[u] += __shfl_xor_sync(0xFFFFFFFFu, f[u], off, W);
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (done + u < rows && !(f[u] > 1e-25f && f[u] < 1e35f)) moved |= f[u] > 1.0f ? 16u << u : 1u << u;
                    const bool any = __any_sync(0xFFFFFFFFu, moved != 0u);
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const float mean = __fmaf_rn(f[u], 1.0f / static_cast<float>(p.D), static_cast<float>(p.eps));
                        if (any) {                              // squares that fp32 cannot hold, or that are all zero: the sum in 64 bits
                            const double wide = row_squares<W, DT>(x[u]);
                            if (moved >> u & 0x11u) f[u] = static_cast<float>(wide_factor(wide, p.D, p.eps) * (moved >> u & 1u ? 0x1p-64 : 0x1p64));
                            else f[u] = rsqrtf(mean);
                        } else {
                            f[u] = rsqrtf(mean);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (done + u >= most) break;                // the same for the whole block
                    float v[8], o[8];
                    unpack8<DT>(x[u], v);
                    if constexpr (NEAR) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) o[i] = rotated ? v[i ^ 1] : 0.0f;      // (an infinity times a sine of 0)
                    } else {
                        uint4 xp;
                        xp.x = __shfl_sync(0xFFFFFFFFu, x[u].x, partner, W);
                        xp.y = __shfl_sync(0xFFFFFFFFu, x[u].y, partner, W);
                        xp.z = __shfl_sync(0xFFFFFFFFu, x[u].z, partner, W);
                        xp.w = __shfl_sync(0xFFFFFFFFu, x[u].w, partner, W);
                        if (!rotated) xp = make_uint4(0, 0, 0, 0);
                        unpack8<DT>(xp, o);
                    }
                    if (NORM && (moved >> u & 0x11u)) {
                        const float move = moved >> u & 1u ? 0x1p64f : 0x1p-64f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) { v[i] *= move; o[i] *= move; }
                    }
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        y[i] = __fmaf_rn(v[i], c[i], o[i] * s[i]);
                        if constexpr (NORM) y[i] *= f[u];
                    }
                    if (done + u < rows)
                        *reinterpret_cast<uint4*>(y_at) =
                            make_uint4(pack16x2<DT>(y[0], y[1]), pack16x2<DT>(y[2], y[3]), pack16x2<DT>(y[4], y[5]), pack16x2<DT>(y[6], y[7]));
                    y_at += y_step;
                }
            }
        }
    }
}

// Any even R and any 2-byte aligned rows: a warp for a row, through shared memory.
template <int DT>
__global__ void __launch_bounds__(kRotateThreads)
k24_norm_rotate_any(const RotateArgs p) {
    constexpr int kWarps = kRotateThreads / 32;
    __shared__ float s_cos[2][kMaxRotated / 2], s_sin[2][kMaxRotated / 2], s_row[kWarps][kMaxHeadDim];
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = p.R / 2;
    const int slice = blockIdx.x % p.slices;
    int buffer = 0;
    for (int64_t t = blockIdx.x / p.slices; t < p.T; t += gridDim.x / p.slices, buffer ^= 1) {
        angles(p, t, s_cos[buffer], s_sin[buffer]);
        __syncthreads();
        for (int kv = 0; kv < 2; ++kv) {
            const RotateSide a = kv == 0 ? p.side[0] : p.side[1];
            const int h0 = static_cast<int>(static_cast<int64_t>(a.heads) * slice / p.slices), h1 = static_cast<int>(static_cast<int64_t>(a.heads) * (slice + 1) / p.slices);
            for (int h = h0 + warp; h < h1; h += kWarps) {
                const uint16_t* x = a.x + t * a.xt + h * a.xh;
                uint16_t* y = a.y + t * a.yt + h * a.yh;
                double sum = 0.0;
                for (int d = lane; d < p.D; d += 32) {
                    const float v = cvt16<DT>(x[d]);
                    s_row[warp][d] = v;
                    sum += static_cast<double>(v) * v;
                }
                if (p.norm) {
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
                    const double f = wide_factor(sum, p.D, p.eps);
                    for (int d = lane; d < p.D; d += 32)
                        s_row[warp][d] = static_cast<float>(s_row[warp][d] * f) * (a.w != nullptr ? cvt16<DT>(a.w[d]) : 1.0f);
                }
                __syncwarp();
                for (int d = lane; d < p.D; d += 32) {
                    float v = s_row[warp][d];
                    if (d < p.R) {
                        const int pair = p.neighbours ? d / 2 : d < half ? d : d - half;
                        const bool later = p.neighbours ? (d & 1) != 0 : d >= half;
                        const float o = s_row[warp][p.neighbours ? d ^ 1 : later ? d - half : d + half];
                        const float sn = s_sin[buffer][pair];
                        v = __fmaf_rn(v, s_cos[buffer][pair], o * (later ? sn : -sn));
                    }
                    y[d] = pack16<DT>(v);
                }
                __syncwarp();
            }
        }
    }
}

template <int W, int DT, bool NORM>
static int launch_rotate_pairs(const RotateArgs& p, dim3 grid, cudaStream_t st) {
    if (p.neighbours) return launch_ex(k24_norm_rotate<W, DT, NORM, true>, grid, kRotateThreads, 0, st, 1, !tuning_no_pdl(), p);
    return launch_ex(k24_norm_rotate<W, DT, NORM, false>, grid, kRotateThreads, 0, st, 1, !tuning_no_pdl(), p);
}
template <int W, int DT>
static int launch_rotate_rows(const RotateArgs& p, dim3 grid, cudaStream_t st) {
    return p.norm ? launch_rotate_pairs<W, DT, true>(p, grid, st) : launch_rotate_pairs<W, DT, false>(p, grid, st);
}

template <int DT>
static int launch_rotate(RotateArgs& p, bool fast, cudaStream_t st) {
    const int W = p.D <= 64 ? 8 : p.D <= 128 ? 16 : 32;
    const int rows = fast ? kRotateThreads / W : kRotateThreads / 32;
    const int heads = std::max(p.side[0].heads, p.side[1].heads);
    // As many tokens at a time as leave all SMs some blocks; few tokens: a token's heads are shared out, a pass to a block.
    p.group = 1;
    while (fast && p.group < kMaxGroup && p.T / (2 * p.group) >= 2 * sm_count()) p.group *= 2;
    const int64_t groups = (p.T + p.group - 1) / p.group;
    const int64_t most = std::max(1, (heads + rows - 1) / rows);
    p.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, 6 * sm_count() / groups)));
    const int64_t blocks = std::min<int64_t>(groups, std::max(1, 48 * sm_count() / p.slices));
    const dim3 grid(static_cast<unsigned>(blocks * p.slices));
    if (!fast) return launch_ex(k24_norm_rotate_any<DT>, grid, kRotateThreads, 0, st, 1, !tuning_no_pdl(), p);
    if (W == 8) return launch_rotate_rows<8, DT>(p, grid, st);
    if (W == 16) return launch_rotate_rows<16, DT>(p, grid, st);
    return launch_rotate_rows<32, DT>(p, grid, st);
}

}  // namespace cq

extern "C" int cq_norm_rotate(const void* Q, int64_t q_token_stride, int64_t q_head_stride, int64_t Hq, const void* K, int64_t k_token_stride,
                              int64_t k_head_stride, int64_t H, int dtype, int64_t T, int64_t D, int64_t R, int neighbours,
                              const int64_t* positions, const double* freq, const void* q_weight, const void* k_weight, double eps,
                              void* q_out, int64_t qo_token_stride, int64_t qo_head_stride, void* k_out, int64_t ko_token_stride,
                              int64_t ko_head_stride, void* stream) {
    using namespace cq;
    if (dtype != CQ_F16 && dtype != CQ_BF16) return CQ_ERR_DTYPE;
    if (T < 0 || T > (int64_t(1) << 31) - 1024 || Hq < 0 || H < 0 || Hq > (1 << 16) || H > (1 << 16) || D < 1 || D > kMaxHeadDim || R < 0 || R > D || R % 2 != 0) return CQ_ERR_SHAPE;
    if (!(eps <= 1e30)) return CQ_ERR_ALPHA;
    if (eps < 0.0 && (q_weight != nullptr || k_weight != nullptr)) return CQ_ERR_ALPHA;         // weights belong to the norms
    if (T == 0 || Hq + H == 0) return CQ_OK;
    if ((Hq > 0 && (Q == nullptr || q_out == nullptr)) || (H > 0 && (K == nullptr || k_out == nullptr)) || (R > 0 && (positions == nullptr || freq == nullptr))) return CQ_ERR_NULL;
    for (const void* ptr : {Q, K, static_cast<const void*>(q_out), static_cast<const void*>(k_out), q_weight, k_weight})
        if (!ptr_aligned(ptr, 2)) return CQ_ERR_ALIGN;
    if (!ptr_aligned(positions, 8) || !ptr_aligned(freq, 8)) return CQ_ERR_ALIGN;
    RotateArgs p;
    p.side[0] = RotateSide{static_cast<const uint16_t*>(Q), q_token_stride, q_head_stride, static_cast<uint16_t*>(q_out), qo_token_stride, qo_head_stride,
                           static_cast<const uint16_t*>(q_weight), static_cast<int>(Hq)};
    p.side[1] = RotateSide{static_cast<const uint16_t*>(K), k_token_stride, k_head_stride, static_cast<uint16_t*>(k_out), ko_token_stride, ko_head_stride,
                           static_cast<const uint16_t*>(k_weight), static_cast<int>(H)};
    p.positions = positions; p.freq = freq; p.T = T; p.D = static_cast<int>(D); p.R = static_cast<int>(R);
    p.norm = eps >= 0.0; p.neighbours = neighbours != 0; p.eps = eps; p.slices = p.group = 1;
    bool fast = D % 8 == 0 && D <= kFastDim && R % 16 == 0;
    for (const RotateSide& a : p.side) {
        if (a.heads == 0) continue;
        int64_t strides = 0;
        if (T > 1) strides |= a.xt | a.yt;
        if (a.heads > 1) strides |= a.xh | a.yh;
        fast = fast && strides % 8 == 0 && ptr_aligned(a.x, 16) && ptr_aligned(a.y, 16) && ptr_aligned(a.w, 16);
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == CQ_F16 ? launch_rotate<CQ_F16>(p, fast, st) : launch_rotate<CQ_BF16>(p, fast, st);
}
