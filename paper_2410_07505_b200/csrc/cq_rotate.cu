// Norms of queries and keys for each head, and the rotation by position, in one pass.
//
//   y_d = w_d x_d / sqrt(mean_d x_d^2 + eps)   (y = x without norms),   then for each pair (a, b) of the first R channels
//   (a, b) -> (a cos f - b sin f, a sin f + b cos f),   f = position * freq[pair]
//
// Bound by HBM (2 bytes in, 2 out).  A lane has sixteen channels of a row, both sides of eight pairs, so that a row's mean is a few shuffles
// and the rotation none.  The angles of a token are the same for all of its heads: a block forms those of a few tokens at a time, as
// a fraction of a turn in 64 bits (position * freq passes 2^24 radians, where 32 bits hold no angle), and each lane keeps its
// token's, times the weights: an element then costs two products and the row's factor.  A block's next rows are on the way while these are
// worked on; the issue slots are 59 % busy, the rest waits at the angles' phase of each group of tokens.
// Measured (GPU alone, operands not in L2): 8192 tokens x 72 heads of 128 with norms, bf16 61.5 us (4.9 TB/s of 6.6 of a copy); 777 x 80 of 64 without
// norms 6.8 us; one token 5.5 us.  Rows that begin anywhere, through shared memory: the first 269 us.
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

// 1 / sqrt(mean + eps)
__device__ __noinline__ double wide_factor(double sum, int D, double eps) { return 1.0 / sqrt(sum / D + eps); }

// A lane's channels as the two sides of its pairs: two pieces of eight, or (NEAR) every other one of sixteen.
template <int DT, bool NEAR>
__device__ __forceinline__ void sides(const uint4& x, const uint4& y, float (&a)[8], float (&b)[8]) {
    const uint32_t r[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = unpack16x2<DT>(r[i]);
        if constexpr (NEAR) { a[i] = f.x; b[i] = f.y; }
        else if (i < 4) { a[2 * i] = f.x; a[2 * i + 1] = f.y; }
        else { b[2 * i - 8] = f.x; b[2 * i - 7] = f.y; }
    }
}

// A row whose squares fp32 cannot hold, or are all zero, in 64 bits: a lane's sixteen channels; nothing is written where out is null.
// Called by whole warps.
template <int W, int DT, bool NEAR>
__device__ __noinline__ void wide_row(const uint16_t* w, const float* s_cos, const float* s_sin, uint4 x, uint4 y, int D, double eps,
                                      bool rotated, int da, int db, uint16_t* out) {
    float a[8], b[8], wa[8], wb[8];
    sides<DT, NEAR>(x, y, a, b);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += static_cast<double>(a[i]) * a[i] + static_cast<double>(b[i]) * b[i];
#pragma unroll
    for (int off = W / 2; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off, W);
    if (out == nullptr) return;
    const double f = wide_factor(sum, D, eps);
    uint4 wx = make_uint4(0, 0, 0, 0), wy = wx;
    if (w != nullptr) {
        wx = *reinterpret_cast<const uint4*>(w + da);
        if (db < D) wy = *reinterpret_cast<const uint4*>(w + db);
    }
    sides<DT, NEAR>(wx, wy, wa, wb);
    uint32_t o[8];
    float va[8], vb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double c = rotated ? s_cos[i] : 1.0f, s = rotated ? s_sin[i] : 0.0f;
        const double u = a[i] * f * (w != nullptr ? wa[i] : 1.0f), v = b[i] * f * (w != nullptr ? wb[i] : 1.0f);
        va[i] = static_cast<float>(rotated ? u * c - v * s : u);
        vb[i] = static_cast<float>(rotated ? u * s + v * c : v);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (NEAR) o[i] = pack16x2<DT>(va[i], vb[i]);
        else o[i] = i < 4 ? pack16x2<DT>(va[(2 * i) & 7], va[(2 * i + 1) & 7]) : pack16x2<DT>(vb[(2 * i) & 7], vb[(2 * i + 1) & 7]);
    }
    *reinterpret_cast<uint4*>(out + da) = make_uint4(o[0], o[1], o[2], o[3]);
    if (db < D) *reinterpret_cast<uint4*>(out + db) = make_uint4(o[4], o[5], o[6], o[7]);
}

// W lanes for a row, sixteen channels each; rows in 16-byte accesses, R a multiple of 16.  The block's rows are `group` tokens x
// kRows / group heads at a time.
constexpr int kMaxGroup = 8;
constexpr int kFastDim = 256;
constexpr int kAhead = 2;                                      // rows of a lane in a pass

// NEAR: neighbours are pairs.  With norms two blocks an SM, which spills 4 to 36 bytes: 8192 tokens x 72 heads 61.3 us, 77 with one block and none.
template <int W, int DT, bool NORM, bool NEAR>
__global__ void __launch_bounds__(kRotateThreads, NORM ? 2 : 3)
k24_norm_rotate(const RotateArgs p) {
    constexpr int kRows = kRotateThreads / W;
    __shared__ float s_cos[2][kMaxGroup * kFastDim / 2], s_sin[2][kMaxGroup * kFastDim / 2];
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x % W, row = threadIdx.x / W;
    const int token = row % p.group, first = row / p.group, step = kRows / p.group;
    // the lane's two pieces of eight channels: of a rotated lane both sides of its pairs, else two neighbours of the rest
    const bool rotated = lane < p.R / 16;
    const int da = NEAR || !rotated ? lane * 16 : lane * 8, db = NEAR || !rotated ? lane * 16 + 8 : lane * 8 + p.R / 2;
    const bool have_a = da < p.D, have_b = db < p.D;
    const int slice = blockIdx.x % p.slices;
    const int64_t stride = static_cast<int64_t>(gridDim.x / p.slices) * p.group;
    int buffer = 0;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x / p.slices) * p.group; t0 < p.T; t0 += stride, buffer ^= 1) {
        const int64_t t = t0 + token;
        // this lane's heads of a side: first, first + step .. of those from `from` on; `passes` of kAhead each, of any lane
        int from[2], rows[2], passes[2];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const int64_t heads = p.side[kv].heads;
            from[kv] = static_cast<int>(heads * slice / p.slices);
            const int n = static_cast<int>(heads * (slice + 1) / p.slices) - from[kv];
            rows[kv] = have_a && t < p.T && n > first ? (n - first + step - 1) / step : 0;
            passes[kv] = (n + kAhead * step - 1) / (kAhead * step);
        }
        const int total = passes[0] + passes[1];
        uint4 x[kAhead], y[kAhead];
        auto load = [&](int pass) {                             // the lane's pieces of pass `pass`
            const bool keys = pass >= passes[0];
            const RotateSide& side = p.side[keys ? 1 : 0];
            const int done = (keys ? pass - passes[0] : pass) * kAhead, have = pass < total ? (keys ? rows[1] : rows[0]) - done : 0;
            const uint16_t* at = side.x + t * side.xt + (static_cast<int64_t>(keys ? from[1] : from[0]) + first + static_cast<int64_t>(done) * step) * side.xh;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                x[u] = y[u] = make_uint4(0, 0, 0, 0);
                if (u < have) {
                    x[u] = __ldcs(reinterpret_cast<const uint4*>(at + da));
                    if (have_b) y[u] = __ldcs(reinterpret_cast<const uint4*>(at + db));
                }
                at += step * side.xh;
            }
        };
        load(0);
        angles(p, t0, s_cos[buffer], s_sin[buffer]);            // (behind the first loads)
        __syncthreads();
        float ca[8], cb[8], sa[8], sb[8];                       // a' = a ca - b sb,  b' = b cb + a sa
        for (int pass = 0; pass < total; ++pass) {
            const bool keys = pass >= passes[0];
            const RotateSide& side = p.side[keys ? 1 : 0];
            const int done = (keys ? pass - passes[0] : pass) * kAhead, have = (keys ? rows[1] : rows[0]) - done;
            if (done == 0) {
                uint4 wx = make_uint4(0, 0, 0, 0), wy = wx;
                if (NORM && side.w != nullptr) {
                    if (have_a) wx = *reinterpret_cast<const uint4*>(side.w + da);
                    if (have_b) wy = *reinterpret_cast<const uint4*>(side.w + db);
                }
                sides<DT, NEAR>(wx, wy, ca, cb);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (!NORM || side.w == nullptr) ca[i] = cb[i] = 1.0f;
                    const int at = token * (p.R / 2) + lane * 8 + i;
                    const float c = rotated ? s_cos[buffer][at] : 1.0f, s = rotated ? s_sin[buffer][at] : 0.0f;
                    sa[i] = s * ca[i];
                    sb[i] = s * cb[i];
                    ca[i] *= c;
                    cb[i] *= c;
                }
            }
            uint4 xn[kAhead], yn[kAhead];                       // this pass's: the next one's are on the way meanwhile
#pragma unroll
            for (int u = 0; u < kAhead; ++u) { xn[u] = x[u]; yn[u] = y[u]; }
            load(pass + 1);
            float f[kAhead];
            uint32_t wide = 0;                                  // rows of these that want 64 bits
            if constexpr (NORM) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    float a[8], b[8];
                    sides<DT, NEAR>(xn[u], yn[u], a, b);
                    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) { s0 = __fmaf_rn(a[i], a[i], s0); s1 = __fmaf_rn(b[i], b[i], s1); }
                    f[u] = s0 + s1;
                }
#pragma unroll
                for (int off = W / 2; off > 0; off >>= 1)
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) f[u] += __shfl_xor_sync(0xFFFFFFFFu, f[u], off, W);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (u < have && !(f[u] > 1e-25f && f[u] < 1e35f)) wide |= 1u << u;
                    f[u] = rsqrtf(__fmaf_rn(f[u], 1.0f / static_cast<float>(p.D), static_cast<float>(p.eps)));
                }
            }
            uint16_t* out = side.y + t * side.yt + (static_cast<int64_t>(keys ? from[1] : from[0]) + first + static_cast<int64_t>(done) * step) * side.yh;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float a[8], b[8];
                sides<DT, NEAR>(xn[u], yn[u], a, b);
                if constexpr (NORM) {                           // (first: an element times its weight may leave fp32's range, its norm times that does not)
#pragma unroll
                    for (int i = 0; i < 8; ++i) { a[i] *= f[u]; b[i] *= f[u]; }
                }
                if (rotated) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v = __fmaf_rn(a[i], ca[i], -(b[i] * sb[i]));
                        b[i] = __fmaf_rn(b[i], cb[i], a[i] * sa[i]);
                        a[i] = v;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) { a[i] *= ca[i]; b[i] *= cb[i]; }
                }
                uint32_t o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (NEAR) o[i] = pack16x2<DT>(a[i], b[i]);
                    else o[i] = i < 4 ? pack16x2<DT>(a[(2 * i) & 7], a[(2 * i + 1) & 7]) : pack16x2<DT>(b[(2 * i) & 7], b[(2 * i + 1) & 7]);
                }
                if (u < have && !(NORM && (wide >> u & 1u))) {
                    *reinterpret_cast<uint4*>(out + u * step * side.yh + da) = make_uint4(o[0], o[1], o[2], o[3]);
                    if (have_b) *reinterpret_cast<uint4*>(out + u * step * side.yh + db) = make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
            if (NORM && __any_sync(0xFFFFFFFFu, wide != 0u)) {
                const int at = rotated ? token * (p.R / 2) + lane * 8 : 0;
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    wide_row<W, DT, NEAR>(side.w, s_cos[buffer] + at, s_sin[buffer] + at, xn[u], yn[u], p.D, p.eps, rotated, da, db,
                                          wide >> u & 1u ? out + u * step * side.yh : nullptr);
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
    const int W = p.D <= 64 ? 4 : p.D <= 128 ? 8 : 16;
    const int rows = fast ? kRotateThreads / W : kRotateThreads / 32;
    const int heads = std::max(p.side[0].heads, p.side[1].heads);
    // Persistent blocks (where a warp has a row, eight times as many: 8192 tokens 269 us, 351).  As many tokens at a time as leave an SM one group
    // of them (two without norms, whose groups take less): 500 tokens x 72 heads of 128 with norms 8.1 us, two groups 11.9; 777 x 80 of 64 without
    // norms 6.7, one group 7.7.  Few tokens: a token's heads are shared out, a pass or more to a block, while all blocks are resident.
    const int64_t resident = (!fast ? 6 : p.norm ? 2 : 3) * sm_count();
    p.group = 1;
    while (fast && p.group < kMaxGroup && p.T / (2 * p.group) >= (p.norm ? 1 : 2) * sm_count()) p.group *= 2;
    const int64_t groups = (p.T + p.group - 1) / p.group;
    const int64_t most = std::max(1, (heads + rows - 1) / rows / (fast ? kAhead : 1));
    p.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, resident / groups)));
    const int64_t blocks = std::min<int64_t>(groups, (fast ? resident : 8 * resident) / p.slices);
    const dim3 grid(static_cast<unsigned>(blocks * p.slices));
    if (!fast) return launch_ex(k24_norm_rotate_any<DT>, grid, kRotateThreads, 0, st, 1, !tuning_no_pdl(), p);
    if (W == 4) return launch_rotate_rows<4, DT>(p, grid, st);
    if (W == 8) return launch_rotate_rows<8, DT>(p, grid, st);
    return launch_rotate_rows<16, DT>(p, grid, st);
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
