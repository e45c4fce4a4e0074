// Low-rank adapters of many requests beside a shared projection:
//
//   out[t] = y[t] + scale_a B_a (A_a x[t]),   a = index[t]   (outside 0 .. n - 1: out[t] = y[t])
//
// Two kernels.  The first forms h[t] = A_a x[t] (R numbers a token), the second adds B_a h[t].  Both are bound by what they read: x and the
// adapters in use, then y.  Tokens are taken in windows of 64 neighbours; inside a window those of one adapter go together, so a
// matrix is read once for all of them whatever the order of the batch, and no sort comes before.  mma.sync feeds on fragments
// that come from memory directly, in 16-byte (8-byte) pieces of rows: which element of the contraction stands where does not matter as
// long as both operands agree, so a lane's piece fills its places of two (one) products.
//
// h is fp32 until it is written: as two 16-bit halves (h 2^-e = high + low, e from the token's largest |h|), so that the second
// product, on 16-bit operands, sees 16 bits of it or more, and fp16 neither overflows nor loses small tokens.
#include "cq_serve.cuh"

#include <algorithm>

namespace cq {

constexpr int kWindow = 64;                   // tokens that are sorted by adapter together
constexpr int kAdThreads = 256;
constexpr int kUnitK = 32;                    // contraction of one step: a 16-byte piece for each of the four lanes of a row
constexpr int kExpandCols = 256;              // columns of a block of the second kernel, 32 for each warp
constexpr int kMaxRank = 128;

struct AdapterArgs {
    const uint16_t* x; int64_t ldx;
    const void* y; int64_t ldy;
    void* out; int64_t ldo;
    const uint16_t* A; const uint16_t* B; const float* scale;
    const int* index;
    uint16_t* high; uint16_t* low; float* factor;               // [T][R], [T][R], [T]
    int64_t T, K, N;
    int R, n;
    bool vec_k, vec_n;                                          // rows of x and A (y and out) in 16-byte accesses
};

// The window's tokens by adapter.  s_rank[i]: how many adapters appear before the one that token i is the first of; -1 if it is not.
struct Window {
    int idx[kWindow];
    int first[kWindow];                       // adapters in order of appearance: their first token
    int list[kWindow];                        // tokens of the adapter at hand
    int n, count, none;
};
__device__ __forceinline__ void read_window(const AdapterArgs& p, int64_t t0, Window& w) {
    const int tid = threadIdx.x;
    if (tid < kWindow) {
        const int64_t t = t0 + tid;
        const int a = t < p.T ? __ldcg(p.index + t) : -1;
        w.idx[tid] = a >= 0 && a < p.n ? a : -1;
    }
    __syncthreads();
    if (tid < kWindow) {
        const int a = w.idx[tid];
        bool earlier = false;
#pragma unroll 8
        for (int j = 0; j < kWindow; ++j) earlier = earlier || (j < tid && w.idx[j] == a);
        const unsigned lead = __ballot_sync(0xFFFFFFFFu, a >= 0 && !earlier);
        if ((tid & 31) == 0) w.list[tid >> 5] = static_cast<int>(lead);
    }
    __syncthreads();
    if (tid < kWindow) {
        const unsigned lo = static_cast<unsigned>(w.list[0]), hi = static_cast<unsigned>(w.list[1]);
        const unsigned mine = tid < 32 ? lo : hi;
        const int before = __popc(mine & ((1u << (tid & 31)) - 1u)) + (tid < 32 ? 0 : __popc(lo));
        if (mine >> (tid & 31) & 1u) w.first[before] = tid;
        if (tid == 0) w.n = __popc(lo) + __popc(hi);
    }
    __syncthreads();
}
// The tokens of adapter `a` in order (a = -1: those without one).
__device__ __forceinline__ void pick_tokens(Window& w, int a, int valid) {
    __syncthreads();
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        const unsigned lo = __ballot_sync(0xFFFFFFFFu, lane < valid && w.idx[lane] == a);
        const unsigned hi = __ballot_sync(0xFFFFFFFFu, 32 + lane < valid && w.idx[32 + lane] == a);
        const unsigned below = (1u << lane) - 1u;
        if (lo >> lane & 1u) w.list[__popc(lo & below)] = lane;
        if (hi >> lane & 1u) w.list[__popc(lo) + __popc(hi & below)] = 32 + lane;
        if (lane == 0) w.count = __popc(lo) + __popc(hi);
    }
    __syncthreads();
}

template <int DT>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3, const uint32_t b0, const uint32_t b1) {
    if constexpr (DT == CQ_BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// eight elements of a row from column k on, zeros from column `end` on
template <bool VEC>
__device__ __forceinline__ uint4 piece8(const uint16_t* row, int64_t k, int64_t end) {
    if constexpr (VEC) {
        return k < end ? __ldcg(reinterpret_cast<const uint4*>(row + k)) : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = k + 2 * i < end ? __ldcg(row + k + 2 * i) : 0, hi = k + 2 * i + 1 < end ? __ldcg(row + k + 2 * i + 1) : 0;
            v[i] = lo | hi << 16;
        }
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
}

__device__ __forceinline__ float ld_rank(const float* p, uint32_t rank) {
    uint32_t remote;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- h = A x ----------------------------------------------------------------------------------------------------
// grid (parts of the contraction = cluster, windows, adapters of a window in turn).  Up to 32 tokens: all eight warps split the part;
// more: four warps for either half of them.  Sums of warps meet in shared memory in a fixed tree, those of the cluster's blocks through
// distributed shared memory in rank order: equal calls give equal bits.
template <int MT>                             // MT x 16 rows of A
constexpr size_t shrink_smem() { return size_t(4) * MT * 16 * 33 * 4 + size_t(kWindow) * (MT * 16 + 1) * 4; }

template <int MT, int DT, bool VEC>
__global__ void __launch_bounds__(kAdThreads, MT <= 4 ? 2 : 1)
k25_adapter_in(const AdapterArgs p) {
    constexpr int kRows = MT * 16;
    extern __shared__ float s_mem[];
    float* s_red = s_mem;                                       // [4][kRows][33]
    float* s_h = s_mem + 4 * kRows * 33;                        // [token][kRows + 1]
    __shared__ Window w;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");         // (only now: the next kernel reads B and y before this one ends)
    const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kWindow;
    const int valid = static_cast<int>(min(static_cast<int64_t>(kWindow), p.T - t0));
    read_window(p, t0, w);
    const int rank = blockIdx.x, ranks = gridDim.x;
    const int64_t units = (p.K + kUnitK - 1) / kUnitK, u0 = units * rank / ranks, u1 = units * (rank + 1) / ranks;
    for (int which = blockIdx.z; which < w.n; which += gridDim.z) {
        const int a = w.idx[w.first[which]];
        pick_tokens(w, a, valid);
        const int count = w.count;
        const bool halves = count > 32;
        const int first = halves ? (warp >> 2) * 32 : 0, split = halves ? 4 : 8, part = halves ? warp & 3 : warp;
        const int groups = min(4, (count - first + 7) / 8);
        const uint16_t* A = p.A + static_cast<int64_t>(a) * p.R * p.K;
        const uint16_t* rows[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = first + j * 8 + g;
            rows[j] = m < count ? p.x + (t0 + w.list[m]) * p.ldx : nullptr;
        }
        float acc[MT][4][4] = {};
        for (int64_t u = u0 + part; u < u1; u += split) {
            const int64_t k = u * kUnitK + t4 * 8;
            uint4 xb[4], wa[MT][2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xb[j] = make_uint4(0, 0, 0, 0);
                if (rows[j] != nullptr) xb[j] = piece8<VEC>(rows[j], k, p.K);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const int r = i * 16 + hh * 8 + g;
                    wa[i][hh] = make_uint4(0, 0, 0, 0);
                    if (r < p.R) wa[i][hh] = piece8<VEC>(A + r * p.K, k, p.K);
                }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j >= groups) break;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    mma16<DT>(acc[i][j], wa[i][0].x, wa[i][1].x, wa[i][0].y, wa[i][1].y, xb[j].x, xb[j].y);
                    mma16<DT>(acc[i][j], wa[i][0].z, wa[i][1].z, wa[i][0].w, wa[i][1].w, xb[j].z, xb[j].w);
                }
            }
        }
        // acc[i][j]: rows i * 16 + g (+ 8), tokens j * 8 + 2 t4 (+ 1) of this warp's 32
        for (int step = split / 2; step > 0; step >>= 1) {
            const int slot = halves ? (warp >> 2) * 2 + (part % step) : part % step;      // (at most two for either half, four without)
            float* buf = s_red + slot * kRows * 33;
            if (part >= step && part < 2 * step) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) buf[(i * 16 + g + (e >> 1) * 8) * 33 + j * 8 + 2 * t4 + (e & 1)] = acc[i][j][e];
            }
            __syncthreads();
            if (part < step) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] += buf[(i * 16 + g + (e >> 1) * 8) * 33 + j * 8 + 2 * t4 + (e & 1)];
            }
            __syncthreads();
        }
        if (part == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s_h[(first + j * 8 + 2 * t4 + (e & 1)) * (kRows + 1) + i * 16 + g + (e >> 1) * 8] = acc[i][j][e];
        }
        __syncthreads();
        if (ranks > 1) cluster_barrier();
        // a warp for each token of this block's share
        for (int m = rank + warp * ranks; m < count; m += ranks * (kAdThreads / 32)) {
            constexpr int kPer = (kRows + 31) / 32;
            float h[kPer], top = 0.0f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = lane + 32 * i;
                h[i] = 0.0f;
                if (r < p.R)
                    for (int k = 0; k < ranks; ++k) h[i] += ranks > 1 ? ld_rank(s_h + m * (kRows + 1) + r, k) : s_h[m * (kRows + 1) + r];
                const float v = fabsf(h[i]);
                top = fmaxf(top, v < INFINITY ? v : 0.0f);
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
            // 2^e, the power of two at or below the largest (e of 0 has the range of fp32's normal numbers): h 2^-e lies below 2
            const uint32_t e = min(max(__float_as_uint(top) >> 23, 2u), 252u);
            const float down = __uint_as_float((254u - e) << 23);
            const int64_t t = t0 + w.list[m];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = lane + 32 * i;
                if (r < p.R) {
                    const float v = h[i] * down;
                    const uint16_t hi = pack16<DT>(v);
                    p.high[t * p.R + r] = hi;
                    p.low[t * p.R + r] = fabsf(v) < INFINITY ? pack16<DT>(v - cvt16<DT>(hi)) : 0;
                }
            }
            if (lane == 0) p.factor[t] = __uint_as_float(e << 23) * (p.scale != nullptr ? p.scale[a] : 1.0f);
        }
        if (ranks > 1) cluster_barrier();     // nobody writes its sums over while they are being read
    }
}

// ---- out = y + B h ---------------------------------------------------------------------------------------------------
// grid (blocks of 256 columns, windows, adapters of a window in turn).  A warp keeps its 32 columns of B_a in registers and takes the adapter's
// tokens 16 at a time.  The four products of 8 columns share them out so that each lane ends up with 8 neighbouring columns.
template <int YT>
__device__ __forceinline__ void add_store8(const AdapterArgs& p, int64_t t, int64_t col, const float (&d)[8], float f) {
    if (col >= p.N) return;
    constexpr int kElem = YT == CQ_F32 ? 4 : 2;
    const uint8_t* y = static_cast<const uint8_t*>(p.y) + (t * p.ldy + col) * kElem;
    uint8_t* out = static_cast<uint8_t*>(p.out) + (t * p.ldo + col) * kElem;
    if (p.vec_n) {
        if constexpr (YT == CQ_F32) {
            float4 a = __ldcg(reinterpret_cast<const float4*>(y)), b = __ldcg(reinterpret_cast<const float4*>(y) + 1);
            a.x = __fmaf_rn(d[0], f, a.x); a.y = __fmaf_rn(d[1], f, a.y); a.z = __fmaf_rn(d[2], f, a.z); a.w = __fmaf_rn(d[3], f, a.w);
            b.x = __fmaf_rn(d[4], f, b.x); b.y = __fmaf_rn(d[5], f, b.y); b.z = __fmaf_rn(d[6], f, b.z); b.w = __fmaf_rn(d[7], f, b.w);
            reinterpret_cast<float4*>(out)[0] = a;
            reinterpret_cast<float4*>(out)[1] = b;
        } else {
            const uint4 w = __ldcg(reinterpret_cast<const uint4*>(y));
            const uint32_t r[4] = {w.x, w.y, w.z, w.w};
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = unpack16x2<YT>(r[i]);
                o[i] = pack16x2<YT>(__fmaf_rn(d[2 * i], f, v.x), __fmaf_rn(d[2 * i + 1], f, v.y));
            }
            *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    } else {
        const int64_t n = min(int64_t(8), p.N - col);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) {
                if constexpr (YT == CQ_F32) reinterpret_cast<float*>(out)[i] = __fmaf_rn(d[i], f, __ldcg(reinterpret_cast<const float*>(y) + i));
                else reinterpret_cast<uint16_t*>(out)[i] = pack16<YT>(__fmaf_rn(d[i], f, cvt16<YT>(__ldcg(reinterpret_cast<const uint16_t*>(y) + i))));
            }
    }
}

template <int MT, int DT, int YT>
__global__ void __launch_bounds__(kAdThreads)
k26_adapter_out(const AdapterArgs p) {
    __shared__ Window w;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;");
    const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kWindow;
    const int valid = static_cast<int>(min(static_cast<int64_t>(kWindow), p.T - t0));
    read_window(p, t0, w);
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kExpandCols + warp * 32;
    bool waited = false;
    for (int which = blockIdx.z; which < w.n; which += gridDim.z) {
        const int a = w.idx[w.first[which]];
        pick_tokens(w, a, valid);
        const int count = w.count;
        // product j takes columns n0 + 8 (q / 2) + 2 j + q % 2, q = 0 .. 7
        uint2 b[4][MT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + 8 * (g >> 1) + 2 * j + (g & 1);
            const uint16_t* row = p.B + (static_cast<int64_t>(a) * p.N + n) * p.R;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int k = i * 16 + t4 * 4;
                b[j][i] = make_uint2(0, 0);
                if (n < p.N && k < p.R) b[j][i] = __ldcg(reinterpret_cast<const uint2*>(row + k));
            }
        }
        if (!waited) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            waited = true;
        }
        for (int m0 = 0; m0 < count; m0 += 16) {
            const int64_t ta = m0 + g < count ? t0 + w.list[m0 + g] : -1, tb = m0 + 8 + g < count ? t0 + w.list[m0 + 8 + g] : -1;
            float acc[4][4] = {};
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int k = i * 16 + t4 * 4;
                if (i * 16 >= p.R) break;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const uint16_t* h = part == 0 ? p.high : p.low;
                    uint2 ha = make_uint2(0, 0), hb = ha;
                    if (ta >= 0 && k < p.R) ha = __ldcg(reinterpret_cast<const uint2*>(h + ta * p.R + k));
                    if (tb >= 0 && k < p.R) hb = __ldcg(reinterpret_cast<const uint2*>(h + tb * p.R + k));
#pragma unroll
                    for (int j = 0; j < 4; ++j) mma16<DT>(acc[j], ha.x, hb.x, ha.y, hb.y, b[j][i].x, b[j][i].y);
                }
            }
            const int64_t col = n0 + 8 * t4;
            if (ta >= 0) {
                const float d[8] = {acc[0][0], acc[0][1], acc[1][0], acc[1][1], acc[2][0], acc[2][1], acc[3][0], acc[3][1]};
                add_store8<YT>(p, ta, col, d, __ldcg(p.factor + ta));
            }
            if (tb >= 0) {
                const float d[8] = {acc[0][2], acc[0][3], acc[1][2], acc[1][3], acc[2][2], acc[2][3], acc[3][2], acc[3][3]};
                add_store8<YT>(p, tb, col, d, __ldcg(p.factor + tb));
            }
        }
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (blockIdx.z == 0 && p.out != p.y) {    // tokens without an adapter
        pick_tokens(w, -1, valid);
        const float zero[8] = {-0.0f, -0.0f, -0.0f, -0.0f, -0.0f, -0.0f, -0.0f, -0.0f};       // (y + -0 is y)
        for (int i = threadIdx.x; i < w.count * (kExpandCols / 8); i += kAdThreads)
            add_store8<YT>(p, t0 + w.list[i / (kExpandCols / 8)], static_cast<int64_t>(blockIdx.x) * kExpandCols + (i % (kExpandCols / 8)) * 8, zero, 0.0f);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
static size_t up256(size_t v) { return (v + 255) / 256 * 256; }
static size_t adapter_workspace(int64_t T, int64_t R) { return 2 * up256(sizeof(uint16_t) * T * R) + up256(sizeof(float) * T); }

template <int MT, int DT, bool VEC>
static int launch_in(const AdapterArgs& p, dim3 grid, cudaStream_t st) {
    static thread_local LaunchMemo memo;
    // (the static shared memory counts towards the 48 KB that need no leave)
    constexpr size_t smem = shrink_smem<MT>(), limit = smem > 47 * 1024 ? smem : 0;
    if (resident_ctas(k25_adapter_in<MT, DT, VEC>, kAdThreads, smem, limit, memo) < 1) return CQ_ERR_CUDA;
    return launch_ex(k25_adapter_in<MT, DT, VEC>, grid, kAdThreads, smem, st, grid.x, !tuning_no_pdl(), p);
}

template <int MT, int DT>
static int launch_adapter(const AdapterArgs& p, int y_dtype, cudaStream_t st) {
    const int sms = sm_count();
    const int64_t windows = (p.T + kWindow - 1) / kWindow;
    const int64_t adapters = std::min<int64_t>(kWindow, std::min<int64_t>(p.n, p.T));
    if (windows > 65535) return CQ_ERR_SHAPE;
    // parts of the contraction of 512 or more, up to a portable cluster; a block for each adapter of a window while they all fit
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(8, p.K / 512));
    const int64_t slots = std::max<int64_t>(1, std::min<int64_t>(adapters, 4 * sms / (windows * parts)));
    const dim3 grid(static_cast<unsigned>(parts), static_cast<unsigned>(windows), static_cast<unsigned>(slots));
    const int rc = p.vec_k ? launch_in<MT, DT, true>(p, grid, st) : launch_in<MT, DT, false>(p, grid, st);
    if (rc != CQ_OK) return rc;
    const int64_t cols = (p.N + kExpandCols - 1) / kExpandCols;
    const int64_t turns = std::max<int64_t>(1, std::min<int64_t>(adapters, 16 * sms / (windows * cols)));
    const dim3 grid2(static_cast<unsigned>(cols), static_cast<unsigned>(windows), static_cast<unsigned>(turns));
    if (y_dtype == CQ_F32) return launch_ex(k26_adapter_out<MT, DT, CQ_F32>, grid2, kAdThreads, 0, st, 1, !tuning_no_pdl(), p);
    if (y_dtype == CQ_F16) return launch_ex(k26_adapter_out<MT, DT, CQ_F16>, grid2, kAdThreads, 0, st, 1, !tuning_no_pdl(), p);
    return launch_ex(k26_adapter_out<MT, DT, CQ_BF16>, grid2, kAdThreads, 0, st, 1, !tuning_no_pdl(), p);
}

template <int DT>
static int launch_adapter_rank(const AdapterArgs& p, int y_dtype, cudaStream_t st) {
    if (p.R <= 16) return launch_adapter<1, DT>(p, y_dtype, st);
    if (p.R <= 32) return launch_adapter<2, DT>(p, y_dtype, st);
    if (p.R <= 64) return launch_adapter<4, DT>(p, y_dtype, st);
    return launch_adapter<8, DT>(p, y_dtype, st);
}

}  // namespace cq

extern "C" {

size_t cq_adapter_add_workspace_bytes(int64_t T, int64_t R) { return T < 0 || R < 1 || R > cq::kMaxRank ? 0 : cq::adapter_workspace(T, R); }

int cq_adapter_add(const void* X, int dtype, int64_t T, int64_t K, int64_t ldx, const void* A, const void* B, const float* scale, int64_t n,
                   int64_t R, int64_t N, const int* index, const void* y, int y_dtype, int64_t ldy, void* out, int64_t ldo,
                   void* workspace, size_t workspace_bytes, void* stream) {
    using namespace cq;
    if (T < 0 || K < 0 || N < 0 || n < 0 || ldx < K || ldy < N || ldo < N || R < 8 || R > kMaxRank || R % 8 != 0) return CQ_ERR_SHAPE;
    if (T > 65535 * kWindow || K > (int64_t(1) << 31) - 1024 || N > (int64_t(1) << 31) - 1024 || n > (int64_t(1) << 31) - 1024) return CQ_ERR_SHAPE;
    if (dtype != CQ_F16 && dtype != CQ_BF16) return CQ_ERR_DTYPE;
    if (y_dtype != CQ_F16 && y_dtype != CQ_BF16 && y_dtype != CQ_F32) return CQ_ERR_DTYPE;
    if (T == 0 || N == 0) return CQ_OK;
    if (y == nullptr || out == nullptr || index == nullptr || (K > 0 && X == nullptr) || (n > 0 && ((K > 0 && A == nullptr) || B == nullptr))) return CQ_ERR_NULL;
    const size_t elem = y_dtype == CQ_F32 ? 4 : 2;
    if (!ptr_aligned(X, 2) || !ptr_aligned(A, 2) || !ptr_aligned(B, 16) || !ptr_aligned(scale, 4) || !ptr_aligned(index, 4) || !ptr_aligned(y, elem) || !ptr_aligned(out, elem)) return CQ_ERR_ALIGN;
    if (workspace == nullptr || !ptr_aligned(workspace, 256) || workspace_bytes < adapter_workspace(T, R)) return CQ_ERR_WORKSPACE;
    AdapterArgs p;
    p.x = static_cast<const uint16_t*>(X); p.ldx = ldx; p.y = y; p.ldy = ldy; p.out = out; p.ldo = ldo;
    p.A = static_cast<const uint16_t*>(A); p.B = static_cast<const uint16_t*>(B); p.scale = scale; p.index = index;
    p.high = static_cast<uint16_t*>(workspace);
    p.low = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(workspace) + up256(sizeof(uint16_t) * T * R));
    p.factor = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 2 * up256(sizeof(uint16_t) * T * R));
    p.T = T; p.K = K; p.N = N; p.R = static_cast<int>(R); p.n = static_cast<int>(n);
    p.vec_k = K % 8 == 0 && (T == 1 || ldx % 8 == 0) && ptr_aligned(X, 16) && ptr_aligned(A, 16);
    p.vec_n = N % 8 == 0 && (T == 1 || (ldy % 8 == 0 && ldo % 8 == 0)) && ptr_aligned(y, 16) && ptr_aligned(out, 16);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == CQ_F16 ? launch_adapter_rank<CQ_F16>(p, y_dtype, st) : launch_adapter_rank<CQ_BF16>(p, y_dtype, st);
}

}  // extern "C"
