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
// Measured (GPU alone, operands not in L2), rank 16: one token x 4096 x 6144 7.2 and then 9.1 us for both; 64 tokens on 57 adapters x 8192 x 8192 14.4 and
// 20.6 us, 33 MB.  What bounds them is latency: the index, the first pieces, the cluster's join, then h.  777 x 2060, rows on 8 bytes:
// 12.5 us.
//
// h is fp32 until it is written: as two 16-bit halves (h 2^-e = high + low, e from the token's largest |h|), so that the second
// product, on 16-bit operands, sees 16 bits of it or more, and fp16 neither overflows nor loses small tokens.
#include "cq_adapter.cuh"

#include <algorithm>
#include <type_traits>

namespace cq {

constexpr int kWindow = 64;                   // tokens that are sorted by adapter together
constexpr int kAdThreads = 256;
constexpr int kUnitK = 32;                    // contraction of one step: a 16-byte piece for each of the four lanes of a row

// A window's adapters, two tokens to a lane of every warp (-1: none), and the tokens of one of them in order, in shared memory.
struct Window {
    int lo, hi;
    __device__ __forceinline__ void read(const AdapterArgs& p, int64_t t0) {
        const int lane = threadIdx.x & 31;
        lo = t0 + lane < p.T ? __ldcg(p.index + t0 + lane) : -1;
        hi = t0 + 32 + lane < p.T ? __ldcg(p.index + t0 + 32 + lane) : -1;
        if (lo >= p.n) lo = -1;
        if (hi >= p.n) hi = -1;
    }
    __device__ __forceinline__ uint64_t any() const {                   // tokens with an adapter
        return __ballot_sync(0xFFFFFFFFu, lo >= 0) | static_cast<uint64_t>(__ballot_sync(0xFFFFFFFFu, hi >= 0)) << 32;
    }
    __device__ __forceinline__ int at(int token) const { return __shfl_sync(0xFFFFFFFFu, token < 32 ? lo : hi, token & 31); }
    __device__ __forceinline__ uint64_t with(int a) const {             // tokens of adapter a
        return __ballot_sync(0xFFFFFFFFu, lo == a) | static_cast<uint64_t>(__ballot_sync(0xFFFFFFFFu, hi == a)) << 32;
    }
};
// The adapters of a window that the slot-th of `slots` blocks takes, in order of their first tokens.
struct Turn {
    uint64_t left;
    int rank;
    bool alone;                               // a block for each token: this one's, if no earlier token has the same adapter
    __device__ __forceinline__ Turn(const Window& w, int slots) : left(w.any()), rank(0), alone(slots >= kWindow) {}
    // the next adapter and its tokens; false when there is none
    __device__ __forceinline__ bool next(const Window& w, int slot, int slots, int& a, uint64_t& tokens) {
        if (alone) {
            if (!(left >> slot & 1u)) return false;
            a = w.at(slot);
            tokens = w.with(a);
            left = 0;
            return __ffsll(tokens) - 1 == slot;
        }
        while (left != 0) {
            a = w.at(__ffsll(left) - 1);
            tokens = w.with(a);
            left &= ~tokens;
            if (rank++ % slots == slot) return true;
        }
        return false;
    }
};
// The tokens of a set in order, written by one warp.
__device__ __forceinline__ void write_list(uint64_t tokens, uint8_t* list) {
    const int lane = threadIdx.x & 31;
    const uint32_t lo = static_cast<uint32_t>(tokens), hi = static_cast<uint32_t>(tokens >> 32), below = (1u << lane) - 1u;
    if (lo >> lane & 1u) list[__popc(lo & below)] = static_cast<uint8_t>(lane);
    if (hi >> lane & 1u) list[__popc(lo) + __popc(hi & below)] = static_cast<uint8_t>(32 + lane);
    __syncwarp();
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

// eight elements of a row from column k on (a multiple of 8), zeros from column `end` on; `vec` elements at a time, all of which
// lie before `end` or none
__device__ __forceinline__ uint4 piece8(const uint16_t* row, int64_t k, int64_t end, int vec) {
    if (vec == 8) return k < end ? __ldcg(reinterpret_cast<const uint4*>(row + k)) : make_uint4(0, 0, 0, 0);
    uint32_t v[4];
    if (vec >= 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = k + 2 * i < end ? __ldcg(reinterpret_cast<const uint32_t*>(row + k) + i) : 0;
    } else {
        // aligned words that hold an element of the piece, moved by half a word where the row begins in the middle of one
        const uint16_t* at = row + k;
        const bool odd = (reinterpret_cast<uintptr_t>(at) & 2u) != 0u;
        const uint32_t* words = reinterpret_cast<const uint32_t*>(at - (odd ? 1 : 0));
        const int n = static_cast<int>(min(max(end - k, int64_t(0)), int64_t(8)));                    // elements there are
        uint32_t r[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) r[i] = n > 0 && 2 * i < n + (odd ? 1 : 0) ? __ldcg(words + i) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = odd ? __funnelshift_r(r[i], r[i + 1], 16) : r[i];
            if (2 * i + 1 >= n) v[i] = 2 * i >= n ? 0 : v[i] & 0xFFFFu;
        }
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}
// the same into shared memory, asynchronously; vec of 2 or more
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool have) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" :: "r"(dst), "l"(src), "n"(BYTES), "r"(have ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void stage8(uint8_t* dst, const uint16_t* row, int64_t k, int64_t end, int vec) {
    const uint32_t at = smem_u32(dst);
    if (vec == 8) {
        copy_async<16>(at, k < end ? row + k : row, k < end);
    } else if (vec == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) copy_async<8>(at + 8 * i, k + 4 * i < end ? row + k + 4 * i : row, k + 4 * i < end);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) copy_async<4>(at + 4 * i, k + 2 * i < end ? row + k + 2 * i : row, k + 2 * i < end);
    }
}
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], const uint8_t* p) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_u32(p)) : "memory");
}

// ---- h = A x ----------------------------------------------------------------------------------------------------
// grid (parts of the contraction = cluster, windows, adapters of a window in turn).  Up to eight tokens of an adapter: fragments straight
// from memory, the eight warps split the part (64 x 8192 x 8192 above 14.4 us, 26.5 through shared memory; one token 7.2, 9.1).  More: tiles of x and A of 64 along the contraction through shared memory, a ring of asynchronous
// copies ahead.  Sums of warps meet in shared memory, those of the cluster's blocks through distributed shared memory in rank order: equal
// calls give equal bits.
constexpr int kUnit = 64;                     // contraction of one stage
template <int MT> __host__ __device__ constexpr int shrink_stages() { return MT <= 2 ? 6 : MT == 4 ? 5 : 3; }
constexpr int kRowBytes = 144;                // of a stage where rows of x and A begin anywhere; 128 where they do not
template <int MT> __host__ __device__ constexpr size_t shrink_stage() { return size_t(kWindow + MT * 16) * kRowBytes; }
template <int MT> __host__ __device__ constexpr size_t shrink_smem() { return shrink_stages<MT>() * shrink_stage<MT>() + size_t(kWindow) * (MT * 16 + 1) * 4; }

template <int MT, int DT>                     // MT x 16 rows of A
__global__ void __launch_bounds__(kAdThreads, 2)
k25_adapter_in(const AdapterArgs p) {
    constexpr int kRows = MT * 16, ST = shrink_stages<MT>();
    constexpr size_t kStage = shrink_stage<MT>();
    extern __shared__ __align__(128) uint8_t s_mem[];
    float* s_red = reinterpret_cast<float*>(s_mem);             // [4][kRows][9], over the stages
    float* s_h = reinterpret_cast<float*>(s_mem + ST * kStage); // [token][kRows + 1]
    static_assert(size_t(4) * kRows * 9 * 4 <= ST * kStage, "sums of warps");
    __shared__ uint8_t s_list[kAdThreads / 32][kWindow];
    __shared__ TileSort s_sort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    uint8_t* list = s_list[warp];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");         // (only now: the next kernel reads B and y before this one ends)
    const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kWindow;
    if (p.tiles && blockIdx.x == 0 && blockIdx.z == 0 && t0 % kTileTokens == 0) sort_tile(p, t0, s_sort, true);
    Window w;
    w.read(p, t0);
    const int rank = blockIdx.x, ranks = gridDim.x;
    const int64_t units = (p.K + kUnit - 1) / kUnit, u0 = units * rank / ranks, u1 = units * (rank + 1) / ranks;
    Turn turn(w, gridDim.z);
    int a;
    uint64_t tokens;
    while (turn.next(w, blockIdx.z, gridDim.z, a, tokens)) {
        write_list(tokens, list);
        const int count = __popcll(tokens);
        const uint16_t* A = p.A + static_cast<int64_t>(a) * p.R * p.K;
        if (count <= 8) {
            constexpr int kAhead = MT == 1 ? 4 : MT == 2 ? 2 : 1;       // steps whose loads are issued together
            const uint16_t* x = g < count ? p.x + (t0 + list[g]) * p.ldx : nullptr;
            float acc[MT][4] = {};
            for (int64_t u = 2 * u0 + warp; u < 2 * u1; u += 8 * kAhead) {
                uint4 xb[kAhead], wa[kAhead][MT][2];
#pragma unroll
                for (int s = 0; s < kAhead; ++s) {
                    const int64_t k = u + 8 * s < 2 * u1 ? (u + 8 * s) * kUnitK + t4 * 8 : p.K + 8;      // (nothing: zeros)
                    xb[s] = x != nullptr ? piece8(x, k, p.K, p.vec_k) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            const int r = i * 16 + hh * 8 + g;
                            wa[s][i][hh] = r < p.R ? piece8(A + r * p.K, k, p.K, p.vec_k) : make_uint4(0, 0, 0, 0);
                        }
                }
#pragma unroll
                for (int s = 0; s < kAhead; ++s)
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        mma16<DT>(acc[i], wa[s][i][0].x, wa[s][i][1].x, wa[s][i][0].y, wa[s][i][1].y, xb[s].x, xb[s].y);
                        mma16<DT>(acc[i], wa[s][i][0].z, wa[s][i][1].z, wa[s][i][0].w, wa[s][i][1].w, xb[s].z, xb[s].w);
                    }
            }
            // acc[i]: rows i * 16 + g (+ 8), tokens 2 t4 (+ 1)
            for (int step = 4; step > 0; step >>= 1) {
                float* buf = s_red + (warp % step) * kRows * 9;
                if (warp >= step && warp < 2 * step) {
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) buf[(i * 16 + g + (e >> 1) * 8) * 9 + 2 * t4 + (e & 1)] = acc[i][e];
                }
                __syncthreads();
                if (warp < step) {
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][e] += buf[(i * 16 + g + (e >> 1) * 8) * 9 + 2 * t4 + (e & 1)];
                }
                __syncthreads();
            }
            if (warp == 0) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s_h[(2 * t4 + (e & 1)) * (kRows + 1) + i * 16 + g + (e >> 1) * 8] = acc[i][e];
            }
        } else {
            // Rows of 128 bytes, 16-byte pieces swapped by the row so that eight rows of one piece lie in different banks; or, where rows
            // begin in the middle of words, the 33 words that hold the row's 64 elements, at 144 bytes a row.
            const bool loose = p.vec_k == 1;
            auto stage_row = [&](uint8_t* base, int r, int c, const uint16_t* row, int64_t u) {
                if (!loose) {
                    stage8(base + r * 128 + ((c ^ (r & 7)) << 4), row, u * kUnit + c * 8, p.K, p.vec_k);
                } else {
                    const uint16_t* at = row + u * kUnit;
                    const int odd = (reinterpret_cast<uintptr_t>(at) & 2u) != 0u ? 1 : 0;
                    const int64_t left = p.K - u * kUnit + odd;         // elements from the first word on
                    for (int i = c; i < 33; i += 8) {
                        const int64_t bytes = min(max((left - 2 * i) * 2, int64_t(0)), int64_t(4));
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;"
                                     :: "r"(smem_u32(base + r * kRowBytes + 4 * i)), "l"(bytes > 0 ? at - odd + 2 * i : at - odd), "r"(static_cast<int>(bytes)) : "memory");
                    }
                }
            };
            const size_t a_at = size_t(kWindow) * (loose ? kRowBytes : 128);
            auto stage = [&](int64_t u) {
                uint8_t* sx = s_mem + (u - u0) % ST * kStage;
                uint8_t* sa = sx + a_at;
#pragma unroll
                for (int i = tid; i < kWindow * 8; i += kAdThreads) {
                    const int r = i >> 3;
                    if (r < count) stage_row(sx, r, i & 7, p.x + (t0 + list[r]) * p.ldx, u);
                }
#pragma unroll
                for (int i = tid; i < kRows * 8; i += kAdThreads) {
                    const int r = i >> 3;
                    if (r < p.R) stage_row(sa, r, i & 7, A + r * p.K, u);
                }
            };
            // which rows that this lane reads begin in the middle of a word (stages are of whole words)
            auto shift_of = [&](const uint16_t* row) { return (reinterpret_cast<uintptr_t>(row) & 2u) != 0u ? 16u : 0u; };
            // warps: two halves of the tokens x four; those share out the rows of A (16 each, 32 of 128), or, with fewer, a stage's steps of 16
            constexpr int MI = MT == 8 ? 2 : 1, KS = MT >= 4 ? 1 : 4 / MT;
            const int half = warp >> 2, m = (warp & 3) % (MT < 4 ? MT : 4), ks = (warp & 3) / (MT < 4 ? MT : 4);
            uint32_t shift_a[MI][2], shift_x[4];
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) shift_a[i][e] = shift_of(A + ((m + 4 * i) * 16 + g + e * 8) * p.K);
#pragma unroll
            for (int j = 0; j < 4; ++j) shift_x[j] = half * 32 + j * 8 + g < count ? shift_of(p.x + (t0 + list[half * 32 + j * 8 + g]) * p.ldx) : 0u;
            float acc[MI][4][4] = {};
            for (int s = 0; s < ST - 1; ++s) {
                if (u0 + s < u1) stage(u0 + s);
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
            for (int64_t u = u0; u < u1; ++u) {
                asm volatile("cp.async.wait_group %0;" :: "n"(ST - 2) : "memory");
                __syncthreads();
                if (u + ST - 1 < u1) stage(u + ST - 1);
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (half * 32 < count) {
                    const uint8_t* sx = s_mem + (u - u0) % ST * kStage + half * 32 * (loose ? kRowBytes : 128);
                    const uint8_t* sa = s_mem + (u - u0) % ST * kStage + a_at;
#pragma unroll
                    for (int kk = ks; kk < 4; kk += KS) {
                        uint32_t fa[MI][4], fb[2][4];
                        if (!loose) {
#pragma unroll
                            for (int i = 0; i < MI; ++i) {
                                const int r = (m + 4 * i) * 16 + (lane & 15);
                                load_matrices(fa[i], sa + r * 128 + (((kk * 2 + (lane >> 4)) ^ (r & 7)) << 4));
                            }
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const int r = j * 16 + (lane & 7) + ((lane >> 4) << 3);
                                load_matrices(fb[j], sx + r * 128 + (((kk * 2 + ((lane >> 3) & 1)) ^ (r & 7)) << 4));
                            }
                        } else {
                            auto pair = [&](const uint8_t* base, int r, int word, uint32_t shift) {
                                const uint32_t* at = reinterpret_cast<const uint32_t*>(base + r * kRowBytes) + word;
                                return __funnelshift_r(at[0], at[1], shift);
                            };
#pragma unroll
                            for (int i = 0; i < MI; ++i)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {           // rows g, g + 8; the first and second eight of the contraction
                                    const int r = (m + 4 * i) * 16 + g + (e & 1) * 8;
                                    fa[i][e] = pair(sa, r, kk * 8 + t4 + (e >> 1) * 4, shift_a[i][e & 1]);
                                }
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int e = 0; e < 2; ++e) fb[j >> 1][(j & 1) * 2 + e] = pair(sx, j * 8 + g, kk * 8 + t4 + e * 4, shift_x[j]);
                        }
#pragma unroll
                        for (int i = 0; i < MI; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) mma16<DT>(acc[i][j], fa[i][0], fa[i][1], fa[i][2], fa[i][3], fb[j >> 1][(j & 1) * 2], fb[j >> 1][(j & 1) * 2 + 1]);
                    }
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (ks == s) {
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float* at = s_h + (half * 32 + j * 8 + 2 * t4 + (e & 1)) * (kRows + 1) + (m + 4 * i) * 16 + g + (e >> 1) * 8;
                                *at = s == 0 ? acc[i][j][e] : *at + acc[i][j][e];
                            }
                }
                if (s + 1 < KS) __syncthreads();
            }
        }
        __syncthreads();
        if (ranks > 1) cluster_barrier();
        // a warp for each token of this block's share
        for (int m = rank + warp * ranks; m < count; m += ranks * (kAdThreads / 32)) {
            finish_token<DT>(p, s_h + m * (kRows + 1), ranks, t0 + list[m], a);
        }
        // nobody writes its sums over while they are being read
        if (ranks > 1) cluster_barrier();
        else __syncthreads();
    }
}

// ---- out = y + B h ---------------------------------------------------------------------------------------------------
// grid (blocks of 32 columns for each warp, windows, adapters of a window in turn).  A warp keeps its 32 columns of B_a in registers and takes the adapter's
// tokens 16 at a time, y of the next 16 on the way.  The four products of 8 columns share them out so that each lane ends up with 8
// neighbouring columns.
template <int YT> struct Piece { uint32_t r[YT == CQ_F32 ? 8 : 4]; };           // 8 columns of a row of y

template <int YT>
__device__ __forceinline__ Piece<YT> load_piece(const AdapterArgs& p, int64_t t, int64_t col) {
    Piece<YT> v = {};
    if (t < 0 || col >= p.N) return v;
    if constexpr (YT == CQ_F32) {
        const uint32_t* y = static_cast<const uint32_t*>(p.y) + t * p.ldy + col;
        if (p.vec_n == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (col + 4 * i < p.N) {
                    const uint4 w = __ldcg(reinterpret_cast<const uint4*>(y) + i);
                    v.r[4 * i] = w.x; v.r[4 * i + 1] = w.y; v.r[4 * i + 2] = w.z; v.r[4 * i + 3] = w.w;
                }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < p.N) v.r[i] = __ldcg(y + i);
        }
    } else {
        const uint4 w = piece8(static_cast<const uint16_t*>(p.y) + t * p.ldy, col, p.N, p.vec_n);
        v.r[0] = w.x; v.r[1] = w.y; v.r[2] = w.z; v.r[3] = w.w;
    }
    return v;
}
// y + f d, rounded once
template <int YT>
__device__ __forceinline__ void add_store(const AdapterArgs& p, int64_t t, int64_t col, const Piece<YT>& y, const float (&d)[8], float f) {
    if (t < 0 || col >= p.N) return;
    if constexpr (YT == CQ_F32) {
        float* out = static_cast<float*>(p.out) + t * p.ldo + col;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __fmaf_rn(d[i], f, __uint_as_float(y.r[i]));
        if (p.vec_n == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (col + 4 * i < p.N) reinterpret_cast<float4*>(out)[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < p.N) out[i] = o[i];
        }
    } else {
        uint16_t* out = static_cast<uint16_t*>(p.out) + t * p.ldo + col;
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = unpack16x2<YT>(y.r[i]);
            o[i] = pack16x2<YT>(__fmaf_rn(d[2 * i], f, v.x), __fmaf_rn(d[2 * i + 1], f, v.y));
        }
        if (p.vec_n == 8) {
            *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
        } else if (p.vec_n >= 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + 2 * i < p.N) reinterpret_cast<uint32_t*>(out)[i] = o[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < p.N) out[i] = static_cast<uint16_t>(o[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// 32 columns from n0 on of up to 16 rows of y, plus d [16][36]: a word or an element of a row for each lane
template <int YT>
__device__ __forceinline__ void add_rows(const AdapterArgs& p, const float* d, const uint8_t* list, int count, int64_t t0, int64_t n0) {
    const int lane = threadIdx.x & 31;
    const uint16_t* y = static_cast<const uint16_t*>(p.y);
    uint16_t* out = static_cast<uint16_t*>(p.out);
    if (p.vec_n >= 2) {
        const int64_t n = n0 + 2 * (lane & 15);
        if (n >= p.N) return;
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = 2 * i + (lane >> 4);
            if (m < count) w[i] = __ldcg(reinterpret_cast<const uint32_t*>(y + (t0 + list[m]) * p.ldy + n));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = 2 * i + (lane >> 4);
            if (m >= count) continue;
            const float2 v = unpack16x2<YT>(w[i]);
            *reinterpret_cast<uint32_t*>(out + (t0 + list[m]) * p.ldo + n) = pack16x2<YT>(v.x + d[m * 36 + 2 * (lane & 15)], v.y + d[m * 36 + 2 * (lane & 15) + 1]);
        }
    } else {
        const int64_t n = n0 + lane;
        if (n >= p.N) return;
        uint16_t w[16];
#pragma unroll
        for (int m = 0; m < 16; ++m)
            if (m < count) w[m] = __ldcg(y + (t0 + list[m]) * p.ldy + n);
#pragma unroll
        for (int m = 0; m < 16; ++m)
            if (m < count) out[(t0 + list[m]) * p.ldo + n] = pack16<YT>(cvt16<YT>(w[m]) + d[m * 36 + lane]);
    }
}

// words between rows of h in shared memory: 8 more than a multiple of 32, so that the rows of a fragment lie in different banks
template <int MT> __host__ __device__ constexpr int h_pitch() { return MT * 8 + (MT == 1 ? 0 : MT == 2 ? 24 : 8); }

// SHARE: the block's tokens have their h in shared memory, else each warp takes it from L2.
// Three blocks an SM for ranks up to 32, although that spills 16 to 100 bytes: 64 x 8192 x 8192 on 64 adapters 20.6 us, 23.6 with two blocks and no
// spills, 100 x 4096 x 11008 on 40 65.4, 69.2; against it 100 x 2060 x 1003 on 3, rows of y on 2 bytes, 18.8, 17.0.  Ranks above spill 32 to 72.
template <int MT, int DT, int YT, bool SHARE>
__global__ void __launch_bounds__(kAdThreads, MT <= 2 ? 3 : 2)
k26_adapter_out(const AdapterArgs p) {
    constexpr int kPitch = h_pitch<MT>();
    constexpr int kHeld = MT == 8 ? 32 : kWindow;               // tokens whose h is in shared memory at a time
    __shared__ uint8_t s_list[kAdThreads / 32][kWindow];
    __shared__ __align__(16) uint32_t s_h[2][SHARE ? kHeld : 1][kPitch];
    __shared__ float s_d[YT == CQ_F32 ? 1 : kAdThreads / 32][16 * 36];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    uint8_t* list = s_list[warp];
    asm volatile("griddepcontrol.launch_dependents;");
    const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kWindow;
    Window w;
    w.read(p, t0);
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * blockDim.x + warp * 32, col = n0 + 8 * t4;
    bool waited = false;
    Turn turn(w, gridDim.z);
    int a;
    uint64_t tokens;
    while (turn.next(w, blockIdx.z, gridDim.z, a, tokens)) {
        __syncwarp();
        write_list(tokens, list);
        const int count = __popcll(tokens);
        auto token = [&](int m) { return m < count ? t0 + list[m] : int64_t(-1); };
        const bool direct = YT == CQ_F32 || p.vec_n == 8;
        Piece<YT> ya = {}, yb = {};
        if (direct) {
            ya = load_piece<YT>(p, token(g), col);
            yb = load_piece<YT>(p, token(8 + g), col);
        }
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
        const bool few = !SHARE || count <= 16;
        for (int base = 0; base < count; base += kHeld) {
            const int held = min(kHeld, count - base), pieces = p.R / 8;         // 16 bytes each
            if (!few) {
                __syncthreads();
                for (int i = tid; i < 2 * held * pieces; i += blockDim.x) {
                    const int part = i >= held * pieces ? 1 : 0, at = i - part * held * pieces, m = at / pieces, c = at - m * pieces;
                    const uint16_t* h = (part == 0 ? p.high : p.low) + (t0 + list[base + m]) * p.R + c * 8;
                    *reinterpret_cast<uint4*>(&s_h[part][m][c * 4]) = __ldcg(reinterpret_cast<const uint4*>(h));
                }
                __syncthreads();
            }
            for (int m0 = 0; m0 < held; m0 += 16) {
                const int64_t ta = token(base + m0 + g), tb = token(base + m0 + 8 + g);
                const float fa = ta >= 0 ? __ldcg(p.factor + ta) : 0.0f, fb = tb >= 0 ? __ldcg(p.factor + tb) : 0.0f;
                Piece<YT> na = {}, nb = {};
                if (direct) {
                    na = load_piece<YT>(p, token(base + m0 + 16 + g), col);
                    nb = load_piece<YT>(p, token(base + m0 + 24 + g), col);
                }
                float acc[4][4] = {};
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (i * 16 >= p.R) break;
                    const bool have_k = i * 16 + t4 * 4 < p.R;
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        uint2 ha = make_uint2(0, 0), hb = ha;
                        if (few) {
                            const uint16_t* h = (part == 0 ? p.high : p.low) + i * 16 + t4 * 4;
                            if (ta >= 0 && have_k) ha = __ldcg(reinterpret_cast<const uint2*>(h + ta * p.R));
                            if (tb >= 0 && have_k) hb = __ldcg(reinterpret_cast<const uint2*>(h + tb * p.R));
                        } else {
                            if (ta >= 0 && have_k) ha = *reinterpret_cast<const uint2*>(&s_h[part][m0 + g][i * 8 + t4 * 2]);
                            if (tb >= 0 && have_k) hb = *reinterpret_cast<const uint2*>(&s_h[part][m0 + 8 + g][i * 8 + t4 * 2]);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma16<DT>(acc[j], ha.x, hb.x, ha.y, hb.y, b[j][i].x, b[j][i].y);
                    }
                }
                if (direct) {
                    const float da[8] = {acc[0][0], acc[0][1], acc[1][0], acc[1][1], acc[2][0], acc[2][1], acc[3][0], acc[3][1]};
                    const float db[8] = {acc[0][2], acc[0][3], acc[1][2], acc[1][3], acc[2][2], acc[2][3], acc[3][2], acc[3][3]};
                    add_store<YT>(p, ta, col, ya, da, fa);
                    add_store<YT>(p, tb, col, yb, db, fb);
                } else {
                    // rows that begin anywhere: the products go through shared memory, so that a warp's accesses to a row lie side by side
                    float* d = s_d[warp];
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            d[g * 36 + 8 * t4 + 2 * j + e] = acc[j][e] * fa;
                            d[(8 + g) * 36 + 8 * t4 + 2 * j + e] = acc[j][2 + e] * fb;
                        }
                    __syncwarp();
                    if constexpr (YT != CQ_F32) add_rows<YT>(p, d, list + base + m0, min(16, held - m0), t0, n0);
                }
                ya = na;
                yb = nb;
            }
        }
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (blockIdx.z == 0 && p.out != p.y) {    // tokens without an adapter
        const int valid = static_cast<int>(min(static_cast<int64_t>(kWindow), p.T - t0));
        const uint64_t bare = ~w.any() & (valid < 64 ? (uint64_t(1) << valid) - 1u : ~uint64_t(0));
        __syncwarp();
        write_list(bare, list);
        const float zero[8] = {-0.0f, -0.0f, -0.0f, -0.0f, -0.0f, -0.0f, -0.0f, -0.0f};       // (y + -0 is y)
        for (int i = lane; i < __popcll(bare) * 4; i += 32) {   // this warp's 32 columns
            const int64_t t = t0 + list[i >> 2], c = n0 + (i & 3) * 8;
            add_store<YT>(p, t, c, load_piece<YT>(p, t, c), zero, 0.0f);
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
static size_t up256(size_t v) { return (v + 255) / 256 * 256; }
static size_t adapter_workspace(int64_t T, int64_t R) {
    return 2 * up256(sizeof(uint16_t) * T * R) + 2 * up256(sizeof(float) * T) + sizeof(int) * kTileInfo * ((T + kTileTokens - 1) / kTileTokens);
}

template <int MT, int DT>
static int launch_adapter(const AdapterArgs& p, int y_dtype, cudaStream_t st) {
    const int sms = sm_count();
    const bool in_tiles = adapter_in_tiles(p);
    const int64_t windows = (p.T + kWindow - 1) / kWindow;
    const int64_t adapters = std::min<int64_t>(kWindow, std::min<int64_t>(p.n, p.T));
    if (windows > 65535) return CQ_ERR_SHAPE;
    // Parts of the contraction of 512 or more, up to a portable cluster and while the windows' blocks fit twice an SM (one token x 4096: 7.2 us, 11.8
    // in one part); a block for each adapter of a window up to four an SM, twice as many as are resident: most windows have fewer adapters
    // than they might, and a block that finds none ends at once (64 tokens on 64 adapters x 8192 x 8192, rank 16: 14.4 us and 20.6 for the second kernel;
    // 28.2 and 26.4 with two an SM; 100 x 4096 x 11008 on 40: 28.9 and 65.4, 27.3 and 68.8).
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, p.K / 512), 2 * sms / windows));
    const int64_t slots = std::max<int64_t>(1, std::min<int64_t>(adapters, 4 * sms / (windows * parts)));
    static thread_local LaunchMemo memo;
    // (the static shared memory counts towards the 48 KB that need no leave)
    constexpr size_t smem = shrink_smem<MT>();
    static_assert(smem > 48 * 1024, "leave is asked for");
    if (resident_ctas(k25_adapter_in<MT, DT>, kAdThreads, smem, smem, memo) < 1) return CQ_ERR_CUDA;
    const dim3 grid(static_cast<unsigned>(parts), static_cast<unsigned>(windows), static_cast<unsigned>(slots));
    int rc = CQ_OK;
    if (in_tiles) rc = launch_adapter_in_tiles(p, DT, st);
    else rc = launch_ex(k25_adapter_in<MT, DT>, grid, kAdThreads, smem, st, grid.x, !tuning_no_pdl(), p);
    if (rc != CQ_OK) return rc;
    if (p.tiles) return launch_adapter_out_tiles(p, DT, y_dtype, st);
    // two, four or eight warps to a block: the most with which there are two blocks an SM (50 x 1003, rank 128: 41.5 us with two, 45.6 with eight)
    int warps = 8;
    while (warps > 2 && windows * adapters * ((p.N + 32 * warps - 1) / (32 * warps)) < 2 * sms) warps /= 2;
    const int64_t cols = (p.N + 32 * warps - 1) / (32 * warps);
    const int64_t turns = std::max<int64_t>(1, std::min<int64_t>(adapters, 16 * sms / (windows * cols)));
    const dim3 grid2(static_cast<unsigned>(cols), static_cast<unsigned>(windows), static_cast<unsigned>(turns));
    const unsigned threads = 32u * warps;
    // Blocks that fill the SMs more than once share their tokens' h in shared memory (64 x 100000, rank 64: 43 us, 62 without); with fewer
    // that costs more than it saves (64 x 6144, rank 64: 20.2 us without, 24.0 with).
    const bool share = windows * cols > 2 * sms;
    auto launch = [&](auto y_type) {
        constexpr int YT = decltype(y_type)::value;
        return share ? launch_ex(k26_adapter_out<MT, DT, YT, true>, grid2, threads, 0, st, 1, !tuning_no_pdl(), p)
                     : launch_ex(k26_adapter_out<MT, DT, YT, false>, grid2, threads, 0, st, 1, !tuning_no_pdl(), p);
    };
    if (y_dtype == CQ_F32) return launch(std::integral_constant<int, CQ_F32>());
    if (y_dtype == CQ_F16) return launch(std::integral_constant<int, CQ_F16>());
    return launch(std::integral_constant<int, CQ_BF16>());
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
    uint8_t* at = static_cast<uint8_t*>(workspace) + up256(sizeof(uint16_t) * T * R);
    p.low = reinterpret_cast<uint16_t*>(at);
    at += up256(sizeof(uint16_t) * T * R);
    p.factor = reinterpret_cast<float*>(at);
    at += up256(sizeof(float) * T);
    p.slot = reinterpret_cast<int*>(at);
    p.info = reinterpret_cast<int*>(at + up256(sizeof(int) * T));
    p.T = T; p.K = K; p.N = N; p.R = static_cast<int>(R); p.n = static_cast<int>(n);
    // the widest access that every row's beginning and length allow
    for (p.vec_k = 8; p.vec_k > 1; p.vec_k /= 2)
        if (K % p.vec_k == 0 && (T == 1 || ldx % p.vec_k == 0) && ptr_aligned(X, 2 * p.vec_k) && ptr_aligned(A, 2 * p.vec_k)) break;
    for (p.vec_n = static_cast<int>(16 / elem); p.vec_n > 1; p.vec_n /= 2)
        if (N % p.vec_n == 0 && (T == 1 || (ldy % p.vec_n == 0 && ldo % p.vec_n == 0)) && ptr_aligned(y, elem * p.vec_n) && ptr_aligned(out, elem * p.vec_n)) break;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    p.tiles = adapter_out_tiles(p, y_dtype);
    return dtype == CQ_F16 ? launch_adapter_rank<CQ_F16>(p, y_dtype, st) : launch_adapter_rank<CQ_BF16>(p, y_dtype, st);
}

}  // extern "C"
