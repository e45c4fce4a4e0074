// Low-rank adapters: what the kernels for few and for many tokens share.
#pragma once

#include "cq_serve.cuh"

namespace cq {

constexpr int kMaxRank = 128;
constexpr int kTileTokens = 128;              // tokens of a tile of the kernels for many tokens
constexpr int kTileInfo = kTileTokens + 4;    // of each: how many adapters it has, then which, in order of their first tokens

struct AdapterArgs {
    const uint16_t* x; int64_t ldx;
    const void* y; int64_t ldy;
    void* out; int64_t ldo;
    const uint16_t* A; const uint16_t* B; const float* scale;
    const int* index;
    uint16_t* high; uint16_t* low; float* factor;               // [T][R], [T][R], [T]
    int* slot; int* info;                                       // [T]: which of its tile's adapters; [tiles][kTileInfo] (many tokens)
    int64_t T, K, N;
    int R, n;
    int vec_k, vec_n;                                           // elements of one access to rows of x and A (of y and out)
    bool tiles;                                                 // the second kernel wants `slot` and `info`
};

// Many tokens on the 5th-generation tensor cores (cq_adapter_tiles.cu): whether either kernel takes them, and its launch.
bool adapter_in_tiles(const AdapterArgs& p);
bool adapter_out_tiles(const AdapterArgs& p, int y_dtype);
int launch_adapter_in_tiles(const AdapterArgs& p, int dtype, cudaStream_t st);
int launch_adapter_out_tiles(const AdapterArgs& p, int dtype, int y_dtype, cudaStream_t st);
int adapter_stage_fault(unsigned int* fault_host);

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

// The adapters of a tile in order of their first tokens, by a block of 128 threads or more; returns how many.
struct __align__(16) TileSort {
    int idx[kTileTokens];                     // of each token (-1: none)
    int first[kTileTokens], rank[kTileTokens], slot[kTileTokens], adapter[kTileTokens], leads[4];
};
__device__ __forceinline__ int sort_tile(const AdapterArgs& p, int64_t t0, TileSort& s, bool write) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid < kTileTokens) {
        const int a = t0 + tid < p.T ? __ldcg(p.index + t0 + tid) : -1;
        s.idx[tid] = a >= 0 && a < p.n ? a : -1;
    }
    __syncthreads();
    if (tid < kTileTokens) {
        const int a = s.idx[tid];
        int first = (warp << 5) + __ffs(__match_any_sync(0xFFFFFFFFu, a)) - 1;
        for (int j = warp * 8 - 1; j >= 0; --j) {               // four tokens of the warps before
            const int4 v = reinterpret_cast<const int4*>(s.idx)[j];
            first = v.w == a ? 4 * j + 3 : first;
            first = v.z == a ? 4 * j + 2 : first;
            first = v.y == a ? 4 * j + 1 : first;
            first = v.x == a ? 4 * j : first;
        }
        s.first[tid] = first;
        const unsigned lead = __ballot_sync(0xFFFFFFFFu, a >= 0 && first == tid);
        s.rank[tid] = __popc(lead & ((1u << lane) - 1u));
        if (lane == 0) s.leads[warp] = __popc(lead);
    }
    __syncthreads();
    const int count = s.leads[0] + s.leads[1] + s.leads[2] + s.leads[3];
    if (tid < kTileTokens && s.idx[tid] >= 0 && s.first[tid] == tid) {
        int rank = s.rank[tid];
        for (int w = 0; w < warp; ++w) rank += s.leads[w];
        s.rank[tid] = rank;
        s.adapter[rank] = s.idx[tid];
    }
    __syncthreads();
    if (tid < kTileTokens) {
        const int slot = s.idx[tid] >= 0 ? s.rank[s.first[tid]] : -1;
        s.slot[tid] = slot;
        if (write) {
            int* info = p.info + t0 / kTileTokens * kTileInfo;
            if (tid == 0) info[0] = count;
            if (tid < count) info[1 + tid] = s.adapter[tid];
            if (t0 + tid < p.T) p.slot[t0 + tid] = slot;
        }
    }
    __syncthreads();
    return count;
}

// h[r] = the sum of `ranks` blocks' s_h[r], in rank order, as two 16-bit halves and a factor; a warp for each token.
template <int DT>
__device__ __forceinline__ void finish_token(const AdapterArgs& p, const float* s_h, int ranks, int64_t t, int a) {
    constexpr int kPer = kMaxRank / 32;
    const int lane = threadIdx.x & 31;
    float h[kPer], top = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = lane + 32 * i;
        h[i] = 0.0f;
        if (r < p.R) {
            if (ranks > 1) {
#pragma unroll 8
                for (int k = 0; k < ranks; ++k) h[i] += ld_rank(s_h + r, k);
            } else {
                h[i] = s_h[r];
            }
        }
        const float v = fabsf(h[i]);
        top = fmaxf(top, v < INFINITY ? v : 0.0f);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
    // 2^e, the power of two at or below the largest, within fp32's normal numbers: h 2^-e lies below 2
    const uint32_t e = min(max(__float_as_uint(top) >> 23, 2u), 252u);
    const float down = __uint_as_float((254u - e) << 23);
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

}  // namespace cq
