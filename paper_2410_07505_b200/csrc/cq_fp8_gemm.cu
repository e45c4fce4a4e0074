// Product of block-quantized 8-bit float matrices (e4m3) on the 5th-generation tensor cores:
//
//   Y[m, n] = sum_b  sa[b, m] sw[n / 128, b]  sum_{k in block b} A[m, k] W[n, k],     blocks of 128 along k
//
// The scales change from block to block along the contraction, so a block's 128-long inner sum is formed by itself
// (four tcgen05.mma of 32, fp32 in tensor memory) and added to the running result in fp32 registers with the block's
// factor, one fused multiply-add for an element and block.  Two to four accumulator buffers in tensor memory let the
// tensor cores form the next block while the epilogue warps read the last one.  Tiles arrive by TMA (128-byte swizzle,
// zero fill past the edges, so odd sizes need no other path); every wait is bounded.
//
// Two kernels, chosen by the number of tiles that the product has (launch_product):
//   k12_product      tiles of 128 rows of A x 256 (or 128) rows of W, one persistent CTA an SM; or, for few tiles, a pair
//                    of CTAs for a tile that take half of the contraction each
//   k13_product_few  the operands swapped (128 rows of W x 16..128 rows of A) and the contraction split over a
//                    thread-block cluster, joined through distributed shared memory in rank order (no atomics: the
//                    same bits every time); few rows of A leave the read of W as the bound
//
// Measured (quantizer included, operands not in L2): 4096 x 8192 x 28672 (rows x K x N) 0.85 ms from a cool chip and 0.99 ms
// in a long run, which the power limit sets (2.26 and 1.94 PFLOP/s); 1 x 8192 x 8192 15.2 us (4.4 TB/s of weights),
// 48 x 5120 x 13824 22.3 us, 777 x 2060 x 1003 15.6 us.  The first is bound by shared memory: a block's operands (48 KB for
// 256 columns) are written once and read once, 768 cycles at 128 bytes each, beside 512 of products and 256 of
// multiply-adds.  Pairs of CTAs, which would halve the reads of W, took 1580 us where this took 952; the cause was not
// isolated.  The next two are the read of W and about 5 us of launches, first loads and joins (the second also 2 parts of 108
// tiles on 148 SMs, 1.37 times the average on the busiest); the last is those alone.
#include "cq_serve.cuh"

#include <atomic>

namespace cq {

__device__ unsigned int g_fp8_fault = 0;      // set if a bounded wait ever gave up

constexpr int kBlkK = 128;                    // bytes and elements of one block along the contraction

template <int OUT>
__device__ __forceinline__ uint16_t to16(float v) {
    if constexpr (OUT == CQ_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    else return __half_as_ushort(__float2half_rn(v));
}

// Four products of 32 along one block: operands in shared memory, fresh accumulator.
__device__ __forceinline__ void mma_block(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
#pragma unroll
    for (int k = 0; k < 4; ++k) tc_mma_fp8(d, a + 2 * k, b + 2 * k, idesc, k != 0);      // 32 bytes further along the swizzled row
}

// ---- thread-block clusters ----------------------------------------------------------------------------
__device__ __forceinline__ float ld_cluster(uint32_t local, uint32_t rank) {
    uint32_t remote;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- many rows ------------------------------------------------------------------------------------
constexpr int kTileM = 128;
constexpr int kGroupM = 32;                   // tiles of A that share a sweep over W, so that both sides come from L2
constexpr int kMainThreads = 384;             // warp 0: loads, warp 1: products, warps 4..11: running sums and stores
constexpr size_t kPatch = 4096;               // staging of one warp's 32 rows x 128 bytes of output

template <int BN> __host__ __device__ constexpr int main_stages() { return BN == 256 ? 4 : 5; }
template <int BN> __host__ __device__ constexpr size_t main_stage_bytes() { return (size_t(128) + BN) * kBlkK; }
template <int BN> __host__ __device__ constexpr size_t main_smem() {
    return main_stages<BN>() * (main_stage_bytes<BN>() + 128 * 4) + 8 * kPatch + 256;
}

struct MainArgs {
    const float* sa; int64_t lds;             // scales of A, [K blocks][lds]
    const float* sw;                          // scales of W, [N blocks][K blocks]
    void* out; int64_t ldo;
    int64_t M, N;
    int kblocks, mtiles, ntiles;
};

struct TilePos { int m, n; };
__device__ __forceinline__ TilePos tile_at(int64_t t, int mtiles, int ntiles) {
    const int64_t per_group = static_cast<int64_t>(kGroupM) * ntiles;
    const int g = static_cast<int>(t / per_group);
    const int64_t r = t - g * per_group;
    const int rows = min(kGroupM, mtiles - g * kGroupM);
    return {g * kGroupM + static_cast<int>(r % rows), static_cast<int>(r / rows)};
}

// SPLIT: two CTAs of a cluster take half of the contraction each, one tile a cluster; each finishes half of the columns.
template <int BN, int OUT, bool SPLIT>
__global__ void __launch_bounds__(kMainThreads, 1)
k12_product(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapW, const MainArgs p) {
    constexpr int ST = main_stages<BN>();
    constexpr size_t kA = size_t(128) * kBlkK, kB = size_t(BN) * kBlkK;
    constexpr int TB = 512 / BN;              // accumulator buffers in tensor memory
    constexpr int kCols = BN / 2;             // columns of the tile for each epilogue warp
    // No static shared memory, so that the dynamic part starts on the 1024-byte boundary that the swizzle wants.
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* s_a = smem;
    uint8_t* s_b = s_a + ST * kA;
    uint8_t* s_patch = s_b + ST * kB;
    float* s_scale = reinterpret_cast<float*>(s_patch + 8 * kPatch);
    uint64_t* full = reinterpret_cast<uint64_t*>(s_scale + ST * 128);
    uint64_t* empty = full + ST;
    uint64_t* tfull = empty + ST;
    uint64_t* tempty = tfull + TB;
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(tempty + TB);
    volatile uint32_t& s_dead = *(reinterpret_cast<volatile uint32_t*>(tempty + TB) + 1);
    static_assert((2 * ST + 2 * TB) * 8 + 8 <= 256, "barriers");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    asm volatile("griddepcontrol.launch_dependents;");
    if (threadIdx.x == 0) {
        if ((smem_u32(smem) & 1023u) != 0u) atomicExch(&g_fp8_fault, 1u);      // cannot be: see above
        for (int i = 0; i < ST; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 8); }
        for (int i = 0; i < TB; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 8); }
        mbar_init_fence();
        s_dead = 0;
        prefetch_map(&mapA);
        prefetch_map(&mapW);
    }
    if (warp == 1) tmem_alloc(&s_tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const int64_t ntotal = static_cast<int64_t>(p.mtiles) * p.ntiles;
    const int rank = SPLIT ? blockIdx.x & 1 : 0;
    const int kb_first = SPLIT && rank == 1 ? p.kblocks / 2 : 0, kb_end = SPLIT && rank == 0 ? p.kblocks / 2 : p.kblocks;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 0) {
            int s = 0;
            uint32_t round = 0, issued = 0;
            bool ok = true;
            asm volatile("griddepcontrol.wait;" ::: "memory");
            for (int64_t t = SPLIT ? blockIdx.x >> 1 : blockIdx.x; ok && t < ntotal; t += SPLIT ? ntotal : gridDim.x) {
                const TilePos pos = tile_at(t, p.mtiles, p.ntiles);
                const int64_t m0 = static_cast<int64_t>(pos.m) * kTileM;
                const uint32_t sbytes = static_cast<uint32_t>(min(int64_t(128), (p.M - m0 + 3) & ~int64_t(3))) * 4;
                for (int kb = kb_first; kb < kb_end; ++kb) {
                    if (!(ok = role_wait(&empty[s], round ^ 1u, &s_dead))) break;
                    if (elect_one()) {
                        mbar_expect_tx(&full[s], static_cast<uint32_t>(kA + kB) + sbytes);
                        tile_load(s_a + s * kA, &mapA, kb * kBlkK, static_cast<int32_t>(m0), &full[s]);
                        tile_load(s_b + s * kB, &mapW, kb * kBlkK, pos.n * BN, &full[s]);
                        bulk_load(s_scale + s * 128, p.sa + kb * p.lds + m0, sbytes, &full[s]);
                    }
                    issued = min(issued + 1, uint32_t(ST));
                    if (++s == ST) { s = 0; round ^= 1u; }
                }
            }
            if (!ok)                          // copies still in flight land before the CTA leaves
                for (; issued > 0; --issued) {
                    if (--s < 0) { s = ST - 1; round ^= 1u; }
                    for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&full[s], round); ++polls) {}
                }
        } else if (warp == 1) {
            const uint32_t idesc = idesc_fp8(kTileM, BN);
            const uint64_t desc_a = smem_desc_k128(s_a), desc_b = smem_desc_k128(s_b);
            int s = 0, b = 0, pending = 0;
            uint32_t round = 0, turn = 0;
            bool ok = true;
            for (int64_t t = SPLIT ? blockIdx.x >> 1 : blockIdx.x; ok && t < ntotal; t += SPLIT ? ntotal : gridDim.x) {
                for (int kb = kb_first; kb < kb_end; ++kb) {
                    if (!(ok = role_wait(&full[s], round, &s_dead) && role_wait(&tempty[b], turn ^ 1u, &s_dead))) break;
                    tc_fence_after();
                    if (elect_one()) {
                        mma_block(tmem + b * BN, desc_a + s * (kA >> 4), desc_b + s * (kB >> 4), idesc);
                        tc_commit(&tfull[b]);             // (the stage is released by the epilogue, which waits for this)
                    }
                    pending = min(pending + 1, TB);
                    if (++s == ST) { s = 0; round ^= 1u; }
                    if (++b == TB) { b = 0; turn ^= 1u; }
                }
            }
            // the last products of each buffer are waited for by the epilogue; after a wait that gave up, here
            if (!ok)
                for (; pending > 0; --pending) {
                    if (--b < 0) { b = TB - 1; turn ^= 1u; }
                    for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&tfull[b], turn); ++polls) {}
                }
        }
        if constexpr (SPLIT) {
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int ew = warp - 4, half = ew >> 2, q = ew & 3;      // half of the columns and 32 rows of the CTA's tile for each warp
        const int row = q * 32 + lane;
        const uint32_t taddr = tmem + (static_cast<uint32_t>(q * 32) << 16) + half * kCols;
        uint8_t* patch = s_patch + ew * kPatch;
        const int64_t nblocks = (p.N + 127) / 128;
        int s = 0, b = 0;
        uint32_t round = 0, turn = 0;
        bool ok = true;
        for (int64_t t = SPLIT ? blockIdx.x >> 1 : blockIdx.x; ok && t < ntotal; t += SPLIT ? ntotal : gridDim.x) {
            const TilePos pos = tile_at(t, p.mtiles, p.ntiles);
            const int64_t nb = min((static_cast<int64_t>(pos.n) * BN + half * kCols) / 128, nblocks - 1);
            const float* sw = p.sw + nb * p.kblocks;
            float acc[kCols];
#pragma unroll
            for (int i = 0; i < kCols; ++i) acc[i] = 0.0f;
            float w = __ldg(sw + kb_first);
            for (int kb = kb_first; kb < kb_end; ++kb) {
                const float w_next = __ldg(sw + min(kb + 1, p.kblocks - 1));
                if (!(ok = role_wait(&tfull[b], turn, &s_dead) && role_wait(&full[s], round, &s_dead))) break;
                tc_fence_after();
                float v[2][32];
                tmem_ld32(taddr + b * BN, v[0]);
                const float f = __fmul_rn(s_scale[s * 128 + row], w);
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[s]);    // the products have read the stage, and this warp its scales
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    tmem_ld_wait(v[c & 1]);
                    if (c + 1 < kCols / 32) {
                        tmem_ld32(taddr + b * BN + (c + 1) * 32, v[(c + 1) & 1]);
                    } else {                  // everything is in registers: the buffer is free
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&tempty[b]);
                    }
                    // (scalar multiply-adds: the packed ones run at 0.37 an SM partition and cycle here, these at 0.93)
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[c * 32 + i] = __fmaf_rn(v[c & 1][i], f, acc[c * 32 + i]);
                }
                w = w_next;
                if (++s == ST) { s = 0; round ^= 1u; }
                if (++b == TB) { b = 0; turn ^= 1u; }
            }
            if constexpr (SPLIT) {
                // every product of this CTA has completed, so the stages may be written over
                float* part = reinterpret_cast<float*>(smem) + q * kCols * 32 + lane;
                if (half != rank) {
#pragma unroll
                    for (int i = 0; i < kCols; ++i) part[i * 32] = acc[i];
                }
                __syncwarp();
                cluster_sync_all();
                if (half == rank) {
#pragma unroll
                    for (int i = 0; i < kCols; ++i) acc[i] = __fadd_rn(acc[i], ld_cluster(smem_u32(part + i * 32), rank ^ 1));
                }
                __syncwarp();
                cluster_sync_all();               // nobody leaves while its sums are being read
                if (half != rank) break;
            }
            if (!ok) break;
            // through a 4 KB patch of shared memory (a row of 128 bytes for each lane, 16-byte pieces rotated by the row)
            // so that the stores to memory are whole rows
            constexpr int kElem = OUT == CQ_F32 ? 4 : 2;
            constexpr int kPer = 128 / kElem;                     // columns of one patch
            const int64_t m0 = static_cast<int64_t>(pos.m) * kTileM + q * 32;
            const int64_t n0 = static_cast<int64_t>(pos.n) * BN + half * kCols;
            uint8_t* out = static_cast<uint8_t*>(p.out);
            const uint32_t align = static_cast<uint32_t>(p.ldo * kElem) | static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p.out));   // of all rows
#pragma unroll
            for (int c = 0; c < kCols / kPer; ++c) {
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint4 o;
                    if constexpr (OUT == CQ_F32) {
                        const float* a = &acc[c * 32 + j * 4];
                        o = make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(a[2]), __float_as_uint(a[3]));
                    } else {
                        const float* a = &acc[c * 64 + j * 8];
                        o = make_uint4(pack16x2<OUT>(a[0], a[1]), pack16x2<OUT>(a[2], a[3]), pack16x2<OUT>(a[4], a[5]), pack16x2<OUT>(a[6], a[7]));
                    }
                    *reinterpret_cast<uint4*>(patch + lane * 128 + ((j + lane) & 7) * 16) = o;
                }
                __syncwarp();
                const int64_t nc = n0 + c * kPer;
                if (nc + kPer <= p.N && (align & 15u) == 0u) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int rr = r * 4 + (lane >> 3);
                        const uint4 o = *reinterpret_cast<const uint4*>(patch + rr * 128 + (((lane & 7) + rr) & 7) * 16);
                        if (m0 + rr < p.M)
                            *reinterpret_cast<uint4*>(out + ((m0 + rr) * p.ldo + nc) * kElem + (lane & 7) * 16) = o;
                    }
                } else if (nc + kPer <= p.N && (align & 3u) == 0u) {       // a word of each row for each lane
#pragma unroll 8
                    for (int rr = 0; rr < 32; ++rr) {
                        const uint32_t o = *reinterpret_cast<const uint32_t*>(patch + rr * 128 + (((lane >> 2) + rr) & 7) * 16 + (lane & 3) * 4);
                        if (m0 + rr < p.M) *reinterpret_cast<uint32_t*>(out + ((m0 + rr) * p.ldo + nc) * kElem + lane * 4) = o;
                    }
                } else {
                    for (int rr = 0; rr < 32 && m0 + rr < p.M; ++rr) {
#pragma unroll
                        for (int e = lane; e < kPer; e += 32) {
                            const int byte = e * kElem;
                            const uint8_t* src = patch + rr * 128 + ((byte / 16 + rr) & 7) * 16 + (byte & 15);
                            if (nc + e < p.N) {
                                if constexpr (OUT == CQ_F32) reinterpret_cast<float*>(out)[(m0 + rr) * p.ldo + nc + e] = *reinterpret_cast<const float*>(src);
                                else reinterpret_cast<uint16_t*>(out)[(m0 + rr) * p.ldo + nc + e] = *reinterpret_cast<const uint16_t*>(src);
                            }
                        }
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    __syncwarp();
    if (warp == 1) tmem_free(tmem, 512);
    if (threadIdx.x == 0 && s_dead != 0u) atomicExch(&g_fp8_fault, 1u);
}

// ---- few rows -------------------------------------------------------------------------------------
// first warps: running sums (four, or eight that halve 64 columns between them); then one for loads, one for products
template <int BN> __host__ __device__ constexpr int few_sum_warps() { return BN >= 64 ? 8 : 4; }
template <int BN> __host__ __device__ constexpr int few_threads() { return 32 * (few_sum_warps<BN>() + 2); }
template <int BN> __host__ __device__ constexpr int few_per_sm() { return BN == 128 ? 1 : BN == 64 ? 2 : 3; }
constexpr int kFewW = 128;                    // rows of W in a tile
template <int BN> __host__ __device__ constexpr int few_buffers() { return 4; }    // accumulators: all CTAs of an SM stay within 512 columns

template <int BN> __host__ __device__ constexpr int few_stages() { return BN == 32 ? 3 : BN == 128 ? 5 : 4; }
template <int BN> __host__ __device__ constexpr size_t few_stage_bytes() { return size_t(kFewW) * kBlkK + size_t(BN) * kBlkK; }
template <int BN> __host__ __device__ constexpr size_t few_smem() {
    return 1024 + few_stages<BN>() * (few_stage_bytes<BN>() + BN * 4);
}
template <int BN> __host__ __device__ constexpr uint32_t few_cols() { return few_buffers<BN>() * BN; }

struct FewArgs {
    const float* sa; int64_t lds;
    const float* sw;
    void* out; int64_t ldo;
    int64_t M, N;
    int kblocks, mtiles, split;
};

template <int BN, int OUT>
__global__ void __launch_bounds__(few_threads<BN>(), few_per_sm<BN>())
k13_product_few(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapW, const FewArgs p) {
    constexpr int kSt = few_stages<BN>(), kFewBuffers = few_buffers<BN>(), EW = few_sum_warps<BN>(), kThr = few_threads<BN>();
    constexpr int kCols = BN * 4 / EW;                             // columns of each summing warp
    static_assert(few_per_sm<BN>() * few_cols<BN>() <= 512, "tensor memory");
    constexpr size_t kB = size_t(BN) * kBlkK;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* s_w = smem;                                            // [stage][128][128]
    uint8_t* s_x = s_w + kSt * size_t(kFewW) * kBlkK;              // [stage][BN][128]
    float* s_scale = reinterpret_cast<float*>(s_x + kSt * kB);     // [stage][BN]
    float* s_part = reinterpret_cast<float*>(smem);                // [BN][128], over the stages once they are done with
    __shared__ uint64_t full[kSt], empty[kSt], tfull[kFewBuffers], tempty[kFewBuffers];
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_dead;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.split;
    const int tile = blockIdx.x / p.split;
    const int64_t m0 = static_cast<int64_t>(tile % p.mtiles) * BN;
    const int64_t nb = tile / p.mtiles;
    const int64_t n0 = nb * kFewW;
    const int kb0 = static_cast<int>(static_cast<int64_t>(p.kblocks) * rank / p.split);
    const int kb1 = static_cast<int>(static_cast<int64_t>(p.kblocks) * (rank + 1) / p.split);
    const int count = kb1 - kb0;

    asm volatile("griddepcontrol.launch_dependents;");
    if (threadIdx.x == 0) {
        for (int i = 0; i < kSt; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], EW); }
        for (int i = 0; i < kFewBuffers; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], EW); }
        mbar_init_fence();
        s_dead = 0;
    }
    if (warp == EW + 1) tmem_alloc(&s_tmem, few_cols<BN>());
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    float acc[kCols];
    if (warp == EW) {
        const uint32_t sbytes = static_cast<uint32_t>(min(static_cast<int64_t>(BN), (p.M - m0 + 3) & ~int64_t(3))) * 4;
        bool ok = true;
        // the weights do not depend on the kernel before this one: their first tiles are on the way before its end
        const int head = min(kSt, count);
        if (elect_one())
            for (int i = 0; i < head; ++i) {
                mbar_expect_tx(&full[i], static_cast<uint32_t>(few_stage_bytes<BN>()) + sbytes);
                tile_load(s_w + i * size_t(kFewW) * kBlkK, &mapW, (kb0 + i) * kBlkK, static_cast<int32_t>(n0), &full[i]);
            }
        asm volatile("griddepcontrol.wait;" ::: "memory");
        int it = 0, s = 0;
        uint32_t round = 0;
        for (; it < count; ++it) {
            const int kb = kb0 + it;
            if (it >= head && !(ok = role_wait(&empty[s], round ^ 1u, &s_dead))) break;
            if (elect_one()) {
                if (it >= head) {
                    mbar_expect_tx(&full[s], static_cast<uint32_t>(few_stage_bytes<BN>()) + sbytes);
                    tile_load(s_w + s * size_t(kFewW) * kBlkK, &mapW, kb * kBlkK, static_cast<int32_t>(n0), &full[s]);
                }
                tile_load(s_x + s * kB, &mapA, kb * kBlkK, static_cast<int32_t>(m0), &full[s]);
                bulk_load(s_scale + s * BN, p.sa + kb * p.lds + m0, sbytes, &full[s]);
            }
            if (++s == kSt) { s = 0; round ^= 1u; }
        }
        if (!ok)                              // copies still in flight land before the CTA leaves
            for (int j = it > kSt ? it - kSt : 0; j < it; ++j)
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&full[j % kSt], (j / kSt) & 1); ++polls) {}
    } else if (warp == EW + 1) {
        const uint32_t idesc = idesc_fp8(kFewW, BN);
        const uint64_t desc_w = smem_desc_k128(s_w), desc_x = smem_desc_k128(s_x);
        bool ok = true;
        int it = 0, s = 0, b = 0;
        uint32_t round = 0, turn = 0;
        for (; it < count; ++it) {
            if (!(ok = role_wait(&full[s], round, &s_dead) && role_wait(&tempty[b], turn ^ 1u, &s_dead))) break;
            tc_fence_after();
            if (elect_one()) {
                mma_block(tmem + b * BN, desc_w + s * ((kFewW * kBlkK) >> 4), desc_x + s * (kB >> 4), idesc);
                tc_commit(&tfull[b]);         // (the stage is released by the epilogue, which waits for this)
            }
            if (++s == kSt) { s = 0; round ^= 1u; }
            if (++b == kFewBuffers) { b = 0; turn ^= 1u; }
        }
        if (!ok)
            for (int j = it > kFewBuffers ? it - kFewBuffers : 0; j < it; ++j)
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&tfull[j % kFewBuffers], (j / kFewBuffers) & 1); ++polls) {}
    } else {
        const int c0 = (warp >> 2) * kCols;
        const uint32_t taddr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + c0;
        const float* sw = p.sw + nb * p.kblocks;
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[i] = 0.0f;
        bool ok = true;
        float w = __ldg(sw + min(kb0, p.kblocks - 1));
        int s = 0, b = 0;
        uint32_t round = 0, turn = 0;
        for (int it = 0; it < count; ++it) {
            const float w_next = __ldg(sw + min(kb0 + it + 1, p.kblocks - 1));
            // the block's factors are ready before its product, so that little is left to do between that and the next
            if (!(ok = role_wait(&full[s], round, &s_dead))) break;
            const float4* sc = reinterpret_cast<const float4*>(s_scale + s * BN + c0);
            float f[kCols];
#pragma unroll
            for (int i = 0; i < kCols / 4; ++i) {
                const float4 t = sc[i];
                f[4 * i] = __fmul_rn(t.x, w); f[4 * i + 1] = __fmul_rn(t.y, w);
                f[4 * i + 2] = __fmul_rn(t.z, w); f[4 * i + 3] = __fmul_rn(t.w, w);
            }
            if (!(ok = role_wait(&tfull[b], turn, &s_dead))) break;
            tc_fence_after();
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[s]);    // the products have read the stage, and this warp its scales
#pragma unroll
            for (int c = 0; c < kCols / 16; ++c) {
                float v[16];
                tmem_ld16(taddr + b * BN + c * 16, v);
                tmem_ld_wait(v);
                if (c + 1 == kCols / 16) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&tempty[b]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[c * 16 + i] = __fmaf_rn(v[i], f[c * 16 + i], acc[c * 16 + i]);
            }
            w = w_next;
            if (++s == kSt) { s = 0; round ^= 1u; }
            if (++b == kFewBuffers) { b = 0; turn ^= 1u; }
        }
    }
    // every product of this CTA has completed (the last buffers were waited for), so the stages may be written over
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    __syncwarp();
    if (warp == EW + 1) tmem_free(tmem, few_cols<BN>());
    if (warp < EW) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) s_part[((warp >> 2) * kCols + j) * kFewW + (threadIdx.x & 127)] = acc[j];
    }
    cluster_sync_all();
    const int rows = static_cast<int>(min(static_cast<int64_t>(BN), p.M - m0));
    const int j0 = rows * rank / p.split, j1 = rows * (rank + 1) / p.split;
    for (int idx = threadIdx.x; idx < (j1 - j0) * kFewW; idx += kThr) {
        const int j = j0 + idx / kFewW, n = idx % kFewW;
        const uint32_t at = smem_u32(s_part + j * kFewW + n);
        float sum = 0.0f;
        for (int r = 0; r < p.split; ++r) sum = __fadd_rn(sum, ld_cluster(at, r));
        if (n0 + n < p.N) {
            const int64_t o = (m0 + j) * p.ldo + n0 + n;
            if constexpr (OUT == CQ_F32) static_cast<float*>(p.out)[o] = sum;
            else static_cast<uint16_t*>(p.out)[o] = to16<OUT>(sum);
        }
    }
    cluster_sync_all();                       // nobody leaves while its partial sums are being read
    if (threadIdx.x == 0 && s_dead != 0u) atomicExch(&g_fp8_fault, 1u);
}

// ---- host ---------------------------------------------------------------------------------------------
bool make_byte_map(CUtensorMap* map, const void* base, uint64_t bytes, uint64_t rows, uint64_t pitch,
                   uint32_t box_bytes, uint32_t box_rows, CUtensorMapSwizzle swizzle) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Encode> known{nullptr};
    Encode encode = known.load(std::memory_order_acquire);
    if (encode == nullptr) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess || fn == nullptr) {
            cudaGetLastError();
            return false;
        }
        encode = reinterpret_cast<Encode>(fn);
        known.store(encode, std::memory_order_release);
    }
    const cuuint64_t dims[2] = {bytes, rows}, strides[1] = {pitch};
    const cuuint32_t box[2] = {box_bytes, box_rows}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int fp8_stage_fault(unsigned int* fault_host) {
    return cudaMemcpyFromSymbol(fault_host, g_fp8_fault, sizeof(unsigned int)) == cudaSuccess ? CQ_OK : CQ_ERR_CUDA;
}

template <int BN, int OUT>
static int launch_few(const CUtensorMap& a, const CUtensorMap& w, FewArgs p, int64_t ntiles, bool dependent, cudaStream_t st) {
    static thread_local LaunchMemo memo;
    if (resident_ctas(k13_product_few<BN, OUT>, few_threads<BN>(), few_smem<BN>(), few_smem<BN>(), memo) < 1) return CQ_ERR_CUDA;
    // As many parts of the contraction (up to a portable cluster's eight CTAs, two blocks each at least) as one round of
    // resident CTAs takes, an eighth left for what clusters cannot fill: a second, partial round costs as much as the first
    // (1 x 8192 x 8192, 64 tiles: 27.4 us with 1 part, 16.4 with 4, 15.2 with 5 or 6, 18.7 with 8).
    const int64_t tiles = p.mtiles * ntiles;
    int64_t split = int64_t(few_per_sm<BN>()) * sm_count() * 7 / 8 / tiles;
    split = split > 8 ? 8 : split;
    split = split > p.kblocks / 2 ? p.kblocks / 2 : split;
    p.split = static_cast<int>(split < 1 ? 1 : split);
    return launch_ex(k13_product_few<BN, OUT>, dim3(static_cast<unsigned>(tiles * p.split)), few_threads<BN>(), few_smem<BN>(), st, p.split,
                     dependent, a, w, p);
}

template <int BN, int OUT, bool SPLIT>
static int launch_main(const CUtensorMap& a, const CUtensorMap& w, const MainArgs& p, bool dependent, cudaStream_t st) {
    static thread_local LaunchMemo memo;
    if (resident_ctas(k12_product<BN, OUT, SPLIT>, kMainThreads, main_smem<BN>(), main_smem<BN>(), memo) < 1) return CQ_ERR_CUDA;
    const int64_t tiles = static_cast<int64_t>(p.mtiles) * p.ntiles;
    const int sms = sm_count();
    const unsigned grid = static_cast<unsigned>(SPLIT ? 2 * tiles : tiles < sms ? tiles : sms);
    return launch_ex(k12_product<BN, OUT, SPLIT>, dim3(grid), kMainThreads, main_smem<BN>(), st, SPLIT ? 2 : 1, dependent, a, w, p);
}

template <int OUT>
static int launch_product(const void* A, int64_t lda, const float* sa, int64_t lds, const void* W, int64_t ldw, const float* sw,
                          int64_t M, int64_t N, int64_t K, void* out, int64_t ldo, bool dependent, cudaStream_t st) {
    const int kblocks = static_cast<int>((K + kBlkK - 1) / kBlkK);
    const int sms = sm_count();
    CUtensorMap mapA, mapW;
    // So few tiles of 128 x 128 that a contraction worth splitting can be split in four or more go the other way too
    // (68 x 3972 x 281, 3 tiles: 16.3 against 9.8 us; split in two that way it loses: 128 x 8192 x 8192, 64 tiles: 27 against 36 us).
    const bool split_up = 5 * ((M + 127) / 128) * ((N + 127) / 128) <= sms && kblocks >= 16;
    if (M > 64 && !split_up) {
        const int64_t mt = (M + kTileM - 1) / kTileM, wide = mt * ((N + 255) / 256), narrow = mt * ((N + 127) / 128);
        // rounds of all SMs times the cost of a block in a tile of either width
        const bool use_wide = ((wide + sms - 1) / sms) * 3 < ((narrow + sms - 1) / sms) * 2;
        const int bn = use_wide ? 256 : 128;
        if (mt * ((N + bn - 1) / bn) > (int64_t(1) << 40)) return CQ_ERR_SHAPE;
        if (!make_byte_map(&mapA, A, K, M, lda, kBlkK, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
            !make_byte_map(&mapW, W, K, N, ldw, kBlkK, bn, CU_TENSOR_MAP_SWIZZLE_128B)) return CQ_ERR_CUDA;
        const MainArgs p{sa, lds, sw, out, ldo, M, N, kblocks, static_cast<int>(mt), static_cast<int>((N + bn - 1) / bn)};
        // Narrow tiles for less than half of the SMs (an eighth left for what clusters cannot fill) split the contraction in two:
        // 128 x 8192 x 8192 (64 tiles) 26.4 -> 19.5 us, 777 x 2060 x 1003 (56 tiles, 17 blocks) 12.5 -> 11.3; below 16 blocks the join
        // takes what it gives (128 x 1600 x 8192, 13 blocks: 8.9 and 9.0).
        if (16 * narrow <= 7 * sms && kblocks >= 16) return launch_main<128, OUT, true>(mapA, mapW, p, dependent, st);
        return use_wide ? launch_main<256, OUT, false>(mapA, mapW, p, dependent, st)
                        : launch_main<128, OUT, false>(mapA, mapW, p, dependent, st);
    }
    const int bn = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
    const int mtiles = static_cast<int>((M + bn - 1) / bn);
    const int64_t ntiles = (N + kFewW - 1) / kFewW;
    if (ntiles * mtiles > (1 << 26)) return CQ_ERR_SHAPE;
    if (!make_byte_map(&mapA, A, K, M, lda, kBlkK, bn, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_byte_map(&mapW, W, K, N, ldw, kBlkK, kFewW, CU_TENSOR_MAP_SWIZZLE_128B)) return CQ_ERR_CUDA;
    const FewArgs p{sa, lds, sw, out, ldo, M, N, kblocks, mtiles, 1};
    switch (bn) {
        case 16: return launch_few<16, OUT>(mapA, mapW, p, ntiles, dependent, st);
        case 32: return launch_few<32, OUT>(mapA, mapW, p, ntiles, dependent, st);
        case 64: return launch_few<64, OUT>(mapA, mapW, p, ntiles, dependent, st);
        default: return launch_few<128, OUT>(mapA, mapW, p, ntiles, dependent, st);
    }
}

static int fp8_matmul_impl(const void* A, int64_t lda, const float* sa, int64_t lds, const void* W, int64_t ldw, const float* sw,
                           int64_t M, int64_t N, int64_t K, void* out, int out_dtype, int64_t ldo, bool dependent, cudaStream_t st) {
    if (M < 0 || N < 0 || K < 0 || lda < K || ldw < K || ldo < N || lds < M) return CQ_ERR_SHAPE;
    if (M > (int64_t(1) << 31) - 1024 || N > (int64_t(1) << 31) - 1024 || K > (int64_t(1) << 31) - 1024) return CQ_ERR_SHAPE;
    if (out_dtype != CQ_F16 && out_dtype != CQ_BF16 && out_dtype != CQ_F32) return CQ_ERR_DTYPE;
    if (M == 0 || N == 0) return CQ_OK;
    const size_t elem = out_dtype == CQ_F32 ? 4 : 2;
    if (out == nullptr) return CQ_ERR_NULL;
    if (!ptr_aligned(out, elem)) return CQ_ERR_ALIGN;
    if (K == 0)                                                     // an empty sum
        return cudaMemset2DAsync(out, ldo * elem, 0, N * elem, M, st) == cudaSuccess ? CQ_OK : CQ_ERR_CUDA;
    if (A == nullptr || W == nullptr || sa == nullptr || sw == nullptr) return CQ_ERR_NULL;
    if (!ptr_aligned(A, 16) || !ptr_aligned(W, 16) || lda % 16 != 0 || ldw % 16 != 0 || !ptr_aligned(sa, 16) || lds % 4 != 0 ||
        !ptr_aligned(sw, 4)) return CQ_ERR_ALIGN;
    if (out_dtype == CQ_F32) return launch_product<CQ_F32>(A, lda, sa, lds, W, ldw, sw, M, N, K, out, ldo, dependent, st);
    if (out_dtype == CQ_F16) return launch_product<CQ_F16>(A, lda, sa, lds, W, ldw, sw, M, N, K, out, ldo, dependent, st);
    return launch_product<CQ_BF16>(A, lda, sa, lds, W, ldw, sw, M, N, K, out, ldo, dependent, st);
}

int fp8_quantize_act_impl(const void* X, int dtype, int64_t T, int64_t K, int64_t ld, void* codes, int64_t ldc,
                          float* scale, int64_t lds, cudaStream_t st);

static int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
static int64_t up4(int64_t v) { return (v + 3) / 4 * 4; }
static size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace cq

extern "C" {

int cq_fp8_matmul(const void* A, int64_t lda, const float* a_scale, int64_t lds, const void* W, int64_t ldw, const float* w_scale,
                  int64_t M, int64_t N, int64_t K, void* out, int out_dtype, int64_t ldo, void* stream) {
    return cq::fp8_matmul_impl(A, lda, a_scale, lds, W, ldw, w_scale, M, N, K, out, out_dtype, ldo, false,
                               static_cast<cudaStream_t>(stream));
}

size_t cq_fp8_linear_workspace_bytes(int64_t M, int64_t K) {
    if (M < 0 || K < 0) return 0;
    return cq::up256(static_cast<size_t>(M) * cq::up16(K)) + cq::up256(sizeof(float) * cq::up4(M) * ((K + 127) / 128)) + 256;
}

int cq_fp8_linear(const void* X, int dtype, int64_t M, int64_t K, int64_t ldx, const void* W, int64_t ldw, const float* w_scale,
                  int64_t N, void* out, int out_dtype, int64_t ldo, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace cq;
    const int rc = check_matrix(X, dtype, M, K, ldx);
    if (rc != CQ_OK) return rc;
    if (M == 0 || N == 0 || K == 0)                                  // nothing to quantize; the product checks the rest
        return fp8_matmul_impl(nullptr, up16(K), nullptr, up4(M), W, ldw, w_scale, M, N, K, out, out_dtype, ldo, false,
                               static_cast<cudaStream_t>(stream));
    if (workspace == nullptr || !ptr_aligned(workspace, 256) || workspace_bytes < cq_fp8_linear_workspace_bytes(M, K))
        return CQ_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // every argument of the product is checked before the quantizer is launched
    if (N < 0 || ldw < K || ldo < N || N > (int64_t(1) << 31) - 1024) return CQ_ERR_SHAPE;
    if (out_dtype != CQ_F16 && out_dtype != CQ_BF16 && out_dtype != CQ_F32) return CQ_ERR_DTYPE;
    if (W == nullptr || w_scale == nullptr || out == nullptr) return CQ_ERR_NULL;
    if (!ptr_aligned(W, 16) || ldw % 16 != 0 || !ptr_aligned(w_scale, 4) || !ptr_aligned(out, out_dtype == CQ_F32 ? 4 : 2)) return CQ_ERR_ALIGN;
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    float* scale = reinterpret_cast<float*>(codes + up256(static_cast<size_t>(M) * up16(K)));
    const int rq = fp8_quantize_act_impl(X, dtype, M, K, ldx, codes, up16(K), scale, up4(M), st);
    if (rq != CQ_OK) return rq;
    return fp8_matmul_impl(codes, up16(K), scale, up4(M), W, ldw, w_scale, M, N, K, out, out_dtype, ldo, !tuning_no_pdl(), st);
}

}  // extern "C"
