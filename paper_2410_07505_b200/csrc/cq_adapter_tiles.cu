// Low-rank adapters for many tokens (cq_adapter.cu has the formula and the kernels for few): both products on tcgen05, everything
// that is large through TMA.
//
// The tokens are taken in tiles of 128 neighbours.  A prompt's tokens share an adapter, so a tile has one or two; one that has more
// (tokens of many requests) costs a product for each, in which the rows of the others are computed in vain, and nothing else.
//   k27  h = A x: a tile's x against the rows of up to 128 / R adapters side by side, so that x is read once for them; the contraction
//        is split over a cluster and joined through distributed shared memory in rank order
//   k28  out = y + B h: persistent over 128 x 256-byte tiles of y; those stream through a ring in shared memory in which the
//        epilogue adds the product to the rows that have the adapter at hand.  Bound by HBM (y in, out out).  Rows that no tensor map takes
//        are brought and taken away by the warps of the epilogue, bound by their instructions: 2223 x 17853, rank 64, 86 us, 35 of 17856 columns
// Measured (operands not in L2): 4096 x 8192 x 28672, rank 64, both 112 us (556 MB, 5.0 TB/s of 6.6 of a copy), k28 by itself 83 us (485 MB, 5.8 TB/s).  A tile of
// many adapters is bound by the round of signals for each: 1024 x 8192 x 8192 with 55 of 64 adapters in every tile, rank 16, 190 us, 0.45 us an
// adapter and tile of columns in k28, of which neither its rows of B nor its epilogue are more than 15 %.
#include "cq_adapter.cuh"

#include <algorithm>

namespace cq {

__device__ unsigned int g_adapter_fault = 0;  // set if a bounded wait ever gave up

__device__ __forceinline__ bool agreed_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* dead) {
    return __all_sync(0xFFFFFFFFu, role_wait(bar, parity, dead)) != 0;
}
__device__ __forceinline__ void tile_store(const CUtensorMap* map, const void* src_smem, int32_t x, int32_t y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 :: "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(src_smem)) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t addr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]) :: "memory");
}

// ---- h = A x --------------------------------------------------------------------------------------------------------
constexpr int kInThreads = 256;               // warp 0: loads, warp 1: products, warps 4..7: rows of the sums
constexpr int kInCols = 128;                  // rows of A (of several adapters) side by side
constexpr int kInMaxStages = 5;
constexpr size_t kXTile = size_t(kTileTokens) * 128, kATile = size_t(kInCols) * 128;

constexpr int in_stages(int R) { return R <= 64 ? kInMaxStages : 4; }
constexpr size_t in_smem(int R) { return 1024 + in_stages(R) * (kXTile + kATile) + size_t(kTileTokens) * (R + 1) * 4; }
// Every rank is launched with this much, which leaves no room for a second block either way: what the runtime says of the kernel is then
// asked once, whatever the ranks of a layer's adapters are.
constexpr size_t kInSmem = in_smem(64) > in_smem(kMaxRank) ? in_smem(64) : in_smem(kMaxRank);

template <int DT>
__global__ void __launch_bounds__(kInThreads, 1)
k27_adapter_in_tiles(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapA, const AdapterArgs p, int stages) {
    extern __shared__ __align__(1024) uint8_t smem[];           // (behind the static part: moved to a 1024-byte boundary below)
    __shared__ uint64_t full[kInMaxStages], empty[kInMaxStages], d_full[2], d_empty[2], drain;
    __shared__ TileSort s_sort;
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_dead;
    uint8_t* s_x = smem + ((1024u - (smem_u32(smem) & 1023u)) & 1023u);
    uint8_t* s_a = s_x + stages * kXTile;
    float* s_h = reinterpret_cast<float*>(s_a + stages * kATile);
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < kInMaxStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&d_full[i], 1); mbar_init(&d_empty[i], 4); }
        mbar_init(&drain, 1);
        mbar_init_fence();
        s_dead = 0;
        prefetch_map(&mapX);
        prefetch_map(&mapA);
    }
    if (warp == 1) tmem_alloc(&s_tmem, 2 * kInCols);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t t0 = static_cast<int64_t>(blockIdx.y) * kTileTokens;
    const int count = sort_tile(p, t0, s_sort, blockIdx.x == 0 && blockIdx.z == 0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;");  // (behind the allocation: see tmem_alloc)
    const uint32_t tmem = s_tmem;
    const int rank = blockIdx.x, ranks = gridDim.x;
    const int kblocks = static_cast<int>((p.K + 63) / 64), kb0 = static_cast<int>(static_cast<int64_t>(kblocks) * rank / ranks),
              kb1 = static_cast<int>(static_cast<int64_t>(kblocks) * (rank + 1) / ranks);
    const int per = kInCols / p.R, groups = (count + per - 1) / per, gr0 = blockIdx.z, turns = gridDim.z;      // this cluster's: gr0, gr0 + turns ..
    if (warp == 0) {
        int s = 0;
        uint32_t round = 0;
        int issued = 0;
        bool ok = true;
        for (int gr = gr0; ok && gr < groups; gr += turns) {
            const int n = min(per, count - gr * per);
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!(ok = agreed_wait(&empty[s], round ^ 1u, &s_dead))) break;
                if (elect_one()) {
                    mbar_expect_tx(&full[s], static_cast<uint32_t>(kXTile) + n * p.R * 128);
                    tile_load(s_x + s * kXTile, &mapX, kb * 128, static_cast<int32_t>(t0), &full[s]);
                    for (int i = 0; i < n; ++i)
                        tile_load(s_a + s * kATile + i * p.R * 128, &mapA, kb * 128, s_sort.adapter[gr * per + i] * p.R, &full[s]);
                }
                issued = min(issued + 1, stages);
                if (++s == stages) { s = 0; round ^= 1u; }
            }
        }
        if (!ok)                              // copies still in flight land before the CTA leaves
            for (; issued > 0; --issued) {
                if (--s < 0) { s = stages - 1; round ^= 1u; }
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&full[s], round); ++polls) {}
            }
    } else if (warp == 1) {
        const uint64_t desc_x = smem_desc_k128(s_x), desc_a = smem_desc_k128(s_a);
        int s = 0;
        uint32_t round = 0;
        bool ok = true;
        for (int gr = gr0, n = 0; ok && gr < groups; gr += turns, ++n) {
            const int b = n & 1, cols = (min(per, count - gr * per) * p.R + 15) & ~15;
            const uint32_t idesc = idesc_f16<DT>(128, cols, false);
            if (!(ok = agreed_wait(&d_empty[b], ((n >> 1) & 1) ^ 1u, &s_dead))) break;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!(ok = agreed_wait(&full[s], round, &s_dead))) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_f16(tmem + b * kInCols, desc_x + ((s * kXTile) >> 4) + 2 * k, desc_a + ((s * kATile) >> 4) + 2 * k, idesc, kb > kb0 || k > 0);
                    tc_commit(&empty[s]);
                    if (kb + 1 == kb1) tc_commit(&d_full[b]);
                }
                if (++s == stages) { s = 0; round ^= 1u; }
            }
        }
        if (!ok) {                            // products in flight end before the CTA leaves
            __syncwarp();
            if (elect_one()) tc_commit(&drain);
            for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&drain, 0); ++polls) {}
        }
    } else if (warp >= 4) {
        const int token = (warp & 3) * 32 + lane;
        const int mine = s_sort.slot[token];
        const uint32_t at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        float* h = s_h + token * (p.R + 1);
        bool ok = true;
        for (int gr = gr0, n = 0; ok && gr < groups; gr += turns, ++n) {
            const int b = n & 1, have = min(per, count - gr * per);
            if (!(ok = agreed_wait(&d_full[b], (n >> 1) & 1, &s_dead))) break;
            tc_fence_after();
            for (int i = 0; i < have; ++i) {
                const bool here = mine == gr * per + i;
                if (!__any_sync(0xFFFFFFFFu, here)) continue;
                for (int c = 0; c < p.R; c += 8) {
                    float v[8];
                    __syncwarp();
                    tmem_ld8(at + b * kInCols + i * p.R + c, v);
                    if (here) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) h[c + k] = v[k];
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&d_empty[b]);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    __syncwarp();
    if (warp == 1) tmem_free(tmem, 2 * kInCols);
    __syncwarp();
    if (ranks > 1) cluster_barrier();
    for (int m = rank + warp * ranks; m < kTileTokens; m += ranks * (kInThreads / 32))
        if (s_sort.idx[m] >= 0 && s_sort.slot[m] / per % turns == gr0) finish_token<DT>(p, s_h + m * (p.R + 1), ranks, t0 + m, s_sort.idx[m]);
    __syncwarp();
    if (ranks > 1) cluster_barrier();         // nobody leaves while its sums are being read
    if (tid == 0 && s_dead != 0u) atomicExch(&g_adapter_fault, 1u);
}

// ---- out = y + B h ---------------------------------------------------------------------------------------------------
constexpr int kOutThreads = 384;              // warp 0: loads, warp 1: products, warp 2: stores, warps 4..11: y + the product
constexpr size_t kYTile = size_t(kTileTokens) * 256;
constexpr int kOutBuffers = 4;                // accumulators

template <int HB> __host__ __device__ constexpr int y_stages() { return HB == 1 ? 4 : 3; }       // HB: halves of 64 of the rank
template <int HB> __host__ __device__ constexpr int b_stages() { return HB == 1 ? 3 : 2; }
template <int YT> __host__ __device__ constexpr int out_cols() { return YT == CQ_F32 ? 64 : 128; }
template <int HB, int YT> __host__ __device__ constexpr size_t b_tile() { return size_t(HB) * out_cols<YT>() * 128; }
template <int HB, int YT> __host__ __device__ constexpr size_t out_smem() {
    return 2 * HB * kXTile + y_stages<HB>() * kYTile + b_stages<HB>() * b_tile<HB, YT>() + 512;
}

// Items of this CTA: first, first + step .. below end.  The columns of tiles are the faster of an item's two places.
struct OutItem { int64_t first, end; int step, cols; };
__device__ __forceinline__ OutItem out_items(const AdapterArgs& p, int width, int group) {
    const int cols = static_cast<int>((p.N + width - 1) / width);
    const int64_t items = (p.T + kTileTokens - 1) / kTileTokens * cols;
    const int at = blockIdx.x / group, groups = gridDim.x / group;
    return {items * at / groups + blockIdx.x % group, items * (at + 1) / groups, group, cols};
}

// y + f v, rounded once, for half a row of a tile in shared memory
template <int YT, int Q>
__device__ __forceinline__ void add_to_row(uint8_t* y, int row, const float (&v)[Q][32], float f) {
    uint4 w[8];                                                 // all at once: one latency instead of eight
#pragma unroll
    for (int c = 0; c < 8; ++c) w[c] = *reinterpret_cast<const uint4*>(y + ((c ^ (row & 7)) << 4));
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t r[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (YT == CQ_F32) {
                o[i] = __float_as_uint(__fmaf_rn(v[0][4 * c + i], f, __uint_as_float(r[i])));
            } else {
                const float2 b = unpack16x2<YT>(r[i]);
                const int e = 8 * c + 2 * i;
                o[i] = pack16x2<YT>(__fmaf_rn(v[e >> 5][e & 31], f, b.x), __fmaf_rn(v[e >> 5][(e & 31) + 1], f, b.y));
            }
        }
        *reinterpret_cast<uint4*>(y + ((c ^ (row & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// Rows of y (and out) that begin anywhere, which no tensor map takes: a warp has sixteen rows of a tile, 64 words of a row in two registers a lane.
// A row that begins in the middle of a word is moved by half a word on its way into shared memory and out of it; its last element, in a
// word of its own, is in lane `row` of `edge`.
struct LooseRows { uint32_t w[16][2]; uint32_t edge; };

template <int YT>
__device__ __forceinline__ int begins_odd(const void* base, int64_t at) {
    return YT == CQ_F32 ? 0 : static_cast<int>((reinterpret_cast<uintptr_t>(base) >> 1) + at) & 1;
}
template <int YT>
__device__ __forceinline__ void fetch_rows(const AdapterArgs& p, int64_t t0, int64_t col, LooseRows& v) {
    constexpr int kPer = YT == CQ_F32 ? 1 : 2, kElem = 4 / kPer, CT = out_cols<YT>();
    const int lane = threadIdx.x & 31, left = static_cast<int>(min(p.N - col, static_cast<int64_t>(CT)));
    const uint8_t* y = static_cast<const uint8_t*>(p.y);
    if (left == CT && t0 + 16 <= p.T) {       // all there: a load and an addition for each word
        const uint8_t* at = y + (t0 * p.ldy + col) * kElem + 4 * lane;
        const int64_t pitch = p.ldy * kElem;
        const int first = begins_odd<YT>(y, t0 * p.ldy + col), turns = begins_odd<YT>(nullptr, p.ldy);
#pragma unroll
        for (int i = 0; i < 16; ++i, at += pitch) {
            const uint32_t* word = reinterpret_cast<const uint32_t*>(YT == CQ_F32 ? at : at - 2 * ((first + i * turns) & 1));
            v.w[i][0] = __ldcg(word);
            v.w[i][1] = __ldcg(word + 32);
        }
    } else
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t at = (t0 + i) * p.ldy + col;
        const int odd = begins_odd<YT>(y, at);
        const uint32_t* words = reinterpret_cast<const uint32_t*>(y + (at - odd) * kElem);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int q = lane + 32 * h;
            v.w[i][h] = t0 + i < p.T && kPer * q - odd < left ? __ldcg(words + q) : 0u;      // (a word that holds an element of the tile)
        }
    }
    v.edge = 0;
    if constexpr (YT != CQ_F32) {
        const int64_t at = (t0 + lane) * p.ldy + col;
        if (lane < 16 && t0 + lane < p.T && left == CT && begins_odd<YT>(y, at) != 0) v.edge = __ldcg(reinterpret_cast<const uint16_t*>(y) + at + CT - 1);
    }
}
__device__ __forceinline__ uint32_t* loose_word(uint8_t* tile, int row, int h) {
    const int lane = threadIdx.x & 31;
    return reinterpret_cast<uint32_t*>(tile + h * kXTile + row * 128 + (((lane >> 2) ^ (row & 7)) << 4)) + (lane & 3);
}
template <int YT>
__device__ __forceinline__ void rows_to_tile(const AdapterArgs& p, int64_t t0, int64_t col, const LooseRows& v, uint8_t* tile, int row0) {
    const int lane = threadIdx.x & 31, first = begins_odd<YT>(p.y, t0 * p.ldy + col), turns = begins_odd<YT>(nullptr, p.ldy);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        uint32_t a = v.w[i][0], b = v.w[i][1];
        if (((first + i * turns) & 1) != 0) { // (the same for the whole warp)
            uint32_t next_a = __shfl_down_sync(0xFFFFFFFFu, a, 1), next_b = __shfl_down_sync(0xFFFFFFFFu, b, 1);
            const uint32_t first_b = __shfl_sync(0xFFFFFFFFu, b, 0), edge = __shfl_sync(0xFFFFFFFFu, v.edge, i);
            if (lane == 31) { next_a = first_b; next_b = edge; }
            a = __funnelshift_r(a, next_a, 16);
            b = __funnelshift_r(b, next_b, 16);
        }
        *loose_word(tile, row0 + i, 0) = a;
        *loose_word(tile, row0 + i, 1) = b;
    }
}
template <int YT>
__device__ __forceinline__ void tile_to_rows(const AdapterArgs& p, int64_t t0, int64_t col, uint8_t* tile, int row0) {
    constexpr int kPer = YT == CQ_F32 ? 1 : 2, kElem = 4 / kPer, CT = out_cols<YT>();
    const int lane = threadIdx.x & 31, left = static_cast<int>(min(p.N - col, static_cast<int64_t>(CT)));
    uint8_t* out = static_cast<uint8_t*>(p.out);
    if (left == CT && t0 + 16 <= p.T) {
        uint8_t* at = out + (t0 * p.ldo + col) * kElem + 4 * lane;
        const int64_t pitch = p.ldo * kElem;
        const int first = begins_odd<YT>(out, t0 * p.ldo + col), turns = begins_odd<YT>(nullptr, p.ldo);
#pragma unroll
        for (int i = 0; i < 16; ++i, at += pitch) {
            uint32_t a = *loose_word(tile, row0 + i, 0), b = *loose_word(tile, row0 + i, 1);
            if (YT != CQ_F32 && ((first + i * turns) & 1) != 0) {
                uint16_t* halves = reinterpret_cast<uint16_t*>(at);
                uint32_t before_a = __shfl_up_sync(0xFFFFFFFFu, a, 1), before_b = __shfl_up_sync(0xFFFFFFFFu, b, 1);
                const uint32_t last_a = __shfl_sync(0xFFFFFFFFu, a, 31);
                if (lane == 0) before_b = last_a;
                uint32_t* words = reinterpret_cast<uint32_t*>(at - 2);
                if (lane == 0) halves[0] = static_cast<uint16_t>(a);
                else words[0] = __funnelshift_r(before_a, a, 16);
                words[32] = __funnelshift_r(before_b, b, 16);
                if (lane == 31) halves[65] = static_cast<uint16_t>(b >> 16);    // (of element 62 on: the 127th)
            } else {
                reinterpret_cast<uint32_t*>(at)[0] = a;
                reinterpret_cast<uint32_t*>(at)[32] = b;
            }
        }
        return;
    }
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
        if (t0 + i >= p.T) break;
        const int64_t at = (t0 + i) * p.ldo + col;
        const int odd = begins_odd<YT>(out, at);
        uint32_t w[2] = {*loose_word(tile, row0 + i, 0), *loose_word(tile, row0 + i, 1)};
        if (odd != 0) {
            if (lane == 31 && left == CT) reinterpret_cast<uint16_t*>(out)[at + CT - 1] = static_cast<uint16_t>(w[1] >> 16);
            uint32_t before_a = __shfl_up_sync(0xFFFFFFFFu, w[0], 1), before_b = __shfl_up_sync(0xFFFFFFFFu, w[1], 1);
            const uint32_t last_a = __shfl_sync(0xFFFFFFFFu, w[0], 31);
            if (lane == 0) before_b = last_a;
            w[0] = __funnelshift_r(before_a, w[0], 16);
            w[1] = __funnelshift_r(before_b, w[1], 16);
        }
        uint32_t* words = reinterpret_cast<uint32_t*>(out + (at - odd) * kElem);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int q = lane + 32 * h, e = kPer * q - odd;    // the word's first element
            if (e >= 0 && e + kPer <= left) {
                words[q] = w[h];
            } else if constexpr (kPer == 2) {
                uint16_t* halves = reinterpret_cast<uint16_t*>(words + q);
                if (e >= 0 && e < left) halves[0] = static_cast<uint16_t>(w[h]);
                if (e + 1 >= 0 && e + 1 < left) halves[1] = static_cast<uint16_t>(w[h] >> 16);
            }
        }
    }
}

template <int HB, int DT, int YT, bool LOOSE>                  // LOOSE: rows of y and out begin anywhere
__global__ void __launch_bounds__(kOutThreads, 1)
k28_adapter_out_tiles(const __grid_constant__ CUtensorMap mapHigh, const __grid_constant__ CUtensorMap mapLow, const __grid_constant__ CUtensorMap mapB,
                      const __grid_constant__ CUtensorMap mapY, const __grid_constant__ CUtensorMap mapOut, const AdapterArgs p, int group) {
    constexpr int SY = y_stages<HB>(), SB = b_stages<HB>(), CT = out_cols<YT>();
    constexpr size_t kB = b_tile<HB, YT>();
    // No static shared memory, so that the dynamic part starts on the 1024-byte boundary that the swizzle wants.
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* s_h = smem;                                        // [high, low][half of the rank][128 tokens][128 bytes]
    uint8_t* s_y = s_h + 2 * HB * kXTile;                       // [stage][half of the columns][128 tokens][128 bytes]
    uint8_t* s_b = s_y + SY * kYTile;                           // [stage][half of the rank][CT columns][128 bytes]
    uint64_t* y_full = reinterpret_cast<uint64_t*>(s_b + SB * kB);
    uint64_t* y_empty = y_full + SY;
    uint64_t* o_full = y_empty + SY;
    uint64_t* b_full = o_full + SY;
    uint64_t* b_empty = b_full + SB;
    uint64_t* d_full = b_empty + SB;
    uint64_t* d_empty = d_full + kOutBuffers;
    uint64_t* h_full = d_empty + kOutBuffers;
    uint64_t* h_empty = h_full + 1;
    uint64_t* drain = h_empty + 1;
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(drain + 1);
    volatile uint32_t& s_dead = *(reinterpret_cast<volatile uint32_t*>(drain + 1) + 1);
    static_assert((3 * SY + 2 * SB + 2 * kOutBuffers + 3) * 8 + 8 <= 512, "barriers");
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) {
        if ((smem_u32(smem) & 1023u) != 0u) atomicExch(&g_adapter_fault, 1u);      // cannot be: see above
        for (int i = 0; i < SY; ++i) { mbar_init(&y_full[i], 1); mbar_init(&y_empty[i], 1); mbar_init(&o_full[i], 8); }
        for (int i = 0; i < SB; ++i) { mbar_init(&b_full[i], 1); mbar_init(&b_empty[i], 1); }
        for (int i = 0; i < kOutBuffers; ++i) { mbar_init(&d_full[i], 1); mbar_init(&d_empty[i], 8); }
        mbar_init(h_full, 1);
        mbar_init(h_empty, 1);
        mbar_init(drain, 1);
        mbar_init_fence();
        s_dead = 0;
        prefetch_map(&mapHigh);
        prefetch_map(&mapLow);
        prefetch_map(&mapB);
        if (!LOOSE) { prefetch_map(&mapY); prefetch_map(&mapOut); }
    }
    if (warp == 1) tmem_alloc(&s_tmem, kOutBuffers * CT);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;");  // (behind the allocation: see tmem_alloc)
    const uint32_t tmem = s_tmem;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const OutItem work = out_items(p, CT, group);

    if (warp == 0) {
        int ys = 0, bs = 0, y_issued = 0, b_issued = 0, count = 0;
        uint32_t y_round = 0, b_round = 0, h_round = 0;
        int64_t tile = -1;
        bool ok = true, h_open = false;
        const int* info = p.info;
        for (int64_t it = work.first; ok && it < work.end; it += work.step) {
            const int64_t tl = it / work.cols;
            const int col = static_cast<int>(it - tl * work.cols) * CT;
            const int32_t t0 = static_cast<int32_t>(tl) * kTileTokens;
            if constexpr (!LOOSE) {
                if (!(ok = agreed_wait(&y_empty[ys], y_round ^ 1u, &s_dead))) break;
                if (elect_one()) {
                    mbar_expect_tx(&y_full[ys], static_cast<uint32_t>(kYTile));
                    tile_load(s_y + ys * kYTile, &mapY, col * (YT == CQ_F32 ? 4 : 2), t0, &y_full[ys]);
                    tile_load(s_y + ys * kYTile + kXTile, &mapY, col * (YT == CQ_F32 ? 4 : 2) + 128, t0, &y_full[ys]);
                }
                y_issued = min(y_issued + 1, SY);
                if (++ys == SY) { ys = 0; y_round ^= 1u; }
            }
            if (tl != tile) {
                tile = tl;
                info = p.info + tl * kTileInfo;
                count = __ldcg(info);
                if (count > 0) {
                    if (!(ok = agreed_wait(h_empty, h_round ^ 1u, &s_dead))) break;
                    if (elect_one()) {
                        mbar_expect_tx(h_full, static_cast<uint32_t>(2 * HB * kXTile));
#pragma unroll
                        for (int h = 0; h < HB; ++h) {
                            tile_load(s_h + h * kXTile, &mapHigh, h * 128, t0, h_full);
                            tile_load(s_h + (HB + h) * kXTile, &mapLow, h * 128, t0, h_full);
                        }
                    }
                    h_open = true;
                    h_round ^= 1u;
                }
            }
            for (int d = 0; ok && d < count; ++d) {
                const int row = __ldcg(info + 1 + d) * static_cast<int>(p.N) + col;
                if (!(ok = agreed_wait(&b_empty[bs], b_round ^ 1u, &s_dead))) break;
                if (elect_one()) {
                    mbar_expect_tx(&b_full[bs], static_cast<uint32_t>(kB));
#pragma unroll
                    for (int h = 0; h < HB; ++h) tile_load(s_b + bs * kB + h * (CT * 128), &mapB, h * 128, row, &b_full[bs]);
                }
                b_issued = min(b_issued + 1, SB);
                if (++bs == SB) { bs = 0; b_round ^= 1u; }
            }
        }
        if (!ok) {                            // copies still in flight land before the CTA leaves
            for (; y_issued > 0; --y_issued) {
                if (--ys < 0) { ys = SY - 1; y_round ^= 1u; }
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&y_full[ys], y_round); ++polls) {}
            }
            for (; b_issued > 0; --b_issued) {
                if (--bs < 0) { bs = SB - 1; b_round ^= 1u; }
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&b_full[bs], b_round); ++polls) {}
            }
            if (h_open)
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(h_full, h_round ^ 1u); ++polls) {}
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_f16<DT>(128, CT, false);
        const uint64_t desc_h = smem_desc_k128(s_h), desc_b = smem_desc_k128(s_b);
        const int steps = (p.R + 15) / 16;
        int bs = 0, db = 0, count = 0;
        uint32_t b_round = 0, d_round = 0, h_round = 0;
        int64_t tile = -1;
        bool ok = true;
        for (int64_t it = work.first; ok && it < work.end; it += work.step) {
            const int64_t tl = it / work.cols;
            if (tl != tile) {
                tile = tl;
                count = __ldcg(p.info + tl * kTileInfo);
                if (count > 0) {
                    if (!(ok = agreed_wait(h_full, h_round, &s_dead))) break;
                    h_round ^= 1u;
                }
            }
            const bool last = it + work.step >= work.end || (it + work.step) / work.cols != tl;
            for (int d = 0; ok && d < count; ++d) {
                if (!(ok = agreed_wait(&b_full[bs], b_round, &s_dead) && agreed_wait(&d_empty[db], d_round ^ 1u, &s_dead))) break;
                tc_fence_after();
                if (elect_one()) {
                    for (int part = 0; part < 2; ++part)
                        for (int k = 0; k < steps; ++k)
                            tc_mma_f16(tmem + db * CT, desc_h + (((part * HB + (k >> 2)) * kXTile + (k & 3) * 32) >> 4),
                                       desc_b + ((bs * kB + (k >> 2) * (CT * 128) + (k & 3) * 32) >> 4), idesc, part > 0 || k > 0);
                    tc_commit(&b_empty[bs]);
                    tc_commit(&d_full[db]);
                    if (last && d + 1 == count) tc_commit(h_empty);
                }
                if (++bs == SB) { bs = 0; b_round ^= 1u; }
                if (++db == kOutBuffers) { db = 0; d_round ^= 1u; }
            }
        }
        if (!ok) {                            // products in flight end before the CTA leaves
            __syncwarp();
            if (elect_one()) tc_commit(drain);
            for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(drain, 0); ++polls) {}
        }
    } else if (warp == 2 && !LOOSE) {
        int ys = 0;
        uint32_t y_round = 0;
        bool ok = true;
        for (int64_t it = work.first; it < work.end; it += work.step) {
            const int64_t tl = it / work.cols;
            const int col = static_cast<int>(it - tl * work.cols) * CT;
            if (!(ok = agreed_wait(&o_full[ys], y_round, &s_dead))) break;
            if (elect_one()) {
                const int32_t x = col * (YT == CQ_F32 ? 4 : 2), t0 = static_cast<int32_t>(tl) * kTileTokens;
                tile_store(&mapOut, s_y + ys * kYTile, x, t0);
                if (col + CT / 2 < p.N) tile_store(&mapOut, s_y + ys * kYTile + kXTile, x + 128, t0);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                mbar_arrive(&y_empty[ys]);
            }
            if (++ys == SY) { ys = 0; y_round ^= 1u; }
        }
        __syncwarp();
        if (elect_one()) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp >= 4) {
        constexpr int kCols = CT / 2;                           // of each warp
        const int half = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * kCols;
        int ys = 0, db = 0, count = 0, mine = -1;
        uint32_t y_round = 0, d_round = 0;
        float f = 0.0f;
        int64_t tile = -1;
        bool ok = true;
        // LOOSE: these warps bring the rows of y themselves, those of the next item while this one is worked on; all eight meet at barriers on
        // either side of the additions, also after a wait that gave up.
        LooseRows rows;
        const int row0 = (warp - 4) * 16;
        auto place = [&](int64_t it, int64_t& t, int64_t& col) {
            t = it / work.cols * kTileTokens + row0;
            col = it % work.cols * CT;
        };
        int64_t t_in = 0, col_in = 0;
        if constexpr (LOOSE) {
            place(work.first, t_in, col_in);
            if (work.first < work.end) fetch_rows<YT>(p, t_in, col_in, rows);
        }
        for (int64_t it = work.first; (ok || LOOSE) && it < work.end; it += work.step) {
            const int64_t tl = it / work.cols;
            if (tl != tile) {
                tile = tl;
                count = __ldcg(p.info + tl * kTileInfo);
                const int64_t t = tl * kTileTokens + row;
                mine = t < p.T ? __ldcg(p.slot + t) : -1;
                f = mine >= 0 ? __ldcg(p.factor + t) : 0.0f;
            }
            const int64_t t_out = t_in, col_out = col_in;
            if constexpr (LOOSE) {
                rows_to_tile<YT>(p, t_in, col_in, rows, s_y, row0);
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (it + work.step < work.end) {
                    place(it + work.step, t_in, col_in);
                    fetch_rows<YT>(p, t_in, col_in, rows);
                }
            } else {
                if (!(ok = agreed_wait(&y_full[ys], y_round, &s_dead))) break;
            }
            uint8_t* y = s_y + ys * kYTile + half * kXTile + row * 128;
            for (int d = 0; ok && d < count; ++d) {
                if (!(ok = agreed_wait(&d_full[db], d_round, &s_dead))) break;
                tc_fence_after();
                if (__any_sync(0xFFFFFFFFu, mine == d)) {
                    float v[kCols / 32][32];
#pragma unroll
                    for (int q = 0; q < kCols / 32; ++q) tmem_ld32(at + db * CT + q * 32, v[q]);
#pragma unroll
                    for (int q = 0; q < kCols / 32; ++q) tmem_ld_wait(v[q]);
                    if (mine == d) {
                        add_to_row<YT>(y, row, v, f);
                    }
                    __syncwarp();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&d_empty[db]);
                if (++db == kOutBuffers) { db = 0; d_round ^= 1u; }
            }
            if constexpr (LOOSE) {
                asm volatile("bar.sync 1, 256;" ::: "memory");
                tile_to_rows<YT>(p, t_out, col_out, s_y, row0);
                __syncwarp();
            } else {
                if (!ok) break;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&o_full[ys]);
                if (++ys == SY) { ys = 0; y_round ^= 1u; }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    __syncwarp();
    if (warp == 1) tmem_free(tmem, kOutBuffers * CT);
    if (tid == 0 && s_dead != 0u) atomicExch(&g_adapter_fault, 1u);
}

// ---- host ----------------------------------------------------------------------------------------------------------
int adapter_stage_fault(unsigned int* fault_host) {
    return cudaMemcpyFromSymbol(fault_host, g_adapter_fault, sizeof(unsigned int)) == cudaSuccess ? CQ_OK : CQ_ERR_CUDA;
}

// A tile of fewer than 128 tokens is mostly empty (40 tokens on 8 adapters x 4096 x 6144, rank 16: 18.0 us, 9.9 in windows; 128 x 8192 x 8192 on 64 adapters
// 48.8 us, 89 in windows; on one 16.5, 18.1), and what a tensor map cannot hold goes the other way too.
constexpr int64_t kMapMost = (int64_t(1) << 31) - 1024;
bool adapter_in_tiles(const AdapterArgs& p) {
    return p.T >= kTileTokens && p.K >= 64 && p.n >= 1 && p.vec_k == 8 && 2 * p.K < kMapMost && static_cast<int64_t>(p.n) * p.R < kMapMost &&
           p.ldx < (int64_t(1) << 38);
}
bool adapter_out_tiles(const AdapterArgs& p, int y_dtype) {
    // Rows that begin anywhere want two tiles of tokens to win (300 x 17853, rank 16: 37.2 us, 38.5 in windows; 130 tokens 30.2, 24.3; 2223, rank 64:
    // 107, 256).
    const int64_t elem = y_dtype == CQ_F32 ? 4 : 2, least = p.vec_n == 16 / elem ? kTileTokens : 2 * kTileTokens;
    return p.T >= least && p.n >= 1 && elem * p.N < kMapMost && p.n * p.N < kMapMost && p.ldy < (int64_t(1) << 37) && p.ldo < (int64_t(1) << 37);
}

template <int HB, int DT, int YT, bool LOOSE>
static int launch_out_tiles(const AdapterArgs& p, cudaStream_t st) {
    constexpr int64_t elem = YT == CQ_F32 ? 4 : 2;
    CUtensorMap high, low, b, y, out;
    const auto sw = CU_TENSOR_MAP_SWIZZLE_128B;
    if (!make_byte_map(&high, p.high, 2 * p.R, p.T, 2 * p.R, 128, kTileTokens, sw) || !make_byte_map(&low, p.low, 2 * p.R, p.T, 2 * p.R, 128, kTileTokens, sw) ||
        !make_byte_map(&b, p.B, 2 * p.R, p.n * p.N, 2 * p.R, 128, out_cols<YT>(), sw)) return CQ_ERR_CUDA;
    if constexpr (LOOSE) y = out = b;         // (not used)
    else if (!make_byte_map(&y, p.y, elem * p.N, p.T, elem * p.ldy, 128, kTileTokens, sw) ||
             !make_byte_map(&out, p.out, elem * p.N, p.T, elem * p.ldo, 128, kTileTokens, sw)) return CQ_ERR_CUDA;
    static thread_local LaunchMemo memo;
    constexpr size_t smem = out_smem<HB, YT>();
    if (resident_ctas(k28_adapter_out_tiles<HB, DT, YT, LOOSE>, kOutThreads, smem, smem, memo) < 1) return CQ_ERR_CUDA;
    const int64_t items = (p.T + kTileTokens - 1) / kTileTokens * ((p.N + out_cols<YT>() - 1) / out_cols<YT>());
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(items, sm_count()));
    // blocks in groups that take neighbouring columns at one time, so that rows of y pass through memory in long pieces: 4096 x 28672
    // 131 us with every block on a run of its own, 127 in groups of 4, 105 of 37 (a quarter of the SMs), 109 of 74, 114 of 148
    const int group = grid >= 16 && grid % 4 == 0 ? grid / 4 : 1;
    return launch_ex(k28_adapter_out_tiles<HB, DT, YT, LOOSE>, dim3(grid), kOutThreads, smem, st, 1, !tuning_no_pdl(), high, low, b, y, out, p, group);
}

// Clusters of 2^i blocks that are resident at one time (asked once for a device).
constexpr int kMaxParts = 4;
template <typename Kernel>
static int resident_clusters(Kernel* kernel, int i) {
    struct Known { int device; int n[kMaxParts]; };
    static thread_local Known k = {-1, {}};
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) return 0;
    if (k.device != device) k = {device, {}};
    if (k.n[i] == 0) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1u << i;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.gridDim = dim3(1u << i, 1, 1);
        cfg.blockDim = dim3(kInThreads);
        cfg.dynamicSmemBytes = kInSmem;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&k.n[i], kernel, &cfg) != cudaSuccess) {
            cudaGetLastError();
            k.n[i] = 0;
        }
    }
    return k.n[i];
}

template <int DT>
static int launch_in_tiles(const AdapterArgs& p, cudaStream_t st) {
    CUtensorMap x, a;
    if (!make_byte_map(&x, p.x, 2 * p.K, p.T, 2 * p.ldx, 128, kTileTokens, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_byte_map(&a, p.A, 2 * p.K, static_cast<uint64_t>(p.n) * p.R, 2 * p.K, 128, p.R, CU_TENSOR_MAP_SWIZZLE_128B)) return CQ_ERR_CUDA;
    static thread_local LaunchMemo memo;
    if (resident_ctas(k27_adapter_in_tiles<DT>, kInThreads, kInSmem, kInSmem, memo) < 1) return CQ_ERR_CUDA;
    // The parts of the contraction, four blocks of 64 or more to each, with which tiles of few adapters end first, as those of prompts do; then, as
    // far as there is room, several clusters a tile, which share out the groups of 128 / R adapters that it may have (a tile with fewer
    // leaves the others idle).
    const int64_t tiles = (p.T + kTileTokens - 1) / kTileTokens, per = kInCols / p.R, blocks = (p.K + 63) / 64;
    const int64_t groups = (std::min<int64_t>(p.n, kTileTokens) + per - 1) / per;
    int64_t parts = 1, turns = 1, least = INT64_MAX;
    for (int i = kMaxParts - 1; i >= 0; --i) {
        const int64_t n = int64_t(1) << i, room = resident_clusters(k27_adapter_in_tiles<DT>, i);
        if (room < 1) return CQ_ERR_CUDA;
        const int64_t length = (tiles + room - 1) / room * ((blocks + n - 1) / n);
        if ((n > 1 && blocks < 4 * n) || length >= least) continue;
        least = length;
        parts = n;
        turns = std::max<int64_t>(1, std::min(groups, room / tiles));
    }
    return launch_ex(k27_adapter_in_tiles<DT>, dim3(static_cast<unsigned>(parts), static_cast<unsigned>(tiles), static_cast<unsigned>(turns)), kInThreads, kInSmem, st,
                     static_cast<unsigned>(parts), !tuning_no_pdl(), x, a, p, in_stages(p.R));
}
int launch_adapter_in_tiles(const AdapterArgs& p, int dtype, cudaStream_t st) {
    return dtype == CQ_F16 ? launch_in_tiles<CQ_F16>(p, st) : launch_in_tiles<CQ_BF16>(p, st);
}

template <int HB, int DT, int YT>
static int launch_out_rows(const AdapterArgs& p, cudaStream_t st) {
    return p.vec_n == (YT == CQ_F32 ? 4 : 8) ? launch_out_tiles<HB, DT, YT, false>(p, st) : launch_out_tiles<HB, DT, YT, true>(p, st);
}
template <int HB, int DT>
static int launch_out_type(const AdapterArgs& p, int y_dtype, cudaStream_t st) {
    if (y_dtype == CQ_F32) return launch_out_rows<HB, DT, CQ_F32>(p, st);
    return y_dtype == CQ_F16 ? launch_out_rows<HB, DT, CQ_F16>(p, st) : launch_out_rows<HB, DT, CQ_BF16>(p, st);
}
template <int DT>
static int launch_out_rank(const AdapterArgs& p, int y_dtype, cudaStream_t st) {
    return p.R <= 64 ? launch_out_type<1, DT>(p, y_dtype, st) : launch_out_type<2, DT>(p, y_dtype, st);
}
int launch_adapter_out_tiles(const AdapterArgs& p, int dtype, int y_dtype, cudaStream_t st) {
    return dtype == CQ_F16 ? launch_out_rank<CQ_F16>(p, y_dtype, st) : launch_out_rank<CQ_BF16>(p, y_dtype, st);
}

}  // namespace cq
