// Causal attention over packed prompts on the 5th-generation tensor cores.
//
// For sequence b with Lq queries and Lk keys (rows q_starts[b].. of Q and k_starts[b].. of K and V), query i sees the keys
// j <= Lk - Lq + i; G = Hq / H query heads share a key/value head:
//   out[i] = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i . k_j - ref_i),   c = softmax_scale log2(e)
// in one pass over the keys.  ref_i is the largest c q_i . k_j so far, renewed only when a block exceeds it by 2^kSlack, so
// that the running result is hardly ever rescaled.  (Beyond 2^20 the last bit of a logit in base 2 is worth more than a weight may be
// off by: there it is rounded before ref_i, one of them, is taken from it, so that the largest has the exponent that it should have.)
// Sums and references are fp32; p is rounded once to the inputs' 16 bits, as an operand of the second product (kind::f16 takes both
// operands in one type), in fp16 with 2^kBias in front so that small weights keep their bits.  That adds about half of the result's own
// rounding to its error (against 64 bits 0.0021 for 0.0016 in bf16, 0.00025 for 0.0002 in fp16).  FINE, the caller's choice, hands over what
// the rounding leaves as well, in the other half of the logits' columns, for a second product: the error is the result's rounding again.
//
// A persistent CTA takes pairs of tiles of 128 rows (tokens x query heads of one key head) over blocks of 128 keys, longest first.  Q, K
// and V come by TMA; the logits S = Q K^T of either tile stand in tensor memory (128 columns), the weights take their place (64), the
// results O are the other half of it.  While a tile's four warps form its weights, one row to a thread, the other tile's products run:
// S of the next block can begin only when O has taken in this one's weights, so that a tile alone would leave the tensor cores idle.
// What bounds it is that chain: products 768 cycles from the last weights to the next logits, signals about 200, loads and maxima 400 to 600, 128
// exponentials a row 1250 (the unit's 1024 and their tail), for either tile in turn; the tensor cores are busy 61 % of the time, the unit for
// exponentials 62 %.  Everything the softmax issues delays the products as well: a product costs its warp some 30 issue slots, which it shares
// with two softmax warps.  Tried and dropped: logits in two buffers of 64 keys (products of 64 columns are bound by shared memory, 970 us),
// two threads to a row (1220 us), a share of the exponentials by polynomial (895 us).
// Measured (GPU alone, operands not in L2): 1 x 8192 tokens, 64 / 8 heads of 128, bf16 869 us (1265 TFLOP/s; 1090 in a long run, which the power limit
// sets); 12 packed prompts up to 2060 tokens, 64 / 8 heads, fp16 338 us; 1000 tokens behind 19011, 32 heads of 64 257 us (bound by exponentials:
// 139 us at one a lane and clock); 1000 tokens, 32 / 8 heads 26.7 us.  FINE: 1132, 412, 306, 34.7 us (products 256 cycles longer on the chain).
#include "cq_serve.cuh"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace cq {

__device__ unsigned int g_prompt_fault = 0;   // set if a bounded wait ever gave up

constexpr int kPromptThreads = 384;           // warps 0..3, 4..7: softmax of the two tiles; warp 8: loads; warps 9, 10: products of either tile; one idle
constexpr int kTileRows = 128;                // rows of a tile: tokens x the query heads that go together
constexpr int kKeys = 128;                    // keys of a block
constexpr float kSlack = 8.0f;
constexpr float kFarLogit = 1048576.0f;       // 2^20: up to here c x - ref, formed in one rounding, is off by 2^-4 at most
constexpr int kMaxSplits = 16;
template <int DT> __host__ __device__ constexpr float prompt_bias() { return DT == CQ_F16 ? 7.0f : 0.0f; }   // 2^(7 + 8) < 65504

template <int D> __host__ __device__ constexpr int prompt_stages() { return D == 128 ? 5 : 8; }
template <int D> __host__ __device__ constexpr size_t prompt_tile() { return size_t(128) * D * 2; }         // bytes of a tile of Q and of a block of K or V
template <int D> __host__ __device__ constexpr size_t prompt_smem() { return (2 + prompt_stages<D>()) * prompt_tile<D>() + 512; }

struct PromptArgs {
    const int* q_starts; const int* k_starts;
    const uint16_t* v; int64_t vt, vh;        // strides of tokens and heads
    uint16_t* out; float* lse; float* part;
    float c;
    int Tq, Tk, B, Hq, G;
    int g, tokens;                            // a tile: `tokens` tokens x g query heads
    int groups;                               // (key heads) x (groups of g query heads of each)
    int splits;                               // parts of the keys of each item
};

// Two tiles of one sequence and head group, over the key blocks [jb, je).
struct PromptItem {
    int q0, tokens;                           // first row of Q, tokens of the item; tokens < 0: no more items
    int k0, sees, keys;                       // first row of K; keys that the item's first token sees (may be below 1); keys of the sequence
    int kv, head0, part;
    int jb, end[2];                           // key blocks of the tiles: [jb, end[t]), none where end[t] <= jb
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Two numbers at a time: half of the instructions, which the warps that issue the products compete with.
__device__ __forceinline__ uint64_t both(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 apart(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void tile_load3(void* dst_smem, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(smem_u32(dst_smem)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
// [128 rows along the contraction][64 elements along N] per 16 KB, 128-byte swizzle: 64 elements further along N lie 16 KB
// further, eight rows of the contraction 1024 bytes further.
__device__ __forceinline__ uint64_t smem_desc_n128(const void* tile) {
    const uint64_t addr = smem_u32(tile);
    return ((addr & 0x3FFFFu) >> 4) | (uint64_t(16384 >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                    "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const float (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 :: "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]),
                    "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// All lanes wait and agree on what came of it, so that a warp's roles never part.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* dead) {
    return __all_sync(0xFFFFFFFFu, role_wait(bar, parity, dead)) != 0;
}

// Two weights 2^(c x - ref), added to a pair of sums and rounded to a pair; FINE: what that leaves of them, rounded too.
template <int DT, bool FINE>
__device__ __forceinline__ uint32_t weights(float x0, float x1, uint64_t c, uint64_t neg, uint64_t& sums, uint32_t& rest) {
    const float2 u = apart(fma2(both(x0, x1), c, neg)), p = make_float2(ex2(u.x), ex2(u.y));
    sums = add2(sums, both(p.x, p.y));
    const uint32_t r = pack16x2<DT>(p.x, p.y);
    if constexpr (FINE) {
        const float2 v = unpack16x2<DT>(r);
        rest = pack16x2<DT>(p.x - v.x, p.y - v.y);
    }
    return r;
}

// nonzero bit 15 or 31 where a 16-bit element is an infinity or NaN
template <int DT>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t exponent = DT == CQ_BF16 ? 0x7F807F80u : 0x7C007C00u, one = DT == CQ_BF16 ? 0x00800080u : 0x04000400u;
    return ((w & exponent) + one) & 0x80008000u;
}

// ---- which item is the i-th ---------------------------------------------------------------------------------
// (Ordinary loads: the kernel before this one, which may have written the starts, can still run when this one begins.)
struct Sequence { int q0, k0, lq, lk; };
__device__ __forceinline__ Sequence sequence_at(const PromptArgs& p, int b) {
    const int q0 = min(max(p.q_starts[b], 0), p.Tq), q1 = min(max(p.q_starts[b + 1], q0), p.Tq);
    const int k0 = min(max(p.k_starts[b], 0), p.Tk), k1 = min(max(p.k_starts[b + 1], k0), p.Tk);
    return {q0, k0, q1 - q0, k1 - k0};
}
// Pairs of tiles of the sequence that need at least x blocks of keys.  Later pairs need more, the i-th
// ceil((lk - lq + min((i + 1) 2 tokens, lq)) / 128) of them.
__device__ __forceinline__ int pairs_from(const Sequence& s, int tokens2, int x) {
    const int n = (s.lq + tokens2 - 1) / tokens2;
    if (x <= 0 || n == 0) return n;
    const int room = (x - 1) * kKeys;                           // pairs whose last token sees no more need less
    if (s.lk <= room) return 0;
    const int below = room - (s.lk - s.lq);
    return n - min(below > 0 ? below / tokens2 : 0, n - 1);
}

// The items in the order of their work, the longest first: all head groups of a pair of tiles side by side, the pairs of all
// sequences by the number of their key blocks.  Computed by a whole warp.  A CTA's items come in falling order: the next one is looked for
// from where the last one was found, and all sequences are counted only where the number of blocks changes (1500 sequences of 64
// tokens, 32 / 8 heads: 410 us of 64 channels, 550 of 128; about 2200 where they were counted for every item).
struct ItemSearch {
    int level, above, upto;                   // pairs with more than `level` blocks, with `level` or more (at first none has as many)
    int b0, before;                           // a group of 32 sequences, and the pairs with `level` blocks of the sequences before it
};
__device__ __forceinline__ bool find_item(const PromptArgs& p, int64_t index, int total_pairs, ItemSearch& f, PromptItem& it) {
    const int lane = threadIdx.x & 31;
    const int per_pair = p.groups * p.splits;
    const int64_t rank64 = index / per_pair;
    if (rank64 >= total_pairs) return false;
    const int rank = static_cast<int>(rank64);
    const int within = static_cast<int>(index - rank64 * per_pair);
    const int tokens2 = 2 * p.tokens;
    auto count = [&](int x) {
        int n = 0;
#pragma unroll 2
        for (int b = lane; b < p.B; b += 32) n += pairs_from(sequence_at(p, b), tokens2, x);
        return __reduce_add_sync(0xFFFFFFFFu, n);
    };
    if (rank >= f.upto) {
        int lo = f.level, hi = lo, above = 0, upto = f.upto;    // count(hi) <= rank < count(lo) in the end
        for (int down = 1; upto <= rank; down *= 2) {
            hi = lo;
            above = upto;
            lo = max(lo - down, 0);
            upto = count(lo);
        }
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1, n = count(mid);
            if (n > rank) { lo = mid; upto = n; } else { hi = mid; above = n; }
        }
        f = {lo, above, upto, 0, 0};
    }
    Sequence seq{};
    int pair = -1;
    for (int b0 = f.b0; b0 < p.B; b0 += 32) {
        const int skip = rank - f.above - f.before;             // of the pairs with exactly that many blocks, from here on
        const bool have = b0 + lane < p.B;
        const Sequence s = have ? sequence_at(p, b0 + lane) : Sequence{0, 0, 0, 0};
        const int from = pairs_from(s, tokens2, f.level);
        int mine = from - pairs_from(s, tokens2, f.level + 1), before = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xFFFFFFFFu, before, off);
            if (lane >= off) before += o;
        }
        const int all = __shfl_sync(0xFFFFFFFFu, before, 31);
        before -= mine;
        const bool here = skip >= before && skip < before + mine;
        const unsigned who = __ballot_sync(0xFFFFFFFFu, here);
        if (who != 0u) {
            const int src = __ffs(who) - 1;
            const int at = (s.lq + tokens2 - 1) / tokens2 - from + (skip - before);
            seq.q0 = __shfl_sync(0xFFFFFFFFu, s.q0, src);
            seq.k0 = __shfl_sync(0xFFFFFFFFu, s.k0, src);
            seq.lq = __shfl_sync(0xFFFFFFFFu, s.lq, src);
            seq.lk = __shfl_sync(0xFFFFFFFFu, s.lk, src);
            pair = __shfl_sync(0xFFFFFFFFu, at, src);
            f.b0 = b0;
            break;
        }
        f.before += all;
    }
    if (pair < 0) return false;
    const int group = within / p.splits, per_kv = p.G / p.g;
    it.part = within - group * p.splits;
    it.kv = group / per_kv;
    it.head0 = it.kv * p.G + (group - it.kv * per_kv) * p.g;
    const int i0 = pair * tokens2;
    it.q0 = seq.q0 + i0;
    it.tokens = min(tokens2, seq.lq - i0);
    it.k0 = seq.k0;
    it.keys = seq.lk;
    it.sees = seq.lk - seq.lq + i0 + 1;
    int n[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int last = min((t + 1) * p.tokens, it.tokens) - 1;
        n[t] = last < t * p.tokens ? 0 : (max(it.sees + last, 0) + kKeys - 1) / kKeys;
    }
    const int blocks = max(n[0], n[1]);
    it.jb = static_cast<int>(static_cast<int64_t>(blocks) * it.part / p.splits);
    const int stop = static_cast<int>(static_cast<int64_t>(blocks) * (it.part + 1) / p.splits);
    it.end[0] = min(stop, n[0]);
    it.end[1] = min(stop, n[1]);
    return true;
}

// ---- the kernel ------------------------------------------------------------------------------------------------
template <int D, int DT, bool FINE>                            // FINE: weights as two 16-bit numbers each
__global__ void __launch_bounds__(kPromptThreads, 1)
k22_prompt(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
           const PromptArgs p) {
    constexpr int ST = prompt_stages<D>();
    constexpr uint32_t kTile = static_cast<uint32_t>(prompt_tile<D>());
    constexpr float kBias = prompt_bias<DT>();
    // No static shared memory, so that the dynamic part starts on the 1024-byte boundary that the swizzle wants.
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* s_q = smem;                                        // [tile][half of D][128 rows][128 bytes]
    uint8_t* s_kv = s_q + 2 * kTile;                            // [stage][half of D][128 keys][128 bytes]
    uint64_t* full = reinterpret_cast<uint64_t*>(s_kv + ST * kTile);
    uint64_t* empty = full + ST;
    uint64_t* q_full = empty + ST;
    uint64_t* q_empty = q_full + 2;
    uint64_t* s_full = q_empty + 2;
    uint64_t* p_full = s_full + 2;
    uint64_t* o_full = p_full + 4;                              // (p_full: two halves of the keys for each tile)
    uint64_t* i_full = o_full + 2;
    uint64_t* i_empty = i_full + 2;
    uint64_t* drain = i_empty + 2;
    uint64_t* turn = drain + 2;
    PromptItem* s_item = reinterpret_cast<PromptItem*>(turn + 2);
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(s_item + 2);
    volatile uint32_t& s_dead = *(reinterpret_cast<volatile uint32_t*>(s_item + 2) + 1);
    volatile uint32_t& s_poison = *(reinterpret_cast<volatile uint32_t*>(s_item + 2) + 2);
    static_assert((2 * ST + 20) * 8 + 2 * sizeof(PromptItem) + 12 <= 512, "barriers");
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        if ((smem_u32(smem) & 1023u) != 0u) atomicExch(&g_prompt_fault, 1u);      // cannot be: see above
        for (int i = 0; i < ST; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 2); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1); mbar_init(&p_full[2 * i], 4); mbar_init(&p_full[2 * i + 1], 4); mbar_init(&o_full[i], 1);
            mbar_init(&i_full[i], 1); mbar_init(&i_empty[i], 10); mbar_init(&drain[i], 1); mbar_init(&turn[i], 4);
        }
        mbar_init_fence();
        s_dead = 0;
        s_poison = 0;
        prefetch_map(&mapQ);
        prefetch_map(&mapK);
        prefetch_map(&mapV);
    }
    if (warp == 9) tmem_alloc(&s_tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    asm volatile("griddepcontrol.launch_dependents;");  // (behind the allocation: see tmem_alloc)
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");    // 128 x 72 + 256 x 216 = 384 x 168
        if (warp == 8) {
            // ---- items and loads
            int total = 0, most = 0;
            for (int b = lane; b < p.B; b += 32) {
                const Sequence s = sequence_at(p, b);
                total += pairs_from(s, 2 * p.tokens, 0);
                if (s.lq > 0) most = max(most, (s.lk + kKeys - 1) / kKeys);
            }
            total = __reduce_add_sync(0xFFFFFFFFu, total);
            ItemSearch search{__reduce_max_sync(0xFFFFFFFFu, most) + 1, 0, 0, 0, 0};
            bool ok = true;
            int s = 0;
            uint32_t round = 0, issued = 0, q_round[2] = {0, 0};
            bool q_open[2] = {false, false};
            for (uint32_t n = 0; ok; ++n) {
                PromptItem it;
                // in rounds of one item for each CTA, every other one in reverse, so that none gets the longest of each
                const int64_t index = static_cast<int64_t>(n) * gridDim.x + ((n & 1u) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
                const bool have = find_item(p, index, total, search, it);
                if (!have) it.tokens = -1;
                if (!(ok = warp_wait(&i_empty[n & 1], ((n >> 1) & 1) ^ 1u, &s_dead))) break;
                if (lane == 0) {
                    s_item[n & 1] = it;
                    mbar_arrive(&i_full[n & 1]);
                }
                __syncwarp();
                if (!have) break;
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (it.end[t] > it.jb) {
                        if (!(ok = warp_wait(&q_empty[t], q_round[t] ^ 1u, &s_dead))) break;
                        if (elect_one()) {
                            mbar_expect_tx(&q_full[t], p.g * p.tokens * D * 2);
#pragma unroll
                            for (int h = 0; h < D / 64; ++h)
                                tile_load3(s_q + t * kTile + h * 16384, &mapQ, h * 64, it.head0, it.q0 + t * p.tokens, &q_full[t]);
                        }
                        q_open[t] = true;
                        q_round[t] ^= 1u;
                    }
                const int je = max(it.end[0], it.end[1]);
                for (int j = it.jb; ok && j < je; ++j)
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        if (!(ok = warp_wait(&empty[s], round ^ 1u, &s_dead))) break;
                        if (elect_one()) {
                            mbar_expect_tx(&full[s], kTile);
#pragma unroll
                            for (int h = 0; h < D / 64; ++h)
                                tile_load3(s_kv + s * kTile + h * 16384, kv == 0 ? &mapK : &mapV, h * 64, it.kv, it.k0 + j * kKeys, &full[s]);
                        }
                        issued = min(issued + 1, uint32_t(ST));
                        if (++s == ST) { s = 0; round ^= 1u; }
                    }
            }
            if (!ok) {                            // copies still in flight land before the CTA leaves
                for (; issued > 0; --issued) {
                    if (--s < 0) { s = ST - 1; round ^= 1u; }
                    for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&full[s], round); ++polls) {}
                }
                for (int t = 0; t < 2; ++t)
                    if (q_open[t])
                        for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&q_full[t], q_round[t] ^ 1u); ++polls) {}
            }
        } else if (warp <= 10) {
            // ---- products, a warp for each tile: a wait costs the tensor cores' queue, which holds two or three products, about 90
            // cycles, unless the other warp feeds it meanwhile
            constexpr uint32_t idesc_s = idesc_f16<DT>(128, kKeys, false), idesc_o = idesc_f16<DT>(128, D, true);
            const int t = warp - 9;
            const uint64_t desc_q = smem_desc_k128(s_q + t * kTile), desc_k = smem_desc_k128(s_kv), desc_v = smem_desc_n128(s_kv);
            const uint32_t at_s = tmem + t * 128, at_o = tmem + 256 + t * 128;
            bool ok = true;
            int s = 0;
            uint32_t round = 0, p_round = 0, q_round = 0;
            for (uint32_t n = 0; ok; ++n) {
                if (!(ok = warp_wait(&i_full[n & 1], (n >> 1) & 1, &s_dead))) break;
                const int jb = s_item[n & 1].jb, end = s_item[n & 1].end[t], je = max(s_item[n & 1].end[0], s_item[n & 1].end[1]);
                const bool last = s_item[n & 1].tokens < 0;
                __syncwarp();
                if (lane == 0) mbar_arrive(&i_empty[n & 1]);
                if (last) break;
                for (int j = jb - 1; ok && j < je; ++j) {       // results of block j, logits of block j + 1
                    const bool results = j >= jb && j < end, next = j + 1 < end;
                    int sv = s, sk = s;
                    uint32_t rv = round, rk = round;
                    if (j >= jb) {
                        if (++s == ST) { s = 0; round ^= 1u; }
                        sk = s;
                        rk = round;
                    }
                    if (j + 1 < je && ++s == ST) { s = 0; round ^= 1u; }
                    if (j >= jb && !(ok = warp_wait(&full[sv], rv, &s_dead))) break;
                    if (j + 1 < je && !(ok = warp_wait(&full[sk], rk, &s_dead))) break;
                    if (next && j < jb) {
                        if (!(ok = warp_wait(&q_full[t], q_round, &s_dead))) break;
                        q_round ^= 1u;
                    }
                    if (results) {
                        if (!(ok = warp_wait(&p_full[2 * t], p_round, &s_dead))) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kKeys / 32; ++k)
                                tc_mma_f16_ts(at_o, at_s + k * 8, desc_v + ((sv * kTile + k * 2048) >> 4), idesc_o, j > jb || k != 0);
                            if constexpr (FINE) {
#pragma unroll
                                for (int k = 0; k < kKeys / 32; ++k)
                                    tc_mma_f16_ts(at_o, at_s + kKeys / 2 + k * 8, desc_v + ((sv * kTile + k * 2048) >> 4), idesc_o, true);
                            }
                        }
                        __syncwarp();
                        if (!(ok = warp_wait(&p_full[2 * t + 1], p_round, &s_dead))) break;
                        p_round ^= 1u;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        if (results) {
#pragma unroll
                            for (int k = kKeys / 32; k < kKeys / 16; ++k)
                                tc_mma_f16_ts(at_o, at_s + k * 8, desc_v + ((sv * kTile + k * 2048) >> 4), idesc_o, true);
                            if constexpr (FINE) {
#pragma unroll
                                for (int k = kKeys / 32; k < kKeys / 16; ++k)
                                    tc_mma_f16_ts(at_o, at_s + kKeys / 2 + k * 8, desc_v + ((sv * kTile + k * 2048) >> 4), idesc_o, true);
                            }
                            if (!next) tc_commit(&o_full[t]);
                        }
                        if (next) {                             // (behind the product that reads the weights in the same columns)
#pragma unroll
                            for (int k = 0; k < D / 16; ++k)    // 32 bytes further along the swizzled row, 16 KB to the other half
                                tc_mma_f16(at_s, desc_q + (((k >> 2) * 16384 + (k & 3) * 32) >> 4),
                                           desc_k + ((sk * kTile + (k >> 2) * 16384 + (k & 3) * 32) >> 4), idesc_s, k != 0);
                            tc_commit(&s_full[t]);
                            if (j + 2 == end) tc_commit(&q_empty[t]);
                        }
                        if (j >= jb) tc_commit(&empty[sv]);
                        if (j + 1 < je) tc_commit(&empty[sk]);
                    }
                    __syncwarp();
                }
            }
            if (!ok) {                        // products in flight end before the CTA leaves
                __syncwarp();
                if (elect_one()) tc_commit(&drain[t]);
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&drain[t], 0); ++polls) {}
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- softmax: one row of a tile for each thread
        const int t = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t at_s = tmem + t * 128 + lanes, at_o = tmem + 256 + t * 128 + lanes;
        const int token = row < p.g * p.tokens ? t * p.tokens + row / p.g : 1 << 30;         // of the item; far behind it: no row of the tile
        uint32_t s_round = 0, o_round = 0, t_round = 0, slot = 0;               // `slot`: places of the ring that items before this one took
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            if (!(ok = warp_wait(&i_full[n & 1], (n >> 1) & 1, &s_dead))) break;
            const PromptItem& it = s_item[n & 1];               // (stays there until the end of the item)
            if (it.tokens < 0) break;
            const int jb = it.jb, end = it.end[t];
            const uint32_t first_slot = slot;
            slot += 2 * max(max(it.end[0], it.end[1]) - jb, 0);
            if (t * p.tokens >= it.tokens) {                    // no such tile
                __syncwarp();
                if (lane == 0) mbar_arrive(&i_empty[n & 1]);
                continue;
            }
            const int sees = it.sees + token;                   // this row's keys are the first `sees`
            const int all_see = it.sees + t * p.tokens;         // those that every row of the tile sees
            const int common = min(it.end[0], it.end[1]);         // blocks before this one are both tiles'
            // Weights are 2^(c x - ref).  Of a row whose reference came to lie beyond kFarLogit it is `far` (-infinity: there is none; kBias would
            // be lost in it) and ref -infinity, so that every block of the row asks for a new one and the far from 0 cost the others nothing.
            // (Rows of no token, whose logits are whatever lay in memory, ask for none.)
            float ref = token < 1 << 30 ? -INFINITY : INFINITY, far = -INFINITY, sum = 0.0f;
            for (int j = jb; j < end; ++j) {
                if (!(ok = warp_wait(&s_full[t], s_round, &s_dead))) break;
                s_round ^= 1u;
                tc_fence_after();
                float x[4][32];
                tmem_ld32(at_s, x[0]);
                tmem_ld32(at_s + 32, x[1]);
                tmem_ld_wait(x[0]);
                tmem_ld_wait(x[1]);
                tmem_ld32(at_s + 64, x[2]);
                tmem_ld32(at_s + 96, x[3]);
                float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 32; ++i) m[i & 3] = max3(m[i & 3], x[i >> 4][(2 * i) & 31], x[i >> 4][((2 * i) & 31) + 1]);
                tmem_ld_wait(x[2]);
                tmem_ld_wait(x[3]);
#pragma unroll
                for (int i = 32; i < 64; ++i) m[i & 3] = max3(m[i & 3], x[i >> 4][(2 * i) & 31], x[i >> 4][((2 * i) & 31) + 1]);
                const bool edge = (j + 1) * kKeys > all_see;
                if (edge) {
                    const int lim = sees - j * kKeys;
#pragma unroll
                    for (int i = 0; i < 128; ++i) x[i >> 5][i & 31] = i < lim ? x[i >> 5][i & 31] : -INFINITY;
                    m[0] = m[1] = m[2] = m[3] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 64; ++i) m[i & 3] = max3(m[i & 3], x[i >> 4][(2 * i) & 31], x[i >> 4][((2 * i) & 31) + 1]);
                    // A weight of 0 does not hide an infinity or NaN in V from the product: such elements become 0 in shared memory
                    // and are added to the rows that see them at the end.
                    const uint32_t place = first_slot + 2 * (j - jb) + 1;
                    if (!(ok = warp_wait(&full[place % ST], (place / ST) & 1, &s_dead))) break;
                    uint4* v4 = reinterpret_cast<uint4*>(s_kv + (place % ST) * kTile) + row;
                    uint32_t bad = 0;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        const uint4 w = v4[i * 128];
                        bad |= not_finite<DT>(w.x) | not_finite<DT>(w.y) | not_finite<DT>(w.z) | not_finite<DT>(w.w);
                    }
                    if (bad != 0u) {
                        s_poison = 1u;
                        __threadfence_block();
                        for (int i = 0; i < D / 8; ++i) {
                            uint16_t* e = reinterpret_cast<uint16_t*>(v4 + i * 128);
                            for (int k = 0; k < 8; ++k)
                                if (not_finite<DT>(e[k]) != 0u) e[k] = 0;
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                }
                auto half_ready = [&](int h) {
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[2 * t + h]);
                };
                const float top = __fmul_rn(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), p.c);
                const bool renew = top > ref + (kBias + kSlack);
                if (__any_sync(0xFFFFFFFFu, renew)) {
                    float keep = 1.0f;
                    if (renew && fabsf(top) < kFarLogit && far == -INFINITY) {
                        keep = ex2(ref - (top - kBias));
                        ref = top - kBias;
                    } else if (renew) {
                        if (far == -INFINITY || top - far > kSlack) {
                            keep = ex2(far == -INFINITY ? ref - top + kBias : far - top);
                            far = top;                          // (infinite too: infinity less infinity is NaN, in one rounding it would be 0)
                            ref = -INFINITY;
                        }
                        const float back = __frcp_rn(p.c);      // the exponent in two roundings, over c
#pragma unroll
                        for (int i = 0; i < 128; ++i) x[i >> 5][i & 31] = (__fmul_rn(x[i >> 5][i & 31], p.c) - far + kBias) * back;
                    }
                    sum *= keep;
                    __syncwarp();                               // (the accesses to tensor memory below are the whole warp's)
                    for (int q = 0; q < (j > jb ? D / 16 : 0); ++q) {
                        float o[16];
                        tmem_ld16(at_o + q * 16, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] *= keep;
                        tmem_st16(at_o + q * 16, o);
                    }
                }
                // The tiles take turns at their exponentials, so that one's stand beside the other's products: at random they meet, and
                // the unit for exponentials is full for both and then idle for both (1 x 8192 tokens: 1069 us).
                if (j < common && (t == 1 || j > jb)) {
                    if (!(ok = warp_wait(&turn[t], t_round, &s_dead))) break;
                    t_round ^= 1u;
                }
                const float neg = ref == -INFINITY ? 0.0f : -ref;
                const uint64_t neg2 = both(neg, neg), c2 = both(p.c, p.c);
                uint64_t l[2] = {0, 0};
                // Weights of 32 keys at a time, to where their logits stood.  A half is handed over behind the next quarter's exponentials, so that
                // their unit does not wait for the stores; the turn goes to the other tile before the last quarter's.
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (q == 3 && lane == 0 && j < common && (t == 0 || j + 1 < common)) mbar_arrive(&turn[t ^ 1]);
                    uint32_t r[16], rest[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        r[i] = weights<DT, FINE>(x[q][2 * i], x[q][2 * i + 1], c2, neg2, l[i & 1], rest[i]);
                    if (q == 2) half_ready(0);
                    tmem_st16(at_s + q * 16, r);
                    if constexpr (FINE) tmem_st16(at_s + kKeys / 2 + q * 16, rest);
                }
                half_ready(1);
                const float2 l2 = apart(add2(l[0], l[1]));
                sum += l2.x + l2.y;
            }
            if (!ok) break;
            const bool any = end > jb;
            if (any) {
                if (!(ok = warp_wait(&o_full[t], o_round, &s_dead))) break;
                o_round ^= 1u;
                tc_fence_after();
            }
            // ---- results of this row
            const bool mine = token < it.tokens;
            const bool poison = s_poison != 0u;
            const int64_t place = (static_cast<int64_t>(it.q0) + token) * p.Hq + it.head0 + row % p.g;
            const float inv = sum == 0.0f ? 0.0f : __frcp_rn(sum);
            // what is said of the row besides its result is in units of 2^ref, of a far one too
            const float unit = far == -INFINITY ? 1.0f : 1.0f / static_cast<float>(1 << static_cast<int>(kBias));
            if (far != -INFINITY) ref = far;
            const int from = max(jb, max(it.sees, 0) / kKeys) * kKeys, to = min(sees, end * kKeys);     // keys whose V may have been emptied
            const int64_t rows = static_cast<int64_t>(p.Tq) * p.Hq;
            float* part = p.part + (it.part * rows + place) * D;
#pragma unroll
            for (int q = 0; q < D / 32; ++q) {
                float o[32];
                __syncwarp();
                if (any) {
                    tmem_ld32(at_o + q * 32, o);
                    tmem_ld_wait(o);
                }
                if (sum == 0.0f || !any) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.0f;
                }
                if (poison && mine && sum != 0.0f)              // (0: nothing has weight, the row is zeros)
                    for (int j = from; j < to; ++j) {
                        const uint16_t* v = p.v + (static_cast<int64_t>(it.k0) + j) * p.vt + it.kv * p.vh + q * 32;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (not_finite<DT>(v[i]) != 0u) o[i] += cvt16<DT>(v[i]);
                    }
                if (!mine) continue;
                if (p.splits > 1) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        reinterpret_cast<float4*>(part + q * 32)[i] = make_float4(o[4 * i] * unit, o[4 * i + 1] * unit, o[4 * i + 2] * unit, o[4 * i + 3] * unit);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float* e = o + 8 * i;
                        reinterpret_cast<uint4*>(p.out + place * D + q * 32)[i] =
                            make_uint4(pack16x2<DT>(e[0] * inv, e[1] * inv), pack16x2<DT>(e[2] * inv, e[3] * inv),
                                       pack16x2<DT>(e[4] * inv, e[5] * inv), pack16x2<DT>(e[6] * inv, e[7] * inv));
                    }
                }
            }
            if (mine) {
                if (p.splits > 1)
                    *reinterpret_cast<float2*>(p.part + p.splits * rows * D + (it.part * rows + place) * 2) = make_float2(ref, sum * unit);
                else if (p.lse != nullptr)
                    p.lse[place] = sum == 0.0f ? -INFINITY : (ref + log2f(sum * unit)) * 0.69314718f;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&i_empty[n & 1]);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    __syncwarp();
    if (warp == 9) tmem_free(tmem, 512);
    if (threadIdx.x == 0 && s_dead != 0u) atomicExch(&g_prompt_fault, 1u);
}

// ---- join of the parts of split items: a warp for each row --------------------------------------------------
template <int D, int DT>
__global__ void __launch_bounds__(256)
k23_prompt_join(const PromptArgs p) {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t rows = static_cast<int64_t>(p.Tq) * p.Hq;
    const int64_t first = static_cast<int64_t>(min(max(p.q_starts[0], 0), p.Tq)) * p.Hq;
    const int64_t stop = static_cast<int64_t>(min(max(p.q_starts[p.B], 0), p.Tq)) * p.Hq;
    const float2* stats = reinterpret_cast<const float2*>(p.part + p.splits * rows * D);
    for (int64_t row = first + static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5); row < stop; row += static_cast<int64_t>(gridDim.x) * 8) {
        float2 st = make_float2(-INFINITY, 0.0f);
        if (lane < p.splits) st = __ldcg(stats + lane * rows + row);
        float top = st.x;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
        const float f = st.y == 0.0f ? 0.0f : ex2(st.x - top);
        float sum = st.y * f;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
        float o[D / 32] = {};
        for (int s = 0; s < p.splits; ++s) {
            const float fs = __shfl_sync(0xFFFFFFFFu, f, s);
            if (__shfl_sync(0xFFFFFFFFu, st.y, s) == 0.0f) continue;
            const float* part = p.part + (s * rows + row) * D + lane * (D / 32);
            if constexpr (D == 128) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(part));
                o[0] = __fmaf_rn(v.x, fs, o[0]); o[1] = __fmaf_rn(v.y, fs, o[1]);
                o[2] = __fmaf_rn(v.z, fs, o[2]); o[3] = __fmaf_rn(v.w, fs, o[3]);
            } else {
                const float2 v = __ldcg(reinterpret_cast<const float2*>(part));
                o[0] = __fmaf_rn(v.x, fs, o[0]); o[1] = __fmaf_rn(v.y, fs, o[1]);
            }
        }
        const float inv = sum == 0.0f ? 0.0f : __frcp_rn(sum);
        uint32_t* out = reinterpret_cast<uint32_t*>(p.out + row * D) + lane * (D / 64);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) out[i] = pack16x2<DT>(o[2 * i] * inv, o[2 * i + 1] * inv);
        if (p.lse != nullptr && lane == 0) p.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
int prompt_stage_fault(unsigned int* fault_host) {
    return cudaMemcpyFromSymbol(fault_host, g_prompt_fault, sizeof(unsigned int)) == cudaSuccess ? CQ_OK : CQ_ERR_CUDA;
}

// Query heads of a key head that share a tile: the largest divisor of G up to 16 whose tiles have at least 120 of 128 rows.
// (All rows of a tile read the same keys, so heads side by side make the tile's tokens few: less of the diagonal is computed in vain,
// and short sequences leave fewer rows empty: 12 prompts up to 100 tokens, 32 / 8 heads of 128 17.4 us, 25.9 with a head a tile; 8192 tokens 469, 474.)
static int heads_of_tile(int G) {
    for (int g = G < 16 ? G : 16; g > 1; --g)
        if (G % g == 0 && g * (kTileRows / g) >= 120) return g;
    return 1;
}

struct PromptPlan { int g, tokens, groups, splits; int64_t items; };
static PromptPlan prompt_plan(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t H) {
    PromptPlan r;
    const int G = static_cast<int>(Hq / H);
    r.g = heads_of_tile(G);
    r.tokens = kTileRows / r.g;
    r.groups = static_cast<int>(Hq / r.g);
    r.items = (Tq / (2 * r.tokens) + std::min(B, Tq)) * r.groups;        // at most
    // Items for at most half of the SMs: the keys of each are split, four blocks or more to a part (100 tokens behind 19000, 8 heads of 128: 36 us
    // with the join, 238 in one part; behind 1000, 16 heads: 22.7, 30.0).  More items stay whole: two parts of each of 128 on 148 SMs are two
    // rounds and a join (1000 tokens behind 19011, 32 heads of 64: 257 us, 245 whole; 32 / 8 of 128 301, 274; 900 behind 3100 87, 66); of 96 they
    // gain only where keys are very many (640 tokens behind 19360, 32 heads of 64: 200, 250; behind 3360 61, 58).
    int64_t splits = r.items > 0 ? sm_count() / r.items : 1;
    splits = std::min(splits, Tk / std::max<int64_t>(B, 1) / (4 * kKeys));
    r.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(splits, kMaxSplits)));
    r.items *= r.splits;
    return r;
}

static bool make_head_map(CUtensorMap* map, const void* base, int64_t D, int64_t heads, int64_t tokens, int64_t head_stride, int64_t token_stride,
                          int box_heads, int box_tokens) {
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
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(head_stride) * 2, static_cast<cuuint64_t>(token_stride) * 2};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_tokens)}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int DT, bool FINE>
static int launch_prompt(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PromptArgs& p, int64_t items, cudaStream_t st) {
    static thread_local LaunchMemo memo;
    if (resident_ctas(k22_prompt<D, DT, FINE>, kPromptThreads, prompt_smem<D>(), prompt_smem<D>(), memo) < 1) return CQ_ERR_CUDA;
    const int64_t grid = std::min<int64_t>(items, sm_count());
    const int rc = launch_ex(k22_prompt<D, DT, FINE>, dim3(static_cast<unsigned>(grid)), kPromptThreads, prompt_smem<D>(), st, 1, !tuning_no_pdl(), q, k, v, p);
    if (rc != CQ_OK || p.splits == 1) return rc;
    const int64_t blocks = std::min<int64_t>((static_cast<int64_t>(p.Tq) * p.Hq + 7) / 8, 8 * sm_count());
    return launch_ex(k23_prompt_join<D, DT>, dim3(static_cast<unsigned>(blocks)), 256, 0, st, 1, !tuning_no_pdl(), p);
}

static bool prompt_shape_ok(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t H, int64_t D) {
    return (D == 64 || D == 128) && H >= 1 && Hq >= H && Hq % H == 0 && Hq <= (1 << 16) && B >= 0 && B <= (1 << 20) && Tq >= 0 && Tk >= 0 &&
           Tq < (int64_t(1) << 30) && Tk < (int64_t(1) << 30);
}

// Strides that a tensor map can hold: multiples of 16 bytes below 2^40.  The stride of an axis of one element is never used.
static int64_t used_stride(int64_t n, int64_t stride, int64_t dense) { return n > 1 ? stride : dense; }
static int check_strides(const void* X, int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride) {
    if (!ptr_aligned(X, 16)) return CQ_ERR_ALIGN;
    for (const int64_t s : {used_stride(tokens, token_stride, 8), used_stride(heads, head_stride, 8)}) {
        if (s <= 0 || s >= (int64_t(1) << 38)) return CQ_ERR_SHAPE;
        if (s % 8 != 0) return CQ_ERR_ALIGN;
    }
    return CQ_OK;
}

static int prompt_attention(bool fine, const void* Q, int64_t q_token_stride, int64_t q_head_stride, const void* K, int64_t k_token_stride,
                            int64_t k_head_stride, const void* V, int64_t v_token_stride, int64_t v_head_stride, int dtype, int64_t B,
                            int64_t Tq, int64_t Tk, int64_t Hq, int64_t H, int64_t D, const int* q_starts, const int* k_starts,
                            double softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!prompt_shape_ok(B, Tq, Tk, Hq, H, D)) return CQ_ERR_SHAPE;
    if (dtype != CQ_F16 && dtype != CQ_BF16) return CQ_ERR_DTYPE;
    if (!(softmax_scale >= 0x1p-100 && softmax_scale <= 1e30)) return CQ_ERR_ALPHA;
    if (B == 0 || Tq == 0) return CQ_OK;
    if (Q == nullptr || out == nullptr || q_starts == nullptr || k_starts == nullptr || (Tk > 0 && (K == nullptr || V == nullptr))) return CQ_ERR_NULL;
    if (!ptr_aligned(out, 16) || !ptr_aligned(lse, 4) || !ptr_aligned(q_starts, 4) || !ptr_aligned(k_starts, 4)) return CQ_ERR_ALIGN;
    int rc = check_strides(Q, Tq, Hq, q_token_stride, q_head_stride);
    if (rc == CQ_OK && Tk > 0) rc = check_strides(K, Tk, H, k_token_stride, k_head_stride);
    if (rc == CQ_OK && Tk > 0) rc = check_strides(V, Tk, H, v_token_stride, v_head_stride);
    if (rc != CQ_OK) return rc;
    const PromptPlan plan = prompt_plan(B, Tq, Tk, Hq, H);
    const size_t need = cq_prompt_attention_workspace_bytes(B, Tq, Tk, Hq, H, D);
    if (need > 0 && (workspace == nullptr || !ptr_aligned(workspace, 256) || workspace_bytes < need)) return CQ_ERR_WORKSPACE;
    PromptArgs p;
    p.q_starts = q_starts; p.k_starts = k_starts;
    p.v = static_cast<const uint16_t*>(V); p.vt = v_token_stride; p.vh = v_head_stride;
    p.out = static_cast<uint16_t*>(out); p.lse = lse; p.part = static_cast<float*>(workspace);
    p.c = static_cast<float>(softmax_scale * 1.4426950408889634);
    p.Tq = static_cast<int>(Tq); p.Tk = static_cast<int>(Tk); p.B = static_cast<int>(B); p.Hq = static_cast<int>(Hq); p.G = static_cast<int>(Hq / H);
    p.g = plan.g; p.tokens = plan.tokens; p.groups = plan.groups; p.splits = plan.splits;
    CUtensorMap mapQ, mapK, mapV;
    // without keys no block is ever loaded: any valid map stands for theirs
    const void* k = Tk > 0 ? K : Q;
    const void* v = Tk > 0 ? V : Q;
    const int64_t keys = Tk > 0 ? Tk : 1;
    if (!make_head_map(&mapQ, Q, D, Hq, Tq, used_stride(Hq, q_head_stride, D), used_stride(Tq, q_token_stride, Hq * D), plan.g, plan.tokens) ||
        !make_head_map(&mapK, k, D, Tk > 0 ? H : 1, keys, used_stride(Tk > 0 ? H : 1, k_head_stride, D), used_stride(keys, k_token_stride, H * D), 1, kKeys) ||
        !make_head_map(&mapV, v, D, Tk > 0 ? H : 1, keys, used_stride(Tk > 0 ? H : 1, v_head_stride, D), used_stride(keys, v_token_stride, H * D), 1, kKeys))
        return CQ_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto width) {
        constexpr int W = decltype(width)::value;
        if (fine) return dtype == CQ_F16 ? launch_prompt<W, CQ_F16, true>(mapQ, mapK, mapV, p, plan.items, st) : launch_prompt<W, CQ_BF16, true>(mapQ, mapK, mapV, p, plan.items, st);
        return dtype == CQ_F16 ? launch_prompt<W, CQ_F16, false>(mapQ, mapK, mapV, p, plan.items, st) : launch_prompt<W, CQ_BF16, false>(mapQ, mapK, mapV, p, plan.items, st);
    };
    return D == 128 ? launch(std::integral_constant<int, 128>()) : launch(std::integral_constant<int, 64>());
}

}  // namespace cq

extern "C" {

size_t cq_prompt_attention_workspace_bytes(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t H, int64_t D) {
    using namespace cq;
    if (!prompt_shape_ok(B, Tq, Tk, Hq, H, D)) return 0;
    const PromptPlan plan = prompt_plan(B, Tq, Tk, Hq, H);
    return plan.splits == 1 ? 0 : sizeof(float) * plan.splits * static_cast<size_t>(Tq) * Hq * (D + 2);
}

int cq_prompt_attention(const void* Q, int64_t q_token_stride, int64_t q_head_stride, const void* K, int64_t k_token_stride,
                        int64_t k_head_stride, const void* V, int64_t v_token_stride, int64_t v_head_stride, int dtype, int64_t B,
                        int64_t Tq, int64_t Tk, int64_t Hq, int64_t H, int64_t D, const int* q_starts, const int* k_starts,
                        double softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return cq::prompt_attention(false, Q, q_token_stride, q_head_stride, K, k_token_stride, k_head_stride, V, v_token_stride, v_head_stride, dtype, B, Tq, Tk,
                                Hq, H, D, q_starts, k_starts, softmax_scale, out, lse, workspace, workspace_bytes, stream);
}

int cq_prompt_attention_fine(const void* Q, int64_t q_token_stride, int64_t q_head_stride, const void* K, int64_t k_token_stride,
                             int64_t k_head_stride, const void* V, int64_t v_token_stride, int64_t v_head_stride, int dtype, int64_t B,
                             int64_t Tq, int64_t Tk, int64_t Hq, int64_t H, int64_t D, const int* q_starts, const int* k_starts,
                             double softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return cq::prompt_attention(true, Q, q_token_stride, q_head_stride, K, k_token_stride, k_head_stride, V, v_token_stride, v_head_stride, dtype, B, Tq, Tk,
                                Hq, H, D, q_starts, k_starts, softmax_scale, out, lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
