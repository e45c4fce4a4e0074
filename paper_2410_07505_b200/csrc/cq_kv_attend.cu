// Attention of a few query tokens over the quantized key/value cache.
//
// With l_j = scale * sum_d q_d kf_d kc_jd * ka_j (codes kc, token scales ka, channel factors kf; likewise vc, va, vf):
//   out_d = vf_d * sum_j softmax(l)_j va_j vc_jd
// Neither factor has to be applied to a cached element: kf goes into the query, ka onto the logit, va onto the
// probability, vf onto the result.  The cache is read once and its codes meet the tensor cores as fp16 integers (exact).
//
// Bound by HBM: 2 (D bits / 8 + 4) bytes for a token and key/value head, and a few query rows (the G heads that share
// it x the query tokens) to use them for, so the products run on mma.sync (m16n8k16, fp32 sums) straight from registers
// while the loads set the pace.
//
// Work: every (sequence, head, tile of rows) is a group of 64-token units; all units in a row are cut into equal parts,
// one for each resident CTA, whatever the lengths are.  A CTA's four warps take 16 tokens of a unit each and keep
// running maxima, sums and results of their own (no barrier between units); they are joined in warp order at the end of
// a group.  A group that ends in another CTA leaves its sums in the workspace and a second kernel joins those in the
// order of the tokens: the same bits every time.
// Each warp feeds itself through a ring of asynchronous copies (tensor-map boxes of 16 tokens, swizzled so that the
// fragments' reads meet no bank conflicts, and the tokens' scales), running ahead across groups.  Waits are bounded.
//
// fp16 operands: a query row (times kf) is scaled by a power of two into [2^14, 2^15) before it is rounded, so its
// rounding is 2^-12 of each element; probabilities times va are scaled by 2^15 over a power of two above the largest va
// seen, so small ones keep 11 bits down to 2^-29 of the largest.  Logits, maxima, sums and results are fp32.
#include "cq_kv.cuh"

namespace cq {

__device__ unsigned int g_attn_fault = 0;      // set if a bounded wait ever gave up

constexpr int kUnit = 64;                       // tokens of a unit: 16 for each warp
constexpr int kAttWarps = 4;
constexpr int kAttThreads = 32 * kAttWarps;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttendArgs {
    const void* q; int64_t qb, ql, qh;          // strides of sequences, tokens and heads, in elements
    int q_vec;                                  // rows of q may be read four elements at a time
    const int* table; int64_t table_stride;     // [B][table_stride] page numbers
    const int* lens;                            // [B]
    const float* scale[2];                      // token scales of keys and values
    const float* col[2];
    void* out;                                  // [B][Lq][Hq][D], dense
    float* lse;                                 // [B][Lq][Hq] or null
    float* part;                                // [2 * CTAs][rows of a tile][D], then [..][2] maxima and sums
    float softmax_scale;
    int64_t pages;
    int B, Lq, Hq, H, G, page_size, row_tiles;
    int64_t capacity;                           // tokens a row of the table can name
};

// ---- the sequence of units ------------------------------------------------------------------------
__device__ __forceinline__ int seq_len(const AttendArgs& p, int b) {
    const int n = __ldg(p.lens + b);
    return n <= 0 ? 0 : static_cast<int>(min(static_cast<int64_t>(n), p.capacity));
}
__device__ __forceinline__ int tiles_of(int len) { return (len + kUnit - 1) / kUnit; }

// Units before sequence `upto` (in tiles of one row group), computed by a whole warp.
__device__ __forceinline__ int64_t tiles_before(const AttendArgs& p, int upto) {
    const int lane = threadIdx.x & 31;
    int64_t sum = 0;
    for (int b = lane; b < upto; b += 32) sum += tiles_of(seq_len(p, b));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
    return sum;
}
__device__ __forceinline__ int64_t part_start(int64_t units, int64_t cta, int64_t ctas) { return units * cta / ctas; }
__device__ __forceinline__ int64_t part_of(int64_t units, int64_t u, int64_t ctas) { return ((u + 1) * ctas - 1) / units; }

struct Cursor {
    int b, group, tile, tiles, len;             // group = head * row_tiles + tile of rows
    __device__ __forceinline__ void enter(const AttendArgs& p, int seq) {
        b = seq;
        len = 0;
        while (b < p.B && (len = seq_len(p, b)) == 0) ++b;
        tiles = tiles_of(len);
        group = 0;
        tile = 0;
    }
    __device__ __forceinline__ void next(const AttendArgs& p) {
        if (++tile < tiles) return;
        tile = 0;
        if (++group < p.H * p.row_tiles) return;
        enter(p, b + 1);
    }
    // the unit with number u, by a whole warp
    __device__ __forceinline__ void seek(const AttendArgs& p, int64_t u) {
        const int lane = threadIdx.x & 31;
        const int64_t per = static_cast<int64_t>(p.H) * p.row_tiles;
        int64_t base = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int mine = b0 + lane < p.B ? seq_len(p, b0 + lane) : 0;
            const int64_t n = tiles_of(mine);
            int64_t incl = n;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int64_t t = __shfl_up_sync(0xFFFFFFFFu, incl, off);
                if (lane >= off) incl += t;
            }
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, u < (base + incl) * per && n > 0);
            if (hit != 0) {
                const int l = __ffs(hit) - 1;
                b = b0 + l;
                len = __shfl_sync(0xFFFFFFFFu, mine, l);
                tiles = tiles_of(len);
                const int64_t before = base + __shfl_sync(0xFFFFFFFFu, incl, l) - tiles;
                const int64_t r = u - before * per;
                group = static_cast<int>(r / tiles);
                tile = static_cast<int>(r - static_cast<int64_t>(group) * tiles);
                return;
            }
            base += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        b = p.B; group = 0; tile = 0; tiles = 0; len = 0;
    }
};

// ---- fragments ------------------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float pow2i(int e) { return e < -126 ? 0.0f : __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (code + bias) in the low bits of fp16 1024, minus 1024 and the bias: exact
constexpr uint32_t kH1152 = 0x64806480u;        // 1024 + 128, twice
constexpr uint32_t kH1032 = 0x64086408u;        // 1024 + 8
constexpr uint32_t kHSixteenth = 0x2C002C00u;   // 1 / 16
constexpr uint32_t kHm72 = 0xD480D480u;         // -(1024 / 16 + 8)
__device__ __forceinline__ uint32_t byte_pair(uint32_t w, uint32_t sel) { return hsub2(__byte_perm(w, 0x64646464u, sel), kH1152); }
__device__ __forceinline__ uint32_t nib_low(uint32_t w) { return hsub2((w & 0x000F000Fu) | 0x64006400u, kH1032); }
__device__ __forceinline__ uint32_t nib_high(uint32_t w) { return hfma2((w & 0x00F000F0u) | 0x64006400u, kHSixteenth, kHm72); }

// 16-byte piece `c` of row `r` in a box of rows of RB bytes under the tensor map's swizzle of that width
template <int RB>
__device__ __forceinline__ uint32_t box_at(int r, int c) {
    if constexpr (RB == 128) return r * 128 + ((c ^ (r & 7)) << 4);
    else if constexpr (RB == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
    else return r * 32 + ((c ^ ((r >> 2) & 1)) << 4);
}

// The place along D of element e (0..3: the fragment's k = 2r, 2r+1, 2r+8, 2r+9) of contraction step kk for lane r of
// a quad: any assignment serves as long as queries and keys share it; this one lets a lane read 16 bytes at a time.
template <int D, int BITS>
__device__ __forceinline__ int place(int r, int kk, int e) {
    if constexpr (BITS == 8) return r * (D / 4) + kk * 4 + e;
    else return r * (D / 4) + (kk >> 1) * 8 + (kk & 1) * 2 + (e >> 1) + (e & 1) * 4;
}

template <int D, int BITS, int MT>
struct AttendShape {
    static constexpr int kRow = D * BITS / 8;                   // bytes of a token's codes
    static constexpr int kBox = 16 * kRow;
    static constexpr int kStages = BITS == 8 && D == 128 ? 3 : 4;
    static constexpr int kRows = 16 * MT;
    static constexpr size_t kSmem = 1024 + size_t(kAttWarps) * kStages * (2 * kBox + 128) + size_t(kRows) * D * 4;
};

// ---- units of a CTA -------------------------------------------------------------------------------
template <int DT, int D, int BITS, int MT>
__global__ void __launch_bounds__(kAttThreads, MT == 1 ? 3 : 2)
k16_kv_attend(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const AttendArgs p) {
    using S = AttendShape<D, BITS, MT>;
    constexpr int RB = S::kRow, ST = S::kStages, KK = D / 16, NT = D / 8, ROWS = S::kRows;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kAttWarps][ST];
    __shared__ int s_valid[kAttWarps][ST];
    __shared__ float s_m[kAttWarps][ROWS], s_l[kAttWarps][ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, r4 = lane & 3;
    uint8_t* s_box = smem + warp * ST * 2 * S::kBox;                                       // [stage][keys, values][16][RB]
    float* s_scale = reinterpret_cast<float*>(smem + kAttWarps * ST * 2 * S::kBox) + warp * ST * 32;   // [stage][keys, values][16]
    float* s_o = reinterpret_cast<float*>(smem + kAttWarps * ST * (2 * S::kBox + 128));    // [ROWS][D]

    asm volatile("griddepcontrol.launch_dependents;");
    const int64_t units = tiles_before(p, p.B) * p.H * p.row_tiles;
    const int64_t parts = min(units, static_cast<int64_t>(gridDim.x));          // so that none is empty
    if (blockIdx.x >= parts) return;
    const int64_t u0 = part_start(units, blockIdx.x, parts), u1 = part_start(units, blockIdx.x + 1, parts);
    if (lane == 0)
        for (int i = 0; i < ST; ++i) mbar_init(&full[warp][i], 1);
    mbar_init_fence();
    __syncwarp();

    // -- the loading side: units ahead of the computing side
    Cursor ahead;
    ahead.seek(p, u0);
    Cursor now = ahead;
    int64_t to_load = u1 - u0;
    int known_b = -1, known_tile = 0, known_page = -1;         // lane i: the page of this warp's tokens in tile known_tile + i
    auto load = [&](int stage) {                               // the next unit's 16 tokens of this warp
        const int tok = ahead.tile * kUnit + warp * 16;
        const int valid = min(16, ahead.len - tok);
        if (known_b != ahead.b || ahead.tile < known_tile || ahead.tile >= known_tile + 32) {
            known_b = ahead.b;
            known_tile = ahead.tile;
            const int mine = (known_tile + lane) * kUnit + warp * 16;
            known_page = mine < ahead.len ? __ldg(p.table + ahead.b * p.table_stride + mine / p.page_size) : -1;
        }
        const int page = __shfl_sync(0xFFFFFFFFu, known_page, ahead.tile - known_tile);
        const bool there = valid > 0 && page >= 0 && page < p.pages;
        if (lane == 0) {
            s_valid[warp][stage] = there ? valid : 0;
            if (there) {
                const int head = ahead.group / p.row_tiles;
                const int64_t row = (static_cast<int64_t>(page) * p.H + head) * p.page_size + tok % p.page_size;
                uint8_t* box = s_box + stage * 2 * S::kBox;
                mbar_expect_tx(&full[warp][stage], 2 * S::kBox + 128);
                tile_load(box, &mapK, 0, static_cast<int32_t>(row), &full[warp][stage]);
                tile_load(box + S::kBox, &mapV, 0, static_cast<int32_t>(row), &full[warp][stage]);
                bulk_load(s_scale + stage * 32, p.scale[0] + row, 64, &full[warp][stage]);
                bulk_load(s_scale + stage * 32 + 16, p.scale[1] + row, 64, &full[warp][stage]);
            }
        }
        --to_load;
        ahead.next(p);
    };
    for (int i = 0; i < ST && to_load > 0; ++i) load(i);
    __syncwarp();

    uint32_t phases = 0;                                       // parity of each stage's barrier
    int stage = 0;
    bool dead = false;
    for (int64_t u = u0; u < u1;) {
        // -- one group, or the part of it that lies in this CTA
        const int head = now.group / p.row_tiles, rt = now.group % p.row_tiles;
        const int first_tile = now.tile, tiles = now.tiles, len = now.len, b = now.b;
        const int n_units = static_cast<int>(min(u1 - u, static_cast<int64_t>(tiles - first_tile)));
        const int R = p.G * p.Lq;
        uint32_t qf[MT][KK][4];
        float fac[MT][2];                                      // logits of row quad, quad + 8: product * fac * ka
        int last[MT][2];                                       // last token that the row sees
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float2 x[2][KK][2];
            float top[2] = {0.0f, 0.0f};
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int row = rt * ROWS + mt * 16 + hf * 8 + quad;
                const int i = row / p.G, g = row - i * p.G;
                const bool there = row < R;
                last[mt][hf] = there ? len - p.Lq + i : -1;
                const uint16_t* src = static_cast<const uint16_t*>(p.q) + b * p.qb + i * p.ql + static_cast<int64_t>(head * p.G + g) * p.qh;
#pragma unroll
                for (int kk = 0; kk < KK; kk += (BITS == 8 ? 1 : 2)) {
                    // the four (INT4: eight) neighbours along D of this step (these two steps)
                    constexpr int kN = BITS == 8 ? 4 : 8;
                    const int d0 = place<D, BITS>(r4, kk, 0);
                    float v[kN];
#pragma unroll
                    for (int e = 0; e < kN; e += 4) {
                        uint2 w = make_uint2(0, 0);
                        if (there) {
                            if (p.q_vec) {
                                w = __ldg(reinterpret_cast<const uint2*>(src + d0 + e));
                            } else {
                                w.x = src[d0 + e] | (static_cast<uint32_t>(src[d0 + e + 1]) << 16);
                                w.y = src[d0 + e + 2] | (static_cast<uint32_t>(src[d0 + e + 3]) << 16);
                            }
                        }
                        const float2 lo = unpack16x2<DT>(w.x), hi = unpack16x2<DT>(w.y);
                        v[e] = lo.x; v[e + 1] = lo.y; v[e + 2] = hi.x; v[e + 3] = hi.y;
                        if (p.col[0] != nullptr) {
                            const float4 c = __ldg(reinterpret_cast<const float4*>(p.col[0] + static_cast<int64_t>(head) * D + d0 + e));
                            v[e] *= c.x; v[e + 1] *= c.y; v[e + 2] *= c.z; v[e + 3] *= c.w;
                        }
                    }
                    if constexpr (BITS == 8) {
                        x[hf][kk][0] = make_float2(v[0], v[1]);
                        x[hf][kk][1] = make_float2(v[2], v[3]);
                    } else {
                        x[hf][kk][0] = make_float2(v[0], v[4]);
                        x[hf][kk][1] = make_float2(v[1], v[5]);
                        x[hf][kk + 1][0] = make_float2(v[2], v[6]);
                        x[hf][kk + 1][1] = make_float2(v[3], v[7]);
                    }
#pragma unroll
                    for (int e = 0; e < kN; ++e) top[hf] = fmaxf(top[hf], fabsf(v[e]));
                }
                top[hf] = fmaxf(top[hf], __shfl_xor_sync(0xFFFFFFFFu, top[hf], 1));
                top[hf] = fmaxf(top[hf], __shfl_xor_sync(0xFFFFFFFFu, top[hf], 2));
                // power of two that brings the largest element into [2^14, 2^15); within the range of a float both ways
                const int e = top[hf] > 0.0f ? max(-100, min(100, 14 - (static_cast<int>(__float_as_uint(top[hf]) >> 23) - 127))) : 0;
                const float up = pow2i(e);
                fac[mt][hf] = pow2i(-e) * p.softmax_scale * kLog2e;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    qf[mt][kk][hf] = pack_half2(x[hf][kk][0].x * up, x[hf][kk][0].y * up);
                    qf[mt][kk][2 + hf] = pack_half2(x[hf][kk][1].x * up, x[hf][kk][1].y * up);
                }
            }
        }
        float o[MT][NT][4], m[MT][2], l[MT][2];
        int va_exp = -126;                                     // results are held in units of 2^(va_exp - 15)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt][0] = m[mt][1] = -INFINITY;
            l[mt][0] = l[mt][1] = 0.0f;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[mt][t][0] = o[mt][t][1] = o[mt][t][2] = o[mt][t][3] = 0.0f;
        }

        for (int n = 0; n < n_units; ++n) {
            const int valid = dead ? 0 : s_valid[warp][stage];
            if (valid > 0) {
                if (!mbar_wait(&full[warp][stage], (phases >> stage) & 1u)) {
                    dead = true;                               // nothing is loaded or computed from here on
                    if (lane == 0) atomicExch(&g_attn_fault, 1u);
                }
                phases ^= 1u << stage;
            }
            if (valid > 0 && !dead) {
                const int tok0 = (first_tile + n) * kUnit + warp * 16;
                const uint8_t* kbox = s_box + stage * 2 * S::kBox;
                const uint8_t* vbox = kbox + S::kBox;
                const float* sc = s_scale + stage * 32;
                // -- logits: 16 rows x 16 tokens for each tile of rows
                float s[MT][2][4];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    constexpr int kWords = RB / 16;            // words of a lane: a quarter of the row
                    uint32_t w[kWords];
                    const int row = nt * 8 + quad;
                    if constexpr (kWords >= 4) {
#pragma unroll
                        for (int c = 0; c < kWords / 4; ++c) {
                            const uint4 t = *reinterpret_cast<const uint4*>(kbox + box_at<RB>(row, r4 * (kWords / 4) + c));
                            w[4 * c] = t.x; w[4 * c + 1] = t.y; w[4 * c + 2] = t.z; w[4 * c + 3] = t.w;
                        }
                    } else {
                        const uint2 t = *reinterpret_cast<const uint2*>(kbox + box_at<RB>(row, r4 >> 1) + (r4 & 1) * 8);
                        w[0] = t.x; w[1] = t.y;
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) s[mt][nt][0] = s[mt][nt][1] = s[mt][nt][2] = s[mt][nt][3] = 0.0f;
#pragma unroll
                    for (int j = 0; j < kWords; ++j) {
                        if constexpr (BITS == 8) {
                            const uint32_t x = w[j] ^ 0x80808080u;
                            const uint32_t b0 = byte_pair(x, 0x4140u), b1 = byte_pair(x, 0x4342u);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) mma16816(s[mt][nt], qf[mt][j], b0, b1);
                        } else {
                            const uint32_t x = w[j] ^ 0x88888888u, y = x >> 8;
                            const uint32_t b0 = nib_low(x), b1 = nib_high(x), b2 = nib_low(y), b3 = nib_high(y);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                mma16816(s[mt][nt], qf[mt][2 * j], b0, b1);
                                mma16816(s[mt][nt], qf[mt][2 * j + 1], b2, b3);
                            }
                        }
                    }
                }
                // -- probabilities; this lane's tokens are 2 r4, 2 r4 + 1 (nt = 0) and those + 8 (nt = 1)
                const float2 ka[2] = {*reinterpret_cast<const float2*>(sc + 2 * r4), *reinterpret_cast<const float2*>(sc + 8 + 2 * r4)};
                float2 va[2] = {*reinterpret_cast<const float2*>(sc + 16 + 2 * r4), *reinterpret_cast<const float2*>(sc + 24 + 2 * r4)};
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {               // what lies past the end may be anything
                    if (nt * 8 + 2 * r4 >= valid) va[nt].x = 0.0f;
                    if (nt * 8 + 2 * r4 + 1 >= valid) va[nt].y = 0.0f;
                }
                const uint32_t vtop = __reduce_max_sync(0xFFFFFFFFu, max(max(__float_as_uint(va[0].x) & 0x7FFFFFFFu, __float_as_uint(va[0].y) & 0x7FFFFFFFu),
                                                                         max(__float_as_uint(va[1].x) & 0x7FFFFFFFu, __float_as_uint(va[1].y) & 0x7FFFFFFFu)));
                const int vexp = max(va_exp, min(126, static_cast<int>(vtop >> 23) - 126));        // 2^vexp > every va
                const float vshift = pow2i(max(va_exp - vexp, -127));
                va_exp = vexp;
                const float vinv = pow2i(-vexp);
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    va[nt].x = va[nt].x * vinv * 32768.0f;
                    va[nt].y = va[nt].y * vinv * 32768.0f;
                }
                const bool edge = tok0 + 15 > len - p.Lq || valid < 16;       // some row does not see some token
                uint32_t pf[MT][4];
                float shrink[MT][2];
                bool any = false;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        float e[2][2];
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            e[nt][0] = s[mt][nt][2 * hf] * (fac[mt][hf] * ka[nt].x);
                            e[nt][1] = s[mt][nt][2 * hf + 1] * (fac[mt][hf] * ka[nt].y);
                            if (edge) {
                                const int t = tok0 + nt * 8 + 2 * r4;
                                if (t > last[mt][hf]) e[nt][0] = -INFINITY;
                                if (t + 1 > last[mt][hf]) e[nt][1] = -INFINITY;
                            }
                        }
                        float top = fmaxf(fmaxf(e[0][0], e[0][1]), fmaxf(e[1][0], e[1][1]));
                        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                        const float was = m[mt][hf], is = fmaxf(was, top);
                        const float ref = is == -INFINITY ? 0.0f : is;
                        const float keep = ex2(was - ref);
                        m[mt][hf] = is;
                        float sum = 0.0f;
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            const float p0 = ex2(e[nt][0] - ref), p1 = ex2(e[nt][1] - ref);
                            sum += p0 + p1;
                            pf[mt][2 * nt + hf] = pack_half2(p0 * va[nt].x, p1 * va[nt].y);
                        }
                        l[mt][hf] = __fmaf_rn(l[mt][hf], keep, sum);
                        shrink[mt][hf] = keep * vshift;
                        any = any || is != was;
                    }
                }
                if (__any_sync(0xFFFFFFFFu, any) || vshift != 1.0f) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            o[mt][t][0] *= shrink[mt][0]; o[mt][t][1] *= shrink[mt][0];
                            o[mt][t][2] *= shrink[mt][1]; o[mt][t][3] *= shrink[mt][1];
                        }
                }
                // -- results: tile t of eight columns holds element t of every lane group's share of the row
                constexpr int kVWords = RB / 32;               // words of a lane and token: an eighth of the row
                uint32_t w[4][kVWords];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = 2 * r4 + (k & 1) + (k >> 1) * 8;
                    if constexpr (kVWords == 4) {
                        const uint4 t = *reinterpret_cast<const uint4*>(vbox + box_at<RB>(row, quad));
                        w[k][0] = t.x; w[k][1] = t.y; w[k][2] = t.z; w[k][3] = t.w;
                    } else if constexpr (kVWords == 2) {
                        const uint2 t = *reinterpret_cast<const uint2*>(vbox + box_at<RB>(row, quad >> 1) + (quad & 1) * 8);
                        w[k][0] = t.x; w[k][1] = t.y;
                    } else {
                        w[k][0] = *reinterpret_cast<const uint32_t*>(vbox + box_at<RB>(row, quad >> 2) + (quad & 3) * 4);
                    }
                }
#pragma unroll
                for (int j = 0; j < kVWords; ++j) {
                    if constexpr (BITS == 8) {
                        uint32_t x[2][2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t a = w[2 * k][j] ^ 0x80808080u, c = w[2 * k + 1][j] ^ 0x80808080u;
                            x[k][0] = __byte_perm(a, c, 0x5140u);
                            x[k][1] = __byte_perm(a, c, 0x7362u);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t sel = (e & 1) ? 0x4342u : 0x4140u;
                            const uint32_t b0 = byte_pair(x[0][e >> 1], sel), b1 = byte_pair(x[1][e >> 1], sel);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) mma16816(o[mt][4 * j + e], pf[mt], b0, b1);
                        }
                    } else {
                        uint32_t x[2][2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t a = w[2 * k][j] ^ 0x88888888u, c = w[2 * k + 1][j] ^ 0x88888888u;
                            x[k][0] = __byte_perm(a, c, 0x5410u);
                            x[k][1] = __byte_perm(a, c, 0x7632u);
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            uint32_t b[2];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const uint32_t y = (e & 2) ? x[k][e >> 2] >> 8 : x[k][e >> 2];
                                b[k] = (e & 1) ? nib_high(y) : nib_low(y);
                            }
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) mma16816(o[mt][8 * j + e], pf[mt], b[0], b[1]);
                        }
                    }
                }
            }
            __syncwarp();                                      // the stage has been read by every lane
            if (to_load > 0 && !dead) load(stage);
            __syncwarp();
            stage = stage + 1 == ST ? 0 : stage + 1;
            now.next(p);
        }

        // -- join the four warps
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                l[mt][hf] += __shfl_xor_sync(0xFFFFFFFFu, l[mt][hf], 1);
                l[mt][hf] += __shfl_xor_sync(0xFFFFFFFFu, l[mt][hf], 2);
                if (r4 == 0) {
                    s_m[warp][mt * 16 + hf * 8 + quad] = m[mt][hf];
                    s_l[warp][mt * 16 + hf * 8 + quad] = l[mt][hf];
                }
            }
        __syncthreads();
        float f[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int row = mt * 16 + hf * 8 + quad;
                float top = s_m[0][row];
#pragma unroll
                for (int w = 1; w < kAttWarps; ++w) top = fmaxf(top, s_m[w][row]);
                f[mt][hf] = ex2(m[mt][hf] - (top == -INFINITY ? 0.0f : top)) * pow2i(va_exp) * (1.0f / 32768.0f);
            }
        for (int w = 0; w < kAttWarps; ++w) {
            if (warp == w) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // columns 2 r4, 2 r4 + 1 of tile t are element t of the shares of lane groups 2 r4, 2 r4 + 1
                            float* at = s_o + (mt * 16 + (e >> 1) * 8 + quad) * D + (2 * r4 + (e & 1)) * (D / 8) + t;
                            const float v = o[mt][t][e] * f[mt][e >> 1];
                            *at = w == 0 ? v : *at + v;
                        }
            }
            __syncthreads();
        }
        const bool begins = first_tile == 0, ends = first_tile + n_units == tiles;
        const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (begins ? 1 : 0);
        const int rows = min(ROWS, R - rt * ROWS);
        for (int idx = threadIdx.x; idx < rows * D; idx += kAttThreads) {
            const int row = idx / D, d = idx % D;
            float top = s_m[0][row];
#pragma unroll
            for (int w = 1; w < kAttWarps; ++w) top = fmaxf(top, s_m[w][row]);
            const float ref = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttWarps; ++w) sum += s_l[w][row] * ex2(s_m[w][row] - ref);
            const float v = s_o[idx];
            if (begins && ends) {
                const int rr = rt * ROWS + row, i = rr / p.G, g = rr - i * p.G;
                const int64_t at = (static_cast<int64_t>(b) * p.Lq + i) * p.Hq + head * p.G + g;
                float res = sum == 0.0f ? 0.0f : __fdiv_rn(v, sum);
                if (p.col[1] != nullptr) res *= __ldg(p.col[1] + static_cast<int64_t>(head) * D + d);
                static_cast<uint16_t*>(p.out)[at * D + d] = pack16<DT>(res);
                if (p.lse != nullptr && d == 0) p.lse[at] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
            } else {
                p.part[(slot * ROWS + row) * D + d] = v;
                if (d < 2) p.part[2 * static_cast<int64_t>(gridDim.x) * ROWS * D + (slot * ROWS + row) * 2 + d] = d == 0 ? top : sum;
            }
        }
        __syncthreads();
        u += n_units;
    }
    if (dead) {                                                // copies still in flight land before the CTA leaves
        for (int i = 0; i < ST; ++i)
            if (s_valid[warp][i] > 0) mbar_wait(&full[warp][i], (phases >> i) & 1u);
    }
}

// ---- join of groups that lie in several CTAs: one block for each query row ---------------------------
template <int DT, int D>
__global__ void __launch_bounds__(D)
k17_kv_join(const AttendArgs p, int64_t ctas, int rows_per_tile) {
    const int64_t row_id = blockIdx.x;                          // (b * Lq + i) * Hq + head * G + g
    const int hq = static_cast<int>(row_id % p.Hq);
    const int i = static_cast<int>(row_id / p.Hq % p.Lq), b = static_cast<int>(row_id / p.Hq / p.Lq);
    const int head = hq / p.G, r = i * p.G + hq % p.G;
    const int rt = r / rows_per_tile, row = r % rows_per_tile;
    const int d = threadIdx.x;
    const int len = seq_len(p, b);
    const int64_t at = row_id * D + d;
    if (len == 0) {                                             // nothing to attend to
        asm volatile("griddepcontrol.wait;" ::: "memory");      // (the memory may still be read by work before the call)
        static_cast<uint16_t*>(p.out)[at] = 0;
        if (p.lse != nullptr && d == 0) p.lse[row_id] = -INFINITY;
        return;
    }
    const int64_t per = static_cast<int64_t>(p.H) * p.row_tiles;
    const int64_t before = tiles_before(p, b), units = tiles_before(p, p.B) * per;
    const int tiles = tiles_of(len);
    const int64_t g0 = before * per + (static_cast<int64_t>(head) * p.row_tiles + rt) * tiles;
    const int64_t parts = min(units, ctas);
    const int64_t c0 = part_of(units, g0, parts), c1 = part_of(units, g0 + tiles - 1, parts);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (c0 == c1) return;                                       // that CTA has written the result
    const float* stats = p.part + 2 * ctas * rows_per_tile * D;
    auto slot = [&](int64_t c) { return ((2 * c + (c == c0 ? 1 : 0)) * rows_per_tile + row); };
    float top = -INFINITY;
    for (int64_t c = c0; c <= c1; ++c) top = fmaxf(top, stats[slot(c) * 2]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, v = 0.0f;
#pragma unroll 4
    for (int64_t c = c0; c <= c1; ++c) {
        const float f = ex2(stats[slot(c) * 2] - ref);
        sum = __fmaf_rn(stats[slot(c) * 2 + 1], f, sum);
        v = __fmaf_rn(p.part[slot(c) * D + d], f, v);
    }
    float res = sum == 0.0f ? 0.0f : __fdiv_rn(v, sum);
    if (p.col[1] != nullptr) res *= __ldg(p.col[1] + static_cast<int64_t>(head) * D + d);
    static_cast<uint16_t*>(p.out)[at] = pack16<DT>(res);
    if (p.lse != nullptr && d == 0) p.lse[row_id] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// ---- host ---------------------------------------------------------------------------------------------
constexpr int kMaxPerSm = 3;

int attn_stage_fault(unsigned int* fault_host) {
    return cudaMemcpyFromSymbol(fault_host, g_attn_fault, sizeof(unsigned int)) == cudaSuccess ? CQ_OK : CQ_ERR_CUDA;
}

static size_t attend_workspace(int64_t D) {
    return static_cast<size_t>(sm_count()) * kMaxPerSm * 2 * 32 * (D + 2) * sizeof(float);
}

template <int DT, int D, int BITS, int MT>
static int launch_attend(const AttendArgs& p, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t st) {
    using S = AttendShape<D, BITS, MT>;
    static thread_local LaunchMemo memo;
    int per_sm = resident_ctas(k16_kv_attend<DT, D, BITS, MT>, kAttThreads, S::kSmem, S::kSmem, memo);
    if (per_sm < 1) return CQ_ERR_CUDA;
    if (per_sm > kMaxPerSm) per_sm = kMaxPerSm;
    int64_t ctas = static_cast<int64_t>(sm_count()) * per_sm;
    const int64_t most = static_cast<int64_t>(p.B) * p.H * p.row_tiles * ((p.capacity + kUnit - 1) / kUnit);
    if (ctas > most) ctas = most;
    const int rc = launch_ex(k16_kv_attend<DT, D, BITS, MT>, dim3(static_cast<unsigned>(ctas)), kAttThreads, S::kSmem, st, 1, false, mapK, mapV, p);
    if (rc != CQ_OK) return rc;
    const int64_t rows = static_cast<int64_t>(p.B) * p.Lq * p.Hq;
    return launch_ex(k17_kv_join<DT, D>, dim3(static_cast<unsigned>(rows)), D, 0, st, 1, !tuning_no_pdl(), p, ctas, S::kRows);
}

template <int DT, int D, int BITS>
static int launch_attend_rows(AttendArgs& p, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t st) {
    const int64_t R = static_cast<int64_t>(p.G) * p.Lq;
    if (R <= 16) {
        p.row_tiles = 1;
        return launch_attend<DT, D, BITS, 1>(p, mapK, mapV, st);
    }
    p.row_tiles = static_cast<int>((R + 31) / 32);
    return launch_attend<DT, D, BITS, 2>(p, mapK, mapV, st);
}

}  // namespace cq

extern "C" {

size_t cq_kv_attention_workspace_bytes(int64_t D) {
    return D < 1 || D > 4096 ? 0 : cq::attend_workspace(D);
}

int cq_kv_attention(const void* Q, int dtype, int64_t q_batch_stride, int64_t q_token_stride, int64_t q_head_stride, int64_t B,
                    int64_t Lq, int64_t Hq, const void* k_codes, const void* v_codes, const float* k_scale, const float* v_scale,
                    const float* k_col, const float* v_col, int bits, int64_t pages, int64_t page_size, int64_t H, int64_t D,
                    const int* page_table, int64_t table_width, int64_t table_stride, const int* lens, double softmax_scale,
                    void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace cq;
    const int rc = check_cache(k_codes, v_codes, k_scale, v_scale, k_col, v_col, bits, pages, page_size, H, D);
    if (rc != CQ_OK) return rc;
    if (dtype != CQ_F16 && dtype != CQ_BF16) return CQ_ERR_DTYPE;
    if (B < 0 || Lq < 0 || Hq < H || Hq % H != 0 || table_width < 0 || table_stride < table_width) return CQ_ERR_SHAPE;
    if (!(softmax_scale > 0.0 && softmax_scale <= 1e30)) return CQ_ERR_ALPHA;
    if (B > (1 << 20) || Lq > (1 << 20) || Hq > (1 << 16) || B * Lq * Hq > 0x7FFFFFFF || Hq / H * Lq > (1 << 24)) return CQ_ERR_SHAPE;
    if (table_width * page_size > (int64_t(1) << 31) - 4096) return CQ_ERR_SHAPE;
    if (B == 0 || Lq == 0) return CQ_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (Q == nullptr || out == nullptr || lens == nullptr) return CQ_ERR_NULL;
    if (table_width > 0 && page_table == nullptr) return CQ_ERR_NULL;
    if (!ptr_aligned(Q, 2) || !ptr_aligned(out, 2) || !ptr_aligned(lens, 4) || !ptr_aligned(page_table, 4) || !ptr_aligned(lse, 4)) return CQ_ERR_ALIGN;
    if (workspace == nullptr || !ptr_aligned(workspace, 256) || workspace_bytes < attend_workspace(D)) return CQ_ERR_WORKSPACE;
    AttendArgs p;
    p.q = Q; p.qb = q_batch_stride; p.ql = q_token_stride; p.qh = q_head_stride;
    p.q_vec = ptr_aligned(Q, 8) && ((q_batch_stride | q_token_stride | q_head_stride) & 3) == 0;
    p.table = page_table; p.table_stride = table_stride; p.lens = lens;
    p.scale[0] = k_scale; p.scale[1] = v_scale; p.col[0] = k_col; p.col[1] = v_col;
    p.out = out; p.lse = lse; p.part = static_cast<float*>(workspace);
    p.softmax_scale = static_cast<float>(softmax_scale);
    p.pages = pages; p.B = static_cast<int>(B); p.Lq = static_cast<int>(Lq); p.Hq = static_cast<int>(Hq); p.H = static_cast<int>(H);
    p.G = static_cast<int>(Hq / H); p.page_size = static_cast<int>(page_size);
    p.row_tiles = 1;
    p.capacity = pages > 0 ? table_width * page_size : 0;
    if (p.capacity == 0) {                                      // no token can be named: every row is empty
        const int64_t rows = B * Lq * Hq;
        if (D == 64) return dtype == CQ_F16 ? launch_ex(k17_kv_join<CQ_F16, 64>, dim3(static_cast<unsigned>(rows)), 64, 0, st, 1, false, p, 1, 16)
                                            : launch_ex(k17_kv_join<CQ_BF16, 64>, dim3(static_cast<unsigned>(rows)), 64, 0, st, 1, false, p, 1, 16);
        return dtype == CQ_F16 ? launch_ex(k17_kv_join<CQ_F16, 128>, dim3(static_cast<unsigned>(rows)), 128, 0, st, 1, false, p, 1, 16)
                               : launch_ex(k17_kv_join<CQ_BF16, 128>, dim3(static_cast<unsigned>(rows)), 128, 0, st, 1, false, p, 1, 16);
    }
    const uint32_t row_bytes = static_cast<uint32_t>(D * bits / 8);
    const CUtensorMapSwizzle swizzle = row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : row_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
    const uint64_t rows = static_cast<uint64_t>(pages) * H * page_size;
    CUtensorMap mapK, mapV;
    if (!make_byte_map(&mapK, k_codes, row_bytes, rows, row_bytes, row_bytes, 16, swizzle) ||
        !make_byte_map(&mapV, v_codes, row_bytes, rows, row_bytes, row_bytes, 16, swizzle)) return CQ_ERR_CUDA;
    if (dtype == CQ_F16) {
        if (D == 128) return bits == 8 ? launch_attend_rows<CQ_F16, 128, 8>(p, mapK, mapV, st) : launch_attend_rows<CQ_F16, 128, 4>(p, mapK, mapV, st);
        return bits == 8 ? launch_attend_rows<CQ_F16, 64, 8>(p, mapK, mapV, st) : launch_attend_rows<CQ_F16, 64, 4>(p, mapK, mapV, st);
    }
    if (D == 128) return bits == 8 ? launch_attend_rows<CQ_BF16, 128, 8>(p, mapK, mapV, st) : launch_attend_rows<CQ_BF16, 128, 4>(p, mapK, mapV, st);
    return bits == 8 ? launch_attend_rows<CQ_BF16, 64, 8>(p, mapK, mapV, st) : launch_attend_rows<CQ_BF16, 64, 4>(p, mapK, mapV, st);
}

int cq_serve_fault(unsigned int* fault_host) {
    if (fault_host == nullptr) return CQ_ERR_NULL;
    unsigned int product = 0, attention = 0;
    int rc = cq::fp8_stage_fault(&product);
    if (rc == CQ_OK) rc = cq::attn_stage_fault(&attention);
    if (rc == CQ_OK) *fault_host = product | attention;
    return rc;
}

}  // extern "C"
