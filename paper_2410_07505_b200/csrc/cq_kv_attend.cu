// Attention of a few query tokens over the quantized key/value cache.
//
// With l_j = scale * sum_d q_d kf_d kc_jd * ka_j (codes kc, token scales ka, channel factors kf; likewise vc, va, vf):
//   out_d = vf_d * sum_j softmax(l)_j va_j vc_jd
// Neither factor has to be applied to a cached element: kf goes into the query, ka onto the logit, va onto the
// probability, vf onto the result.  The cache is read once and its codes meet the tensor cores as they are.
//
// Bound by HBM: 2 (D bits / 8 + 4) bytes for a token and key/value head, and few query rows (the G heads that share it
// times the query tokens) to use them for, so the products run on mma.sync (m16n8k16, fp32 sums) from registers while
// the loads set the pace.  Tokens (and, for the result, channels) are the 16-row side and query rows the 8-column side,
// so that up to 8 query rows cost one product where the other way round would pad them to 16.
//
// Work: every (sequence, head, tile of rows) is a group of 64-token units; all units in a row are cut into equal parts,
// one for each resident CTA, whatever the lengths are.  (A group counts kLead units more than it has, which is what its
// beginning and end cost, so that a part of many short groups is no longer than one of a few long ones.)  A CTA's four
// computing warps take 16 tokens of a unit each and keep running references, sums and results of their own (no barrier
// between units); they are joined in a fixed order at the end of a group.  A group that ends in another CTA leaves its
// sums in the workspace and a second kernel joins those in a fixed order: the same bits every time.
// A fifth warp keeps a ring of units filled by asynchronous copies (tensor-map boxes, swizzled so that the fragments'
// reads meet no bank conflicts, and the tokens' scales), running ahead across groups.  Waits are bounded.
//
// fp16 operands.  A key's code goes in as the subnormal (code + bias) * 2^-24, bias 128 or 8: its bits are the biased code,
// no arithmetic needed.  The bias is taken out of a logit by starting its sum at -bias * sum_d q_d.  (The other nibble of a
// byte comes in as 16 times its value; the query holds a sixteenth there.)  The tensor cores align a subnormal by its
// nominal exponent, which costs a sum about 2^-13 of one code: nothing beside a logit's other terms, but too much for a
// result whose likely tokens hold code 0, so a value's code goes in exactly, as fp16 1024 + code + bias minus 1024 + bias.
// A query row (times kf) is scaled by a power of two into [2^14, 2^15) before it is rounded, so its rounding is 2^-12 of
// each element.  A row's probabilities times va go in as fp16 in units of a power of two that put its largest between 2^4 and 2^16:
// what lies 2^-18 below that has 11 bits, what lies below has fewer.  Logits, maxima, sums and results are fp32.
// A bf16 result hides these roundings (2^-12 and 2^-12 beside 2^-9); an fp16 result does not, so for fp16 (FINE) queries
// and probabilities go in as two halves each, the second what the first leaves, at twice the products.
// The running reference of a row is a logit that was the largest when it was taken, rounded up to a whole number (base 2).  It is
// renewed, with the row's sum and results rescaled, when some logit exceeds it by more than 10; the row's unit likewise, when some
// probability times va nears the end of fp16.  Both are the row's own and follow from what it sees alone: a token behind a
// query's position, whatever its scales are, leaves no trace in that query's bits (its probability times va is set to 0, not formed:
// 0 times an infinite va is none).  One unit for all rows of a warp, above the largest va, took 2 to 7 % less time (4 x 100003 INT4,
// 16 rows a head: 114 against 118 us), but lost rows beside a large value that they do not see or give no weight: with 1e30 behind
// it, a value of 100 read as 0.  Less room above the reference (2^5) makes rows ask more often: 124 us.
#include "cq_kv.cuh"

namespace cq {

__device__ unsigned int g_attn_fault = 0;      // set if a bounded wait ever gave up

constexpr int kUnit = 64;                       // tokens of a unit: 16 for each computing warp
constexpr int kAttWarps = 4;
constexpr int kAttThreads = 32 * (kAttWarps + 1);
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLeastFac = 1.17549435e-38f;    // 2^-126
constexpr float kNoRef = -3.402823466e38f;      // the reference of a row that has seen nothing
constexpr float kMostProb = 1024.0f;            // a probability may be so many times the reference's,
constexpr float kMostUnits = 61440.0f;          // and a probability times va be so many of its row's units (fp16 ends at 65504);
constexpr int kPlace = 5;                       // new units put the row's largest between 2^4 and 2^5 of them

struct AttendArgs {
    const void* q; int64_t qb, ql, qh;          // strides of sequences, tokens and heads, in elements
    int q_vec;                                  // rows of q may be read four elements at a time
    const int* table; int64_t table_stride;     // [B][table_stride] page numbers
    const int* lens;                            // [B]
    const float* scale[2];                      // token scales of keys and values
    const float* col[2];
    void* out;                                  // [B][Lq][Hq][D], dense
    float* lse;                                 // [B][Lq][Hq] or null
    float* part;                                // [2 * CTAs][rows of a tile][D], then [..][2] maxima and sums, then Split[CTAs]
    float softmax_scale;
    int64_t pages;
    int B, Lq, Hq, H, G, page_size, row_tiles;
    int box;                                    // tokens of a copy: 16, 32 or 64, a divisor of the page size
    int unit_pages, unit_rest;                  // whole pages in a unit of tokens, and what is left
    int64_t capacity;                           // tokens a row of the table can name
};

// A group that begins in a CTA and ends in a later one: where its sums are to be joined.  parts: 0: there is none.
struct __align__(16) Split { int b, group, parts, unused; };
__device__ __forceinline__ Split* splits_of(const AttendArgs& p, int64_t ctas, int rows, int D) {
    return reinterpret_cast<Split*>(p.part + 2 * ctas * rows * (D + 2));
}

// ---- the sequence of units ------------------------------------------------------------------------
__device__ __forceinline__ int seq_len(const AttendArgs& p, int b) {
    const int n = __ldcg(p.lens + b);
    return n <= 0 ? 0 : static_cast<int>(min(static_cast<int64_t>(n), p.capacity));
}
__device__ __forceinline__ int tiles_of(int len) { return (len + kUnit - 1) / kUnit; }

// Units before sequence `upto` for one head and tile of rows, the groups' leads included; by a whole warp.
// (32 sequences up to 8191 tokens, INT8: 86.1 us with a lead of 1, 73.7 with 3, 66.4 with 4, 61.3 with 6, 65.0 with 9.)
constexpr int kLead = 7;
// A part has this many places at least: more parts of less than a tile or two would only make more to join (one sequence of
// 4096 tokens, 8 heads: 19.1 us with 1, 15.4 with 4, 16.9 with 9; 32 heads of 513 tokens: 11.2, 12.0, 15.8).
constexpr int kLeast = 4;
__device__ __forceinline__ int span_of(int len) { return len > 0 ? tiles_of(len) + kLead : 0; }
__device__ __forceinline__ int64_t spans_before(const AttendArgs& p, int upto) {
    const int lane = threadIdx.x & 31;
    int64_t sum = 0;
    for (int b = lane; b < upto; b += 32) sum += span_of(seq_len(p, b));
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
    __device__ __forceinline__ void next_group(const AttendArgs& p) {
        tile = 0;
        if (++group < p.H * p.row_tiles) return;
        enter(p, b + 1);
    }
    __device__ __forceinline__ bool same_group(const Cursor& o) const { return b == o.b && group == o.group; }
    // the first real unit at or behind place u, by a whole warp
    __device__ __forceinline__ void seek(const AttendArgs& p, int64_t u) {
        const int lane = threadIdx.x & 31;
        const int64_t per = static_cast<int64_t>(p.H) * p.row_tiles;
        int64_t base = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int mine = b0 + lane < p.B ? seq_len(p, b0 + lane) : 0;
            const int64_t n = span_of(mine);
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
                const int64_t span = tiles + kLead, before = base + __shfl_sync(0xFFFFFFFFu, incl, l) - span;
                const int64_t r = u - before * per;
                group = static_cast<int>(r / span);
                tile = max(0, static_cast<int>(r - group * span) - kLead);
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
__device__ __forceinline__ float max_nan(float a, float b) {          // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float over_tokens(float v) {          // maximum over the lanes that hold the same rows (lane & 3)
    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 4));
    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 8));
    return fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 16));
}
__device__ __forceinline__ float lg2(float x) {
    float r;
    asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float pow2i(int e) { return e < -126 ? 0.0f : __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
// (code + bias) in the low bits of fp16 1024, minus 1024 and the bias: exact
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t byte_pair(uint32_t w, uint32_t sel) { return hsub2(__byte_perm(w, 0x64646464u, sel), 0x64806480u); }
// (a & mask) ^ bits in one instruction, with both in registers
__device__ __forceinline__ uint32_t and_xor(uint32_t a, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
    return r;
}
__device__ __forceinline__ uint32_t nib_low(uint32_t w) { return hsub2(and_xor(w, 0x000F000Fu, 0x64086408u), 0x64086408u); }      // the flip of the sign bit included
__device__ __forceinline__ uint32_t nib_high(uint32_t w) {          // 16 (code + 8) in those bits: times 1 / 16, minus 1024 / 16 + 8
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(and_xor(w, 0x00F000F0u, 0x64806480u)), "r"(0x2C002C00u), "r"(0xD480D480u));
    return r;
}
__device__ __forceinline__ float unpack_half_lo(uint32_t h) { return __half2float(__ushort_as_half(static_cast<uint16_t>(h & 0xFFFFu))); }
__device__ __forceinline__ float unpack_half_hi(uint32_t h) { return __half2float(__ushort_as_half(static_cast<uint16_t>(h >> 16))); }
// two floats as fp16, and what that leaves of them
__device__ __forceinline__ uint32_t split_half2(float& lo, float& hi) {
    const uint32_t h = pack_half2(lo, hi);
    lo -= unpack_half_lo(h);
    hi -= unpack_half_hi(h);
    return h;
}
__device__ __forceinline__ void warps_barrier() { asm volatile("bar.sync 1, %0;" :: "n"(32 * kAttWarps) : "memory"); }   // computing warps

// 16-byte piece `c` of row `r` in a box of rows of RB bytes under the tensor map's swizzle of that width
template <int RB>
__device__ __forceinline__ uint32_t box_at(int r, int c) {
    if constexpr (RB == 128) return r * 128 + ((c ^ (r & 7)) << 4);
    else if constexpr (RB == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
    else return r * 32 + ((c ^ ((r >> 2) & 1)) << 4);
}

template <int D, int BITS, int NT, bool FINE>
struct AttendShape {
    static constexpr int kRow = D * BITS / 8;                   // bytes of a token's codes
    static constexpr int kTile = kUnit * kRow;                  // of a unit's keys or values
    static constexpr int kRows = 8 * NT;
    static constexpr int kPerSm = NT * D <= 128 ? 3 : 2;         // by the registers that results take
    static constexpr int kStages = D * BITS == 1024 ? (kPerSm == 2 ? 4 : 3) : (kPerSm == 3 ? 5 : 8);
    static constexpr int kPitch = D + 2;                        // floats of a joined row: pairs of lanes' stores meet two to a bank
    static constexpr size_t kSmem = 1024 + size_t(kStages) * (2 * kTile + 2 * kUnit * 4) + size_t(kRows) * D * (FINE ? 4 : 2) + size_t(2) * kRows * kPitch * 4;
};

// ---- units of a CTA -------------------------------------------------------------------------------
template <int D, int BITS, int NT, bool FINE>
__global__ void __launch_bounds__(kAttThreads, AttendShape<D, BITS, NT, FINE>::kPerSm)
k16_kv_attend(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const AttendArgs p) {
    using S = AttendShape<D, BITS, NT, FINE>;
    constexpr int RB = S::kRow, ST = S::kStages, KK = D / 16, MT = D / 16, ROWS = S::kRows, PITCH = S::kPitch;
    constexpr float kBias = BITS == 8 ? 128.0f : 8.0f;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* s_scale = reinterpret_cast<float*>(smem + ST * 2 * S::kTile);       // [stage][keys, values][64]
    uint4* s_q = reinterpret_cast<uint4*>(s_scale + ST * 2 * kUnit);           // [FINE: whole, rest][tile of rows][two steps][lane]
    float* s_o = reinterpret_cast<float*>(s_q + (FINE ? 2 : 1) * NT * (KK / 2) * 32);           // [2][ROWS][PITCH]
    __shared__ uint64_t full[ST], empty[ST];
    __shared__ unsigned s_boxes[ST];                                            // boxes of the unit that are there
    __shared__ __align__(16) float s_start[ROWS];                               // of the group's rows: start of logits' sums,
    __shared__ float s_fac[ROWS];                                               // their factor
    __shared__ int s_last[ROWS];                                                // and the last token that the row sees
    __shared__ float s_m[kAttWarps][ROWS], s_l[kAttWarps][ROWS], s_top[ROWS], s_sum[ROWS];
    __shared__ volatile uint32_t s_dead;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, r4 = lane & 3;

    asm volatile("griddepcontrol.launch_dependents;");
    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kAttWarps); }
        mbar_init_fence();
        s_dead = 0;
        prefetch_map(&mapK);
        prefetch_map(&mapV);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");         // launched while the kernel before it may still run
    const int64_t units = spans_before(p, p.B) * p.H * p.row_tiles;
    const int64_t parts = max(min((units + kLeast - 1) / kLeast, static_cast<int64_t>(gridDim.x)), int64_t(units > 0));
    Split* split = splits_of(p, gridDim.x, ROWS, D) + blockIdx.x;
    if (threadIdx.x == 0) *split = Split{0, 0, 0, 0};
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {        // sequences with nothing to attend to
        if (seq_len(p, b) > 0) continue;
        const int64_t row0 = static_cast<int64_t>(b) * p.Lq * p.Hq, rows = static_cast<int64_t>(p.Lq) * p.Hq;
        for (int64_t i = threadIdx.x; i < rows * D; i += kAttThreads) static_cast<uint16_t*>(p.out)[row0 * D + i] = 0;
        if (p.lse != nullptr)
            for (int64_t i = threadIdx.x; i < rows; i += kAttThreads) p.lse[row0 + i] = -INFINITY;
    }
    if (blockIdx.x >= parts) return;
    Cursor at, end;
    at.seek(p, part_start(units, blockIdx.x, parts));
    end.seek(p, part_start(units, blockIdx.x + 1, parts));
    __syncthreads();

    if (warp == kAttWarps) {
        // -- the loading warp: lane i takes the i-th box of a unit.  One warp's chain of dependent instructions for each unit is what
        //    it costs, so everything that a group shares is kept, and places advance by additions.
        const int nbox = kUnit / p.box;
        const int box_row = lane * p.box;
        const bool mine = lane < nbox;
        const uint32_t box_bytes = static_cast<uint32_t>(p.box) * (2 * RB + 8);
        bool ok = true;
        int stage = 0, issued = 0;
        uint32_t round = 0;                                    // parity of the stage's turn
        while (ok && at.b < p.B && !(at.same_group(end) && at.tile >= end.tile)) {
            const int n_units = (at.same_group(end) ? end.tile : at.tiles) - at.tile;
            const int* table = p.table + at.b * p.table_stride;
            const int head_row = (at.group / p.row_tiles) * p.page_size, page_rows = p.H * p.page_size;
            int tok = at.tile * kUnit + (mine ? box_row : 0);
            int idx = tok / p.page_size, off = tok - idx * p.page_size;
            int known_first = idx - 32, known_page = -1;       // lane i: page number known_first + i of the sequence
            for (int n = 0; n < n_units; ++n) {
                const int first = __shfl_sync(0xFFFFFFFFu, idx, 0);
                if (first + nbox > known_first + 32) {
                    known_first = first;
                    known_page = static_cast<int64_t>(first + lane) * p.page_size < at.len ? __ldcg(table + first + lane) : -1;
                }
                const int page = __shfl_sync(0xFFFFFFFFu, known_page, idx - known_first);
                const bool there = mine && tok < at.len && page >= 0 && page < p.pages;
                const unsigned boxes = __ballot_sync(0xFFFFFFFFu, there);
                if (!(ok = role_wait(&empty[stage], round ^ 1u, &s_dead))) break;
                if (lane == 0) {
                    s_boxes[stage] = boxes;
                    mbar_expect_tx(&full[stage], __popc(boxes) * box_bytes);
                }
                __syncwarp();
                if (there) {
                    const int row = page * page_rows + head_row + off;          // below 2^31
                    uint8_t* box = smem + stage * 2 * S::kTile + box_row * RB;
                    float* sc = s_scale + stage * 2 * kUnit + box_row;
                    tile_load(box, &mapK, 0, row, &full[stage]);
                    bulk_load(sc, p.scale[0] + row, p.box * 4, &full[stage]);
                    tile_load(box + S::kTile, &mapV, 0, row, &full[stage]);
                    bulk_load(sc + kUnit, p.scale[1] + row, p.box * 4, &full[stage]);
                }
                tok += kUnit;
                idx += p.unit_pages;
                off += p.unit_rest;
                if (off >= p.page_size) { off -= p.page_size; ++idx; }
                issued = min(issued + 1, ST);
                if (++stage == ST) { stage = 0; round ^= 1u; }
            }
            at.tile += n_units;
            if (at.tile >= at.tiles) at.next_group(p);
        }
        if (!ok)                                                // copies still in flight land before the CTA leaves
            for (; issued > 0; --issued) {
                if (--stage < 0) { stage = ST - 1; round ^= 1u; }
                for (uint32_t polls = 0; polls < (1u << 21) && !mbar_try(&full[stage], round); ++polls) {}
            }
        return;
    }

    // -- the computing warps
    const uint8_t* k_row = smem + warp * 16 * RB;               // this warp's tokens in a stage
    const int my_box = warp * 16 / p.box;
    int stage = 0;
    uint32_t round = 0;
    bool dead = false;
    while (at.b < p.B && !(at.same_group(end) && at.tile >= end.tile)) {
        // one group, or the part of it that lies in this CTA
        const int head = at.group / p.row_tiles, rt = at.group - head * p.row_tiles;
        const int first_tile = at.tile, tiles = at.tiles, len = at.len, b = at.b;
        const int n_units = (at.same_group(end) ? end.tile : tiles) - first_tile;
        const int R = p.G * p.Lq;
        // The queries as the products want them, once for all warps: tile nt of eight rows is warp nt's.  They stay in shared
        // memory (two steps of a lane in 16 bytes): registers for them would cost a resident CTA.
        if (warp < NT) {
            // this lane: a quarter of row g8, the elements that it meets in the keys
            const int row = rt * ROWS + warp * 8 + g8;
            const int i = row / p.G, g = row - i * p.G;
            const bool there = row < R;
            const uint16_t* src = static_cast<const uint16_t*>(p.q) + b * p.qb + i * p.ql + static_cast<int64_t>(head * p.G + g) * p.qh + r4 * (D / 4);
            const float* kcol = p.col[0] != nullptr ? p.col[0] + static_cast<int64_t>(head) * D + r4 * (D / 4) : nullptr;
            float v[D / 4];
            float top = 0.0f;
#pragma unroll
            for (int e = 0; e < D / 4; e += 4) {
                uint2 w = make_uint2(0, 0);
                if (there) {
                    if (p.q_vec) {
                        w = *reinterpret_cast<const uint2*>(src + e);
                    } else {
                        w.x = src[e] | (static_cast<uint32_t>(src[e + 1]) << 16);
                        w.y = src[e + 2] | (static_cast<uint32_t>(src[e + 3]) << 16);
                    }
                }
                const float2 lo = unpack16x2<FINE ? CQ_F16 : CQ_BF16>(w.x), hi = unpack16x2<FINE ? CQ_F16 : CQ_BF16>(w.y);
                v[e] = lo.x; v[e + 1] = lo.y; v[e + 2] = hi.x; v[e + 3] = hi.y;
                if (kcol != nullptr) {
                    const float4 c = *reinterpret_cast<const float4*>(kcol + e);
                    v[e] *= c.x; v[e + 1] *= c.y; v[e + 2] *= c.z; v[e + 3] *= c.w;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) top = fmaxf(top, fabsf(v[e + k]));
            }
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            // power of two that brings the largest element into [2^14, 2^15); within the range of a float both ways
            const int up_exp = top > 0.0f ? max(-100, min(100, 14 - (static_cast<int>(__float_as_uint(top) >> 23) - 127))) : 0;
            const float up = pow2i(up_exp);
            float sum = 0.0f;                                   // of the rounded elements, whichever units they are held in
#pragma unroll
            for (int k2 = 0; k2 < KK / 2; ++k2) {
                uint32_t f[4], rest[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // INT4: nibbles (0, 4 | 1, 5) of a word in even steps, (2, 6 | 3, 7) in odd ones; the second pair comes in sixteenfold
                    const int kk = 2 * k2 + h, e = BITS == 8 ? 4 * kk : k2 * 8 + h * 2;
                    float x[4] = {v[e], BITS == 8 ? v[e + 1] : v[e + 4], BITS == 8 ? v[e + 2] : v[e + 1], BITS == 8 ? v[e + 3] : v[e + 5]};
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const float unit = BITS == 4 && q == 1 ? 0.0625f : 1.0f;
                        float lo = x[2 * q] * up * unit, hi = x[2 * q + 1] * up * unit;
                        const uint32_t w = split_half2(lo, hi);
                        float both = unpack_half_lo(w) + unpack_half_hi(w);
                        f[2 * h + q] = w;
                        if constexpr (FINE) {
                            rest[2 * h + q] = pack_half2(lo, hi);
                            both += unpack_half_lo(rest[2 * h + q]) + unpack_half_hi(rest[2 * h + q]);
                        }
                        sum = __fmaf_rn(both, 1.0f / unit, sum);
                    }
                }
                s_q[(warp * (KK / 2) + k2) * 32 + lane] = make_uint4(f[0], f[1], f[2], f[3]);
                if constexpr (FINE) s_q[((NT + warp) * (KK / 2) + k2) * 32 + lane] = make_uint4(rest[0], rest[1], rest[2], rest[3]);
            }
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
            if (r4 == 0) {
                // codes come in as 2^-24; not 0, which times the -infinity of an unseen token would be NaN
                s_fac[warp * 8 + g8] = fmaxf(pow2i(-up_exp) * p.softmax_scale * (kLog2e * 16777216.0f), kLeastFac);
                s_start[warp * 8 + g8] = -sum * (kBias / 16777216.0f);
                s_last[warp * 8 + g8] = there ? len - p.Lq + i : -1;
            }
        }
        warps_barrier();
        float fac[NT][2];                                       // of rows 2 r4, 2 r4 + 1: factor of logits
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            fac[nt][0] = s_fac[nt * 8 + 2 * r4];
            fac[nt][1] = s_fac[nt * 8 + 2 * r4 + 1];
        }
        // results of channels g8 * D/8 + 2 t, + 1 (elements 0 1 | 2 3) and rows 2 r4, 2 r4 + 1
        float o[NT][MT][4], ref[NT][2], l[NT][2];               // ref: references, in base 2; below every logit where nothing was seen
        float unit[NT][2], finest = 1.0f;                      // powers of two: results are held in units of 1 / unit; the largest of this lane's
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            ref[nt][0] = ref[nt][1] = kNoRef;
            l[nt][0] = l[nt][1] = 0.0f;
            unit[nt][0] = unit[nt][1] = 1.0f;
#pragma unroll
            for (int t = 0; t < MT; ++t) o[nt][t][0] = o[nt][t][1] = o[nt][t][2] = o[nt][t][3] = 0.0f;
        }

        for (int n = 0; n < n_units; ++n) {
            if (!dead && !role_wait(&full[stage], round, &s_dead)) {
                dead = true;                                   // nothing is computed from here on
                if (lane == 0) atomicExch(&g_attn_fault, 1u);
            }
            const int tok0 = (first_tile + n) * kUnit + warp * 16;
            const int valid = len - tok0;                      // tokens from here to the end
            if (valid > 0 && !dead && ((s_boxes[stage] >> my_box) & 1u) != 0u) {
                const uint8_t* kbox = k_row + stage * 2 * S::kTile;
                const uint8_t* vbox = kbox + S::kTile;
                const float* sc = s_scale + stage * 2 * kUnit + warp * 16;
                // -- logits of tokens g8 (elements 0 1) and g8 + 8 (2 3), rows 2 r4, 2 r4 + 1
                float s[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float2 first = *reinterpret_cast<const float2*>(s_start + nt * 8 + 2 * r4);
                    s[nt][0] = s[nt][2] = first.x;
                    s[nt][1] = s[nt][3] = first.y;
                }
                constexpr int kWords = RB / 16;                // words of a lane and token: a quarter of the row
                uint32_t w[2][kWords], qf[(FINE ? 2 : 1) * NT][2][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (kWords >= 4) {
#pragma unroll
                        for (int c = 0; c < kWords / 4; ++c) {
                            const uint4 t = *reinterpret_cast<const uint4*>(kbox + box_at<RB>(h * 8 + g8, r4 * (kWords / 4) + c));
                            w[h][4 * c] = t.x; w[h][4 * c + 1] = t.y; w[h][4 * c + 2] = t.z; w[h][4 * c + 3] = t.w;
                        }
                    } else {
                        const uint2 t = *reinterpret_cast<const uint2*>(kbox + box_at<RB>(h * 8 + g8, r4 >> 1) + (r4 & 1) * 8);
                        w[h][0] = t.x; w[h][1] = t.y;
                    }
                }
#pragma unroll
                for (int j = 0; j < kWords; ++j) {
                    if constexpr (BITS == 8) {
                        if ((j & 1) == 0) {
#pragma unroll
                            for (int nt = 0; nt < (FINE ? 2 : 1) * NT; ++nt) {
                                const uint4 t = s_q[(nt * (KK / 2) + j / 2) * 32 + lane];
                                qf[nt][0][0] = t.x; qf[nt][0][1] = t.y; qf[nt][1][0] = t.z; qf[nt][1][1] = t.w;
                            }
                        }
                        const uint32_t x0 = w[0][j] ^ 0x80808080u, x1 = w[1][j] ^ 0x80808080u;         // two's complement -> biased
                        const uint32_t a0 = __byte_perm(x0, 0, 0x4140), a1 = __byte_perm(x1, 0, 0x4140);
                        const uint32_t a2 = __byte_perm(x0, 0, 0x4342), a3 = __byte_perm(x1, 0, 0x4342);
#pragma unroll
                        for (int nt = 0; nt < (FINE ? 2 : 1) * NT; ++nt) mma16816(s[nt % NT], a0, a1, a2, a3, qf[nt][j & 1]);
                    } else {
#pragma unroll
                        for (int nt = 0; nt < (FINE ? 2 : 1) * NT; ++nt) {
                            const uint4 t = s_q[(nt * (KK / 2) + j) * 32 + lane];
                            qf[nt][0][0] = t.x; qf[nt][0][1] = t.y; qf[nt][1][0] = t.z; qf[nt][1][1] = t.w;
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t y0 = w[0][j] >> (8 * h), y1 = w[1][j] >> (8 * h);
                            const uint32_t a0 = and_xor(y0, 0x000F000Fu, 0x00080008u), a1 = and_xor(y1, 0x000F000Fu, 0x00080008u);
                            const uint32_t a2 = and_xor(y0, 0x00F000F0u, 0x00800080u), a3 = and_xor(y1, 0x00F000F0u, 0x00800080u);
#pragma unroll
                            for (int nt = 0; nt < (FINE ? 2 : 1) * NT; ++nt) mma16816(s[nt % NT], a0, a1, a2, a3, qf[nt][h]);
                        }
                    }
                }
                // -- probabilities
                // an infinite key scale goes in as NaN: a head that held an infinity has codes 0, whose sum is 0 up to a rounding of
                // either sign, and times the infinity that would be NaN or a token without probability as it falls
                const float ka[2] = {__fmaf_rn(sc[g8], 0.0f, sc[g8]), __fmaf_rn(sc[g8 + 8], 0.0f, sc[g8 + 8])};
                float va[2] = {sc[kUnit + g8], sc[kUnit + g8 + 8]};
                if (g8 >= valid) va[0] = 0.0f;                 // what lies past the end may be anything
                if (g8 + 8 >= valid) va[1] = 0.0f;
                const bool edge = tok0 + 15 > len - p.Lq;      // some row does not see some token
                float x[NT][2][2];                             // [row][token]: logits in units of fac
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        x[nt][e][0] = s[nt][e] * ka[0];
                        x[nt][e][1] = s[nt][2 + e] * ka[1];
                    }
                if (edge) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int last = s_last[nt * 8 + 2 * r4 + e];
                            if (tok0 + g8 > last) x[nt][e][0] = -INFINITY;
                            if (tok0 + g8 + 8 > last) x[nt][e][1] = -INFINITY;
                        }
                }
                // a product with fac is rounded once, as the reference, and used for all that refers to it: its rounding cancels
                float pr[NT][2][2], most = 0.0f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        pr[nt][e][0] = ex2(__fmaf_rn(x[nt][e][0], fac[nt][e], -ref[nt][e]));
                        pr[nt][e][1] = ex2(__fmaf_rn(x[nt][e][1], fac[nt][e], -ref[nt][e]));
                        most = fmaxf(most, fmaxf(pr[nt][e][0], pr[nt][e][1]));
                    }
                float pv[NT][2][2];                            // probability times va, in the row's units
                if (__any_sync(0xFFFFFFFFu, most > kMostProb || !(max_nan(fabsf(va[0]), fabsf(va[1])) * finest * most <= kMostUnits))) {
                    // Perhaps new references and units, for the rows that need them; a va that is not finite comes here too.
                    // All rows at once, so that their shuffles overlap; a row that needs nothing is multiplied by 1.
                    const unsigned row = 0x11111111u << r4;    // the lanes of this lane's rows
                    const float lv[2] = {lg2(fabsf(va[0])), lg2(fabsf(va[1]))};
                    float top[NT][2], heavy[NT][2];            // in base 2: the largest logit, the largest probability times va
                    unsigned asks = 0;
                    finest = 0.0f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float most_units = 0.0f;
                            heavy[nt][e] = -INFINITY;
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                if (x[nt][e][k] != -INFINITY) {
                                    most_units = fmaxf(most_units, fabsf(pr[nt][e][k] * va[k] * unit[nt][e]));
                                    heavy[nt][e] = fmaxf(heavy[nt][e], __fmaf_rn(x[nt][e][k], fac[nt][e], lv[k]));
                                }
                            const bool high = fmaxf(pr[nt][e][0], pr[nt][e][1]) > kMostProb;
                            if ((__ballot_sync(0xFFFFFFFFu, high) & row) != 0u) asks |= 3u << (4 * nt + 2 * e);
                            if ((__ballot_sync(0xFFFFFFFFu, most_units > kMostUnits) & row) != 0u) asks |= 1u << (4 * nt + 2 * e);
                            top[nt][e] = __fmul_rn(over_tokens(fmaxf(x[nt][e][0], x[nt][e][1])), fac[nt][e]);
                            heavy[nt][e] = over_tokens(heavy[nt][e]);
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const unsigned ask = (asks >> (4 * nt + 2 * e)) & 3u;
                            // whole numbers, so that no bits are lost; `held`: what the row's results are held under, with the new reference
                            const float next = (ask & 2u) != 0u ? ceilf(top[nt][e]) : ref[nt][e], fall = ref[nt][e] - next;
                            const int had = static_cast<int>(__float_as_uint(unit[nt][e]) >> 23) - 127;
                            const float held = static_cast<float>(kPlace - had) + fall, need = floorf(heavy[nt][e] - next) + 1.0f;
                            const int now = ask != 0u ? static_cast<int>(fminf(fmaxf(kPlace - fmaxf(held, need), -116.0f), 110.0f)) : had;
                            const float keep = ex2(fall + static_cast<float>(now - had));
                            unit[nt][e] = pow2i(now);
                            finest = fmaxf(finest, unit[nt][e]);
                            ref[nt][e] = next;
                            l[nt][e] *= ex2(fall);
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                pr[nt][e][k] = ex2(__fmaf_rn(x[nt][e][k], fac[nt][e], -next));
                                pv[nt][e][k] = x[nt][e][k] == -INFINITY ? 0.0f : pr[nt][e][k] * va[k] * unit[nt][e];
                            }
#pragma unroll
                            for (int t = 0; t < MT; ++t) {
                                o[nt][t][e] *= keep;
                                o[nt][t][2 + e] *= keep;
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            pv[nt][e][0] = pr[nt][e][0] * va[0] * unit[nt][e];
                            pv[nt][e][1] = pr[nt][e][1] * va[1] * unit[nt][e];
                        }
                }
                uint32_t pf[(FINE ? 2 : 1) * NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    l[nt][0] += pr[nt][0][0] + pr[nt][0][1];
                    l[nt][1] += pr[nt][1][0] + pr[nt][1][1];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        if constexpr (FINE) {
                            pf[nt][k] = transpose8x8(split_half2(pv[nt][0][k], pv[nt][1][k]));
                            pf[NT + nt][k] = transpose8x8(pack_half2(pv[nt][0][k], pv[nt][1][k]));
                        } else {
                            pf[nt][k] = transpose8x8(pack_half2(pv[nt][0][k], pv[nt][1][k]));
                        }
                    }
                }
                // -- results
                constexpr int kVWords = RB / 32;               // words of a lane and token: an eighth of the row
                uint32_t z[4][kVWords];                        // tokens 2 r4, 2 r4 + 1, 2 r4 + 8, 2 r4 + 9
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = 2 * r4 + (k & 1) + (k >> 1) * 8;
                    if constexpr (kVWords == 4) {
                        const uint4 t = *reinterpret_cast<const uint4*>(vbox + box_at<RB>(row, g8));
                        z[k][0] = t.x; z[k][1] = t.y; z[k][2] = t.z; z[k][3] = t.w;
                    } else if constexpr (kVWords == 2) {
                        const uint2 t = *reinterpret_cast<const uint2*>(vbox + box_at<RB>(row, g8 >> 1) + (g8 & 1) * 8);
                        z[k][0] = t.x; z[k][1] = t.y;
                    } else {
                        z[k][0] = *reinterpret_cast<const uint32_t*>(vbox + box_at<RB>(row, g8 >> 2) + (g8 & 3) * 4);
                    }
                }
#pragma unroll
                for (int j = 0; j < kVWords; ++j) {
                    uint32_t x[2][2];                          // [tokens +0, +8][half of the word]: the two tokens' bytes side by side
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t flip = BITS == 8 ? 0x80808080u : 0u;
                        const uint32_t a = z[2 * k][j] ^ flip, c = z[2 * k + 1][j] ^ flip;
                        x[k][0] = __byte_perm(a, c, BITS == 8 ? 0x5140 : 0x5410);
                        x[k][1] = __byte_perm(a, c, BITS == 8 ? 0x7362 : 0x7632);
                    }
                    if constexpr (BITS == 8) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t a0 = byte_pair(x[0][e], 0x4140), a1 = byte_pair(x[0][e], 0x4342);
                            const uint32_t a2 = byte_pair(x[1][e], 0x4140), a3 = byte_pair(x[1][e], 0x4342);
#pragma unroll
                            for (int nt = 0; nt < (FINE ? 2 : 1) * NT; ++nt) mma16816(o[nt % NT][2 * j + e], a0, a1, a2, a3, pf[nt]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t lo = (e & 1) ? x[0][e >> 1] >> 8 : x[0][e >> 1], hi = (e & 1) ? x[1][e >> 1] >> 8 : x[1][e >> 1];
                            const uint32_t a0 = nib_low(lo), a1 = nib_high(lo), a2 = nib_low(hi), a3 = nib_high(hi);
#pragma unroll
                            for (int nt = 0; nt < (FINE ? 2 : 1) * NT; ++nt) mma16816(o[nt % NT][4 * j + e], a0, a1, a2, a3, pf[nt]);
                        }
                    }
                }
            }
            __syncwarp();                                      // the stage has been read by every lane
            if (lane == 0) mbar_arrive(&empty[stage]);
            if (++stage == ST) { stage = 0; round ^= 1u; }
        }
        const bool here_ends = first_tile + n_units == tiles;
        if (here_ends) at.next_group(p);
        else at.tile = first_tile + n_units;

        // -- join the four warps: maxima and sums first, then results (warps 0 and 1 store, 2 and 3 add to them)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][e], 4);
                l[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][e], 8);
                l[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][e], 16);
                if (l[nt][e] == 0.0f) ref[nt][e] = -INFINITY;   // has seen nothing
                if (g8 == 0) {
                    s_m[warp][nt * 8 + 2 * r4 + e] = ref[nt][e];
                    s_l[warp][nt * 8 + 2 * r4 + e] = l[nt][e];
                }
            }
        warps_barrier();
        const int rows = min(ROWS, R - rt * ROWS);
        if (threadIdx.x < ROWS) {
            const int row = threadIdx.x;
            const float top = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
            const float ref = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttWarps; ++w) sum += s_l[w][row] * ex2(s_m[w][row] - ref);
            s_top[row] = top;
            s_sum[row] = sum;
        }
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
            if ((warp >> 1) == pass) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = nt * 8 + 2 * r4 + e;
                        if (row < rows) {
                            const float top = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
                            const float f = ex2(ref[nt][e] - (top == -INFINITY ? 0.0f : top)) * __uint_as_float((254u << 23) - __float_as_uint(unit[nt][e]));
                            float* dst = s_o + (warp & 1) * ROWS * PITCH + row * PITCH + g8 * (D / 8);
#pragma unroll
                            for (int t = 0; t < MT; ++t) {
                                float2 v = make_float2(o[nt][t][e] * f, o[nt][t][2 + e] * f);
                                float2* at2 = reinterpret_cast<float2*>(dst + 2 * t);
                                if (pass == 1) { const float2 w2 = *at2; v.x += w2.x; v.y += w2.y; }
                                *at2 = v;
                            }
                        }
                    }
            }
            warps_barrier();
        }
        const bool whole = first_tile == 0 && here_ends;
        const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (first_tile == 0 ? 1 : 0);
        if (first_tile == 0 && !here_ends && threadIdx.x == 0) {               // begins here: at most one group does, the last
            const int64_t place = part_start(units, blockIdx.x + 1, parts);
            // the group's last place is as far behind this part's end as its tiles that are left
            const int64_t last = place + (tiles - (first_tile + n_units)) - 1;
            *split = Split{b, head * p.row_tiles + rt, static_cast<int>(part_of(units, last, parts) - blockIdx.x) + 1, 0};
        }
        for (int idx = threadIdx.x; idx < rows * D; idx += 32 * kAttWarps) {
            const int row = idx / D, d = idx % D;
            const float top = s_top[row], sum = s_sum[row];
            const float v = s_o[row * PITCH + d] + s_o[(ROWS + row) * PITCH + d];
            if (whole) {
                const int rr = rt * ROWS + row, i = rr / p.G, g = rr - i * p.G;
                const int64_t dst = (static_cast<int64_t>(b) * p.Lq + i) * p.Hq + head * p.G + g;
                float res = sum == 0.0f ? 0.0f : __fdiv_rn(v, sum);
                if (p.col[1] != nullptr) res *= __ldcg(p.col[1] + static_cast<int64_t>(head) * D + d);
                static_cast<uint16_t*>(p.out)[dst * D + d] = pack16<FINE ? CQ_F16 : CQ_BF16>(res);
                if (p.lse != nullptr && d == 0) p.lse[dst] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
            } else {
                p.part[(slot * ROWS + row) * D + d] = v;
                if (d < 2) p.part[2 * static_cast<int64_t>(gridDim.x) * ROWS * D + (slot * ROWS + row) * 2 + d] = d == 0 ? top : sum;
            }
        }
        warps_barrier();
    }
}

// ---- join of groups that lie in several CTAs: one block for a CTA's split group and one of its rows ----------
// Maxima and weights of all parts first, then the parts' results, dealt out to the block's D-wide teams and added in a
// fixed order.  (A loop over the parts in one team took 20 us for one sequence of 4096 tokens, cut into 55 parts a head.)
constexpr int kJoinThreads = 256;
constexpr int kJoinParts = 1024;                                // more than CTAs that can be resident

template <int D, int DT>
__global__ void __launch_bounds__(kJoinThreads)
k17_kv_join(const AttendArgs p, int ctas, int rows_per_tile) {
    constexpr int kTeams = kJoinThreads / D;
    __shared__ float s_w[kJoinParts], s_red[kJoinThreads / 32], s_v[kTeams][D];
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 at = __ldcg(reinterpret_cast<const int4*>(splits_of(p, ctas, rows_per_tile, D) + blockIdx.x));
    const Split sp{at.x, at.y, at.z, at.w};
    const int head = sp.group / p.row_tiles, rt = sp.group - head * p.row_tiles;
    const int row = blockIdx.y, r = rt * rows_per_tile + row;
    if (sp.parts == 0 || r >= p.G * p.Lq) return;
    const int n = min(sp.parts, kJoinParts), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float* stats = p.part + 2 * static_cast<int64_t>(ctas) * rows_per_tile * D;
    auto slot = [&](int k) { return (2 * (static_cast<int64_t>(blockIdx.x) + k) + (k == 0 ? 1 : 0)) * rows_per_tile + row; };
    auto over_block = [&](float v, bool sum) {                  // maximum or sum over the block, in a fixed order
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float o = __shfl_xor_sync(0xFFFFFFFFu, v, off);
            v = sum ? v + o : fmaxf(v, o);
        }
        __syncthreads();
        if (lane == 0) s_red[warp] = v;
        __syncthreads();
        v = s_red[0];
#pragma unroll
        for (int w = 1; w < kJoinThreads / 32; ++w) v = sum ? v + s_red[w] : fmaxf(v, s_red[w]);
        return v;
    };
    float top = -INFINITY;
    for (int k = threadIdx.x; k < n; k += kJoinThreads) {
        const float m = __ldcg(stats + slot(k) * 2);
        s_w[k] = m;
        top = fmaxf(top, m);
    }
    top = over_block(top, false);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
    for (int k = threadIdx.x; k < n; k += kJoinThreads) {
        const float f = ex2(s_w[k] - ref);
        s_w[k] = f;
        sum = __fmaf_rn(__ldcg(stats + slot(k) * 2 + 1), f, sum);
    }
    sum = over_block(sum, true);                                // (its barriers also publish the weights)
    const int d = threadIdx.x % D, team = threadIdx.x / D;
    float v = 0.0f;
#pragma unroll 8
    for (int k = team; k < n; k += kTeams) v = __fmaf_rn(__ldcg(p.part + slot(k) * D + d), s_w[k], v);
    s_v[team][d] = v;
    __syncthreads();
    if (team != 0) return;
#pragma unroll
    for (int t = 1; t < kTeams; ++t) v += s_v[t][d];
    const int i = r / p.G, g = r - i * p.G;
    const int64_t row_id = (static_cast<int64_t>(sp.b) * p.Lq + i) * p.Hq + head * p.G + g;
    float res = sum == 0.0f ? 0.0f : __fdiv_rn(v, sum);
    if (p.col[1] != nullptr) res *= __ldcg(p.col[1] + static_cast<int64_t>(head) * D + d);
    static_cast<uint16_t*>(p.out)[row_id * D + d] = pack16<DT>(res);
    if (p.lse != nullptr && d == 0) p.lse[row_id] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// ---- host ---------------------------------------------------------------------------------------------
constexpr int kMaxPerSm = 3;

int attn_stage_fault(unsigned int* fault_host) {
    return cudaMemcpyFromSymbol(fault_host, g_attn_fault, sizeof(unsigned int)) == cudaSuccess ? CQ_OK : CQ_ERR_CUDA;
}

static size_t attend_workspace(int64_t D) {
    return static_cast<size_t>(sm_count()) * kMaxPerSm * (2 * 32 * (D + 2) * sizeof(float) + sizeof(Split));
}

template <int D, int BITS, int NT, bool FINE>
static int launch_attend(AttendArgs& p, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t st) {
    using S = AttendShape<D, BITS, NT, FINE>;
    static thread_local LaunchMemo memo;
    // (the static shared memory counts towards the 48 KB that need no leave, so leave is asked for in any case)
    int per_sm = resident_ctas(k16_kv_attend<D, BITS, NT, FINE>, kAttThreads, S::kSmem, S::kSmem > 50000 ? S::kSmem : 50000, memo);
    if (per_sm < 1) return CQ_ERR_CUDA;
    if (per_sm > kMaxPerSm) per_sm = kMaxPerSm;
    p.row_tiles = (p.G * p.Lq + S::kRows - 1) / S::kRows;
    int64_t ctas = static_cast<int64_t>(sm_count()) * per_sm;
    const int64_t most = static_cast<int64_t>(p.B) * p.H * p.row_tiles * ((p.capacity + kUnit - 1) / kUnit);       // real units
    if (ctas > most) ctas = most;
    const int rc = launch_ex(k16_kv_attend<D, BITS, NT, FINE>, dim3(static_cast<unsigned>(ctas)), kAttThreads, S::kSmem, st, 1, !tuning_no_pdl(), mapK, mapV, p);
    if (rc != CQ_OK) return rc;
    const int rows = p.G * p.Lq < S::kRows ? p.G * p.Lq : S::kRows;
    return launch_ex(k17_kv_join<D, FINE ? CQ_F16 : CQ_BF16>, dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(rows)), kJoinThreads, 0, st, 1, !tuning_no_pdl(),
                     p, static_cast<int>(ctas), S::kRows);
}

// Rows beyond 16 of 128 channels go into further tiles of 16: registers for 32 would leave one CTA an SM (16 sequences of
// 4000 tokens, 32 rows a head: 84 us with one tile of 32).
template <int D, int BITS, bool FINE>
static int launch_attend_rows(AttendArgs& p, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t st) {
    const int R = p.G * p.Lq;
    if (R <= 8) return launch_attend<D, BITS, 1, FINE>(p, mapK, mapV, st);
    if (R <= 16 || D == 128) return launch_attend<D, BITS, 2, FINE>(p, mapK, mapV, st);
    if constexpr (D == 64) {
        if (R <= 24) return launch_attend<D, BITS, 3, FINE>(p, mapK, mapV, st);
        return launch_attend<D, BITS, 4, FINE>(p, mapK, mapV, st);
    }
    return CQ_ERR_SHAPE;
}

// Every row empty, when no token can be named.
__global__ void k18_no_tokens(uint16_t* out, float* lse, int64_t rows, int D) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < rows * D; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        out[i] = 0;
        if (lse != nullptr && i < rows) lse[i] = -INFINITY;
    }
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
    p.box = page_size % 64 == 0 ? 64 : page_size % 32 == 0 ? 32 : 16;
    p.unit_pages = static_cast<int>(kUnit / page_size);
    p.unit_rest = static_cast<int>(kUnit % page_size);
    p.out = out; p.lse = lse; p.part = static_cast<float*>(workspace);
    p.softmax_scale = static_cast<float>(softmax_scale);
    p.pages = pages; p.B = static_cast<int>(B); p.Lq = static_cast<int>(Lq); p.Hq = static_cast<int>(Hq); p.H = static_cast<int>(H);
    p.G = static_cast<int>(Hq / H); p.page_size = static_cast<int>(page_size);
    p.row_tiles = 1;
    p.capacity = pages > 0 ? table_width * page_size : 0;
    if (p.capacity == 0) {                                      // no token can be named: every row is empty
        const int64_t rows = B * Lq * Hq;
        k18_no_tokens<<<static_cast<unsigned>(rows < 4096 ? rows : 4096), 128, 0, st>>>(static_cast<uint16_t*>(out), lse, rows, static_cast<int>(D));
        return launch_status();
    }
    const uint32_t row_bytes = static_cast<uint32_t>(D * bits / 8);
    const CUtensorMapSwizzle swizzle = row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : row_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
    const uint64_t rows = static_cast<uint64_t>(pages) * H * page_size;
    CUtensorMap mapK, mapV;
    if (!make_byte_map(&mapK, k_codes, row_bytes, rows, row_bytes, row_bytes, p.box, swizzle) ||
        !make_byte_map(&mapV, v_codes, row_bytes, rows, row_bytes, row_bytes, p.box, swizzle)) return CQ_ERR_CUDA;
    const bool fine = dtype == CQ_F16;
    if (D == 128) {
        if (bits == 8) return fine ? launch_attend_rows<128, 8, true>(p, mapK, mapV, st) : launch_attend_rows<128, 8, false>(p, mapK, mapV, st);
        return fine ? launch_attend_rows<128, 4, true>(p, mapK, mapV, st) : launch_attend_rows<128, 4, false>(p, mapK, mapV, st);
    }
    if (bits == 8) return fine ? launch_attend_rows<64, 8, true>(p, mapK, mapV, st) : launch_attend_rows<64, 8, false>(p, mapK, mapV, st);
    return fine ? launch_attend_rows<64, 4, true>(p, mapK, mapV, st) : launch_attend_rows<64, 4, false>(p, mapK, mapV, st);
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
