// Layout of the quantized key/value cache, shared by the kernels that write, read and attend over it.
//
// A cache of pages holds, for keys and values each,
//   codes  int8 [pages][H][page_size][D]  (INT4: two per byte, [D / 2], element 2k in the low nibble)
//   scale  float [pages][H][page_size]
// and, optional, a channel factor float [H][D] that all tokens share.  Token slot n = page * page_size + offset.
// An element stands for code * (scale * factor): the CrossQuant form (row factor times column factor) with the
// row = one token's head, so either factor leaves the sums of the attention as a whole.
#pragma once

#include "cq_serve.cuh"

namespace cq {

struct KvCache {
    const int8_t* codes[2];      // keys, values
    const float* scale[2];
    const float* col[2];         // null: ones
    int64_t pages;
    int page_size, H, D;
};

int check_cache(const void* k_codes, const void* v_codes, const void* k_scale, const void* v_scale, const void* k_col,
                const void* v_col, int bits, int64_t pages, int64_t page_size, int64_t H, int64_t D);

}  // namespace cq
