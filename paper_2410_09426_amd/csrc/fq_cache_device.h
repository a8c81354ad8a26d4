// What the kernels of the paged key/value cache share.
#pragma once
#include "fq_internal.h"

namespace fq {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ half2v as_half2(uint32_t x) { return __builtin_bit_cast(half2v, x); }
__device__ __forceinline__ uint32_t as_u32(half2v x) { return __builtin_bit_cast(uint32_t, x); }

// Place of row t of head `head` in the code and parameter arrays, counted in rows; NO_TOKEN if its token has none, NO_ROW if t is no row of the batch.
// The first guess is where the row would lie if all sequences had the same number of rows (a decode step: it is right); then bisection.
constexpr int64_t NO_TOKEN = -1, NO_ROW = -2;
__device__ __forceinline__ int64_t token_place(const CacheDev& c, int64_t t, int head) {
    if (t >= c.T) return NO_ROW;
    int lo = 0, hi = c.B - 1;                                   // the sequence is the last one that starts at t or before and has rows
    const int guess = min(hi, (int)((float)t * ((float)c.B / (float)c.T)));
    if (c.row_starts[guess] <= t && t < c.row_starts[guess + 1]) {
        lo = guess;
    } else {
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (c.row_starts[mid] <= t) lo = mid;
            else hi = mid - 1;
        }
    }
    const int64_t first = c.row_starts[lo], last = c.row_starts[lo + 1];
    if (t < first || t >= last) return NO_ROW;                  // padding behind the last sequence
    const int64_t pos = c.lengths[lo] - (last < c.T ? last : c.T) + t;
    if (pos < 0) return NO_TOKEN;
    const int64_t j = pos >> c.page_shift;
    if (j >= c.table_width) return NO_TOKEN;
    const int page = c.page_table[lo * c.table_stride + j];
    if (page < 0 || page >= c.pages) return NO_TOKEN;
    return (((int64_t)page * c.H + head) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

}  // namespace fq
