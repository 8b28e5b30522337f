// What the kernels over packed sequences and paged caches share.
#pragma once
#include "conv_common.h"

namespace cw {

// The last s of [0, sequences) with at(s) <= what, for at() that does not fall; 0 where none is.  All 64 lanes of a wave, a step for 64 candidates.
template <typename F>
__device__ static inline int last_not_above(int sequences, int64_t what, F at) {
    const int lane = threadIdx.x & 63;
    int low = 0, high = sequences;
    while (high - low > 1) {
        const int step = (high - low + 63) >> 6, i = low + lane * step;
        const int c = __popcll(__ballot(i < high && at(i) <= what));
        low += (c > 1 ? c - 1 : 0) * step;
        high = low + step < high ? low + step : high;
    }
    return __builtin_amdgcn_readfirstlane(low);
}

// Page of token t of a sequence, or -1.
__device__ static inline int page_of(const CacheView &c, const int32_t *table, int table_pages, int t) {
    const int at = t >> c.page_shift;
    if (t < 0 || at >= table_pages) return -1;
    const int page = table[at];
    return (unsigned)page < (unsigned)c.pages ? page : -1;
}

// e4m3 to fp32: exact.
__device__ static inline void decode4(unsigned codes, float *to) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    to[0] = a[0]; to[1] = a[1]; to[2] = b[0]; to[3] = b[1];
}

}  // namespace cw
