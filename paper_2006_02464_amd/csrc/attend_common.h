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

// Of cw_attend.
constexpr int kAttendWaves = 4;
constexpr int attend_rows(int split) { return 32 * kAttendWaves / split; }   // of a workgroup, whose waves share rows `split` at a time
inline int64_t attend_workgroups(const AttendArgs &a) { return (int64_t)a.tokens * a.heads / attend_rows(1) + (int64_t)a.sequences * a.kv_heads; }   // that share none, and a few more

// Of cw_attend_one.
constexpr int kOneHeads = 16, kOneWaves = 4;
constexpr int one_tokens(int row_bytes) { return row_bytes > 256 ? 16 : 32; }   // of a step: 16 KB at most

// How a call is cut: into items, sequences and blocks of heads, of so many tokens and steps at most.
struct OneForm {
    int row_bytes;                  // in LDS
    int64_t items, tokens, steps;
    int64_t slots;                  // workgroups of four waves that run at once, as LDS has it
    bool wave_each;                 // of an item; else workgroups of four waves
};
inline OneForm one_form(const AttendOneArgs &a) {
    const bool codes = a.cache.dtype == DT_E4M3;
    const int bytes = a.cache.head_dim * (codes ? 1 : 2);
    int row_bytes = codes ? 64 : 128;
    while (row_bytes < bytes) row_bytes *= 2;
    const int tokens_a_step = one_tokens(row_bytes);
    OneForm f{row_bytes, (int64_t)a.sequences * ((a.heads / a.cache.kv_heads + kOneHeads - 1) / kOneHeads) * a.cache.kv_heads, (int64_t)a.table_pages << a.cache.page_shift, 0,
              2 * kOneWaves * (2 * tokens_a_step * row_bytes + 256) > 80 * 1024 ? 256 : 512, false};
    if (a.window > 0 && f.tokens > (int64_t)a.window + tokens_a_step - 1) f.tokens = (int64_t)a.window + tokens_a_step - 1;
    f.steps = (f.tokens + tokens_a_step - 1) / tokens_a_step;
    // Many items of few tokens get a wave each: 200 of 30 to 150, 8 heads of 128 18.5 us for 28.8, 150 of 30 to 300 29.5 for 34.1, 40 of 3 to 30 5.0 for 8.2; but 34 of 30 to 300 (272 items) 14.1 for 10.0, 60 of 30 to 400 17.6 for 14.8.
    f.wave_each = f.items > f.slots && (f.tokens <= 128 || (f.tokens <= 320 && f.items > 2 * f.slots));
    return f;
}

}  // namespace cw
