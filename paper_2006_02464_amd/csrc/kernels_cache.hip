// Tokens' keys and values to the pages of a cache and back (cw_cache_write and cw_cache_read have the definitions).
#include <algorithm>
#include <cmath>

#include "attend_common.h"

namespace cw {

// Nothing but moving bytes.  A row is a token's keys or values of one head; its lanes are a power of two, 8 numbers each, so that its largest magnitude is a few exchanges
// away.  A wave takes a run of rows, kCacheBatch times 64 lanes of them under way at once: first a lane for each of its tokens finds the token's sequence, page and place, which takes trips to
// memory that wait for one another, then the rows follow one another.  HBM bounds it: 34 k tokens of 8 heads of 128 fp16 to e4m3 in 43.5 us (4.9 TB/s; a copy of 1 GiB reaches 5.1), of 16 bits to 16 bits in 52 either way
// (5.4); back from e4m3 in 59 to 61 (3.5 TB/s), or 38 where what is read and written lies in the last level's cache.  fp32 rows: to e4m3 78 us (4.5 TB/s; 168 registers a lane where 16-bit rows take 64), to 16 bits 76, back 91 and 93.  A row at a time was
// slower: 49 for 43.  Stores go past the caches: what they would keep there is what the reads need (back from e4m3 64 us otherwise, from 16 bits 56).
constexpr int kCacheWaves = 4, kCacheBatch = 4;

struct CacheKernel {
    CacheArgs a;
    FastDiv by_rows;             // rows of a token
    int32_t lanes, lane_shift;   // of a row
    int32_t passes;              // of a wave, 64 lanes of rows each
};

template <typename T>
__device__ static inline void load8(const T *from, float (&x)[8]) {
    typedef T T8 __attribute__((ext_vector_type(8)));
    const T8 v = *reinterpret_cast<const T8 *>(from);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
template <typename T>
__device__ static inline void store8(T *to, const float (&x)[8]) {
    typedef T T8 __attribute__((ext_vector_type(8)));
    T8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
    __builtin_nontemporal_store(v, reinterpret_cast<T8 *>(to));
}

// The least e from -127 on with largest <= 448 * 2^e, for the bits of a finite largest; 448 = 1.75 * 2^8.
__device__ static inline int exponent_for(unsigned bits) {
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return e < -127 ? -127 : e;
}

// Bits of the largest magnitude of eight numbers, as of fp32: at least those of infinity where one is none.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
template <typename T8>
__device__ static inline unsigned largest_of(const T8 &x) {
    if constexpr (sizeof(x) == 16) {
        const u32x4 w = __builtin_bit_cast(u32x4, x) & 0x7fff7fffu;
        const unsigned w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3];
        const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(u16x2, w0), __builtin_bit_cast(u16x2, w1)),
                                                  __builtin_elementwise_max(__builtin_bit_cast(u16x2, w2), __builtin_bit_cast(u16x2, w3)));
        const unsigned short most = m[0] > m[1] ? m[0] : m[1];
        if constexpr (std::is_same<decltype(x[0] + x[0]), f16>::value) return __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(f16, most));
        else return (unsigned)most << 16;
    } else {
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = x[i];
            const unsigned bits = __builtin_bit_cast(unsigned, v) & 0x7fffffffu;
            most = most > bits ? most : bits;
        }
        return most;
    }
}
// Of the lanes of a row, a power of two from 2 to 32, in all of them.
__device__ static inline unsigned of_row(unsigned v, int lanes) {
    auto larger = [](unsigned p, unsigned q) { return p > q ? p : q; };
    auto dpp = [](unsigned x, auto control) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(control)::value, 0xf, 0xf, false); };
    v = larger(v, dpp(v, std::integral_constant<int, 0xB1>{}));                       // lanes 1 0 3 2
    if (lanes > 2) v = larger(v, dpp(v, std::integral_constant<int, 0x4E>{}));        // lanes 2 3 0 1
    if (lanes > 4) v = larger(v, dpp(v, std::integral_constant<int, 0x141>{}));       // mirrored in 8
    if (lanes > 8) v = larger(v, dpp(v, std::integral_constant<int, 0x140>{}));       // mirrored in 16
    if (lanes > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = larger((unsigned)r[0], (unsigned)r[1]);
    }
    return v;
}

// Eight numbers divided by 2^e as codes, rounded to nearest even.
template <typename T, typename T8>
__device__ static inline u32x2 encode8(const T8 &x, int e) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    typedef T T2 __attribute__((ext_vector_type(2)));
    const float by = __builtin_bit_cast(float, e < -126 ? 0x400000u : (unsigned)(e + 127) << 23);
    s16x2 lo = {0, 0}, hi = {0, 0};
    if constexpr (std::is_same<T, float>::value) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, x[0], x[1], by, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, x[2], x[3], by, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, x[4], x[5], by, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, x[6], x[7], by, true);
    } else if constexpr (std::is_same<T, f16>::value) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, T2{x[0], x[1]}, by, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, T2{x[2], x[3]}, by, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(hi, T2{x[4], x[5]}, by, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(hi, T2{x[6], x[7]}, by, true);
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, T2{x[0], x[1]}, by, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, T2{x[2], x[3]}, by, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, T2{x[4], x[5]}, by, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, T2{x[6], x[7]}, by, true);
    }
    return u32x2{__builtin_bit_cast(unsigned, lo), __builtin_bit_cast(unsigned, hi)};
}

// CT: element type of the pages, unsigned char for e4m3.
template <typename T, typename CT, bool WRITE>
__global__ __launch_bounds__(64 * kCacheWaves) void cache_kernel(const CacheKernel f) {
    constexpr bool CODES = std::is_same<CT, unsigned char>::value;
    const CacheArgs &a = f.a;
    const CacheView &c = a.cache;
    const int lane = threadIdx.x & 63, wave = blockIdx.x * kCacheWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = 2 * c.kv_heads, each = 64 >> f.lane_shift, total = a.tokens * rows;
    const int row0 = wave * f.passes * each, row1 = min(total, row0 + f.passes * each);
    if (row0 >= total) return;
    const int t0 = fast_div(row0, f.by_rows), n = (int)fast_div(row1 - 1, f.by_rows) - t0 + 1;   // the tokens of its rows, at most 64

    // Lane j: token t0 + j.  `place`: of its numbers in the pages, -1 if it has none, -2 for a row that belongs to no sequence.
    int64_t place = -2, place_exp = 0;
    {
        int s = t0 + lane, ahead = 1;    // rows from this one to the sequence's end
        bool some = lane < n;
        if (a.first) {
            const int s0 = last_not_above(a.sequences, t0, [&](int i) { return (int64_t)a.first[i]; });
            const int at = s0 + 1 + lane, next = at < a.sequences ? a.first[at] : INT32_MAX;   // where the 64 sequences behind s0 begin
            s = s0;
            for (int j = 1; j < n; ++j) {
                const int more = __popcll(__ballot(next <= t0 + j));
                const int of_j = more < 64 ? s0 + more : last_not_above(a.sequences, t0 + j, [&](int i) { return (int64_t)a.first[i]; });
                if (lane == j) s = of_j;
            }
            if (some) {
                ahead = a.first[s + 1] - (t0 + lane);
                some = ahead > 0 && t0 + lane >= a.first[s];
            }
        }
        if (some) {
            const int64_t t = (int64_t)a.lengths[s] - ahead;
            const int page = t < 0 || t > kCacheMostTokens ? -1 : page_of(c, a.table + s * a.table_stride, a.table_pages, (int)t);
            const int in_page = (int)t & ((1 << c.page_shift) - 1);
            place = page < 0 ? -1 : page * c.page_stride + in_page * c.token_stride;
            if (CODES) place_exp = page < 0 ? 0 : page * c.exp_page_stride + in_page * c.exp_token_stride;
        }
    }

    const int chunk = lane & (f.lanes - 1);
    const bool inside = chunk * 8 < c.head_dim;
    for (int row = row0 + (lane >> f.lane_shift); row - (lane >> f.lane_shift) < row1; row += kCacheBatch * each) {
        typedef T T8 __attribute__((ext_vector_type(8)));
        float v[kCacheBatch][8];
        T8 raw[kCacheBatch];
        T *x[kCacheBatch];
        CT *to[kCacheBatch];
        uint8_t *exponent[kCacheBatch];
        int64_t at[kCacheBatch];
        int e[kCacheBatch];
        auto of_lane = [&](int64_t value, int j) { return (int64_t)__shfl((int)(value >> 32), j) << 32 | (unsigned)__shfl((int)value, j); };
#pragma unroll
        for (int u = 0; u < kCacheBatch; ++u) {
            const int r = min(row + u * each, row1 - 1), token = fast_div(r, f.by_rows), of = r - token * rows;
            const bool value = of >= c.kv_heads;
            const int head = value ? of - c.kv_heads : of;
            at[u] = of_lane(place, token - t0);
            if (row + u * each >= row1) at[u] = -2;
            x[u] = static_cast<T *>(value ? a.v : a.k) + token * (value ? a.v_stride : a.k_stride) + head * (value ? a.v_head_stride : a.k_head_stride) + chunk * 8;
            to[u] = static_cast<CT *>(value ? c.v : c.k) + (at[u] < 0 ? 0 : at[u]) + head * c.head_stride + chunk * 8;
            if constexpr (CODES) exponent[u] = (value ? c.v_exp : c.k_exp) + of_lane(place_exp, token - t0) + head * c.exp_head_stride;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
            raw[u] = T8{};
            e[u] = 0;
            if (inside && at[u] >= 0) {
                if constexpr (WRITE && CODES) {
                    raw[u] = *reinterpret_cast<const T8 *>(x[u]);
                } else if constexpr (WRITE) {
                    load8(x[u], v[u]);
                } else if constexpr (CODES) {
                    const u32x2 codes = *reinterpret_cast<const u32x2 *>(to[u]);
                    const unsigned lo = codes[0], hi = codes[1];
                    e[u] = *exponent[u] - 127;
                    decode4(lo, v[u]);
                    decode4(hi, v[u] + 4);
                } else {
                    load8(to[u], v[u]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kCacheBatch; ++u) {
            if constexpr (!WRITE) {
                if constexpr (CODES) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[u][i] = ldexpf(v[u][i], e[u]);
                }
                if (inside && at[u] >= -1) store8(x[u], v[u]);
            } else if constexpr (CODES) {
                unsigned largest = largest_of(raw[u]);
                if (__builtin_expect(__any(largest >= 0x7f800000u), 0)) {   // what is no number has no part in it, and becomes a NaN
                    largest = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float one = (float)raw[u][i];
                        const unsigned bits = __builtin_bit_cast(unsigned, one) & 0x7fffffffu;
                        if (bits >= 0x7f800000u) raw[u][i] = (T)NAN;
                        else largest = largest > bits ? largest : bits;
                    }
                }
                const int power = exponent_for(of_row(largest, f.lanes));
                const u32x2 codes = encode8<T>(raw[u], power);
                if (inside && at[u] >= 0) __builtin_nontemporal_store(codes, reinterpret_cast<u32x2 *>(to[u]));
                if (chunk == 0 && at[u] >= 0) *exponent[u] = (uint8_t)(power + 127);
            } else {
                if (inside && at[u] >= 0) store8(to[u], v[u]);
            }
        }
    }
}

// The kernel's arguments, and its workgroups.
static CacheKernel cache_form(const CacheArgs &a, int64_t *workgroups) {
    CacheKernel f{a, make_fast_div((uint32_t)(2 * a.cache.kv_heads)), 2, 1, 1};
    while (f.lanes * 8 < a.cache.head_dim) {
        f.lanes *= 2;
        ++f.lane_shift;
    }
    // A batch, or fewer where that leaves a CU less than eight waves; at most 62 tokens.  Longer runs leave the waves that are at work at the same time further apart in memory: 34 k tokens
    // of 8 heads of 128 fp16 read from e4m3 38.5 us out of the last level's cache, and 46 for 36 where heads are two of 64.
    const int64_t each = 64 / f.lanes, rows = (int64_t)a.tokens * 2 * a.cache.kv_heads, all = (rows + each - 1) / each;
    f.passes = (int)std::max<int64_t>(1, std::min({all / 2048, (int64_t)kCacheBatch, 62 * 2 * a.cache.kv_heads / each}));
    const int64_t waves = (all + f.passes - 1) / f.passes;
    *workgroups = (waves + kCacheWaves - 1) / kCacheWaves;
    return f;
}

bool cache_fits(const CacheArgs &a) {
    int64_t workgroups;
    cache_form(a, &workgroups);
    return (int64_t)a.tokens * 2 * a.cache.kv_heads <= kCacheMostRows && workgroups * 64 * kCacheWaves <= kMostThreads;
}

template <typename T, bool WRITE>
static hipError_t launch_cache_as(const CacheArgs &a, hipStream_t s) {
    int64_t workgroups;
    const CacheKernel f = cache_form(a, &workgroups);
    const dim3 grid((unsigned)workgroups);
    if (a.cache.dtype == DT_E4M3) cache_kernel<T, unsigned char, WRITE><<<grid, 64 * kCacheWaves, 0, s>>>(f);
    else if (a.cache.dtype == DT_F16) cache_kernel<T, f16, WRITE><<<grid, 64 * kCacheWaves, 0, s>>>(f);
    else cache_kernel<T, bf16, WRITE><<<grid, 64 * kCacheWaves, 0, s>>>(f);
    return hipGetLastError();
}

template <bool WRITE>
static hipError_t launch_cache(const CacheArgs &a, hipStream_t s) {
    if (a.tokens < 1 || a.sequences < 1 || a.cache.head_dim % 16 != 0 || a.cache.head_dim > kAttendMostDim || !cache_fits(a)) return hipErrorInvalidValue;
    if (a.dtype == DT_F32) return launch_cache_as<float, WRITE>(a, s);
    return a.dtype == DT_F16 ? launch_cache_as<f16, WRITE>(a, s) : launch_cache_as<bf16, WRITE>(a, s);
}

hipError_t launch_cache_write(const CacheArgs &a, hipStream_t s) { return launch_cache<true>(a, s); }
hipError_t launch_cache_read(const CacheArgs &a, hipStream_t s) { return launch_cache<false>(a, s); }

}  // namespace cw
