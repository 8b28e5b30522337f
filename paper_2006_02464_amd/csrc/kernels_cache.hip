// Tokens' keys and values to the pages of a cache and back (cw_cache_write and cw_cache_read have the definitions).
#include <cmath>

#include "attend_common.h"

namespace cw {

// Nothing but moving bytes.  A wave takes a token: its sequence by a search of `first`, its page, then 8 numbers a lane; the lanes of a head are a power of two, next to
// each other, so that its largest magnitude is a few exchanges away.
constexpr int kCacheWaves = 4;

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
    *reinterpret_cast<T8 *>(to) = v;
}

// The least e from -127 on with largest <= 448 * 2^e, for a finite largest; 448 = 1.75 * 2^8.
__device__ static inline int exponent_for(float largest) {
    const unsigned bits = __builtin_bit_cast(unsigned, largest);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return e < -127 ? -127 : e;
}

// CT: element type of the pages, unsigned char for e4m3.
template <typename T, typename CT, bool WRITE>
__global__ __launch_bounds__(64 * kCacheWaves) void cache_kernel(const CacheArgs a, int lanes) {
    constexpr bool CODES = std::is_same<CT, unsigned char>::value;
    const int lane = threadIdx.x & 63, token = blockIdx.x * kCacheWaves + (threadIdx.x >> 6);
    if (token >= a.tokens) return;
    const CacheView &c = a.cache;
    int s = token, ahead = 1;    // rows from this one to the sequence's end
    if (a.first) {
        if (token < a.first[0] || token >= a.first[a.sequences]) return;
        s = last_not_above(a.sequences, token, [&](int i) { return (int64_t)a.first[i]; });
        ahead = a.first[s + 1] - token;
        if (ahead < 1) return;
    }
    const int64_t t64 = (int64_t)a.lengths[s] - ahead;
    const int t = t64 < 0 || t64 > INT32_MAX ? -1 : (int)t64;
    const int page = page_of(c, a.table + s * a.table_stride, a.table_pages, t);
    if (WRITE && page < 0) return;
    const int in_page = t & ((1 << c.page_shift) - 1);
    const int chunk = lane & (lanes - 1), first_row = lane / lanes, rows = 2 * c.kv_heads, step = 64 / lanes;
    const bool inside = chunk * 8 < c.head_dim;
    for (int row = first_row; row < rows; row += step) {
        const bool value = row >= c.kv_heads;
        const int head = value ? row - c.kv_heads : row;
        T *x = static_cast<T *>(value ? a.v : a.k) + token * (value ? a.v_stride : a.k_stride) + head * (value ? a.v_head_stride : a.k_head_stride) + chunk * 8;
        CT *at = static_cast<CT *>(value ? c.v : c.k) + page * c.page_stride + head * c.head_stride + in_page * c.token_stride + chunk * 8;
        uint8_t *exponent = CODES ? (value ? c.v_exp : c.k_exp) + page * c.exp_page_stride + head * c.exp_head_stride + in_page * c.exp_token_stride : nullptr;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if constexpr (WRITE) {
            if (inside) load8(x, v);
            if constexpr (CODES) {
                float largest = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float m = fabsf(v[i]);
                    if (!(m < INFINITY)) v[i] = NAN;
                    largest = fmaxf(largest, m < INFINITY ? m : 0.f);
                }
                for (int o = 1; o < lanes; o *= 2) largest = fmaxf(largest, __shfl_xor(largest, o));
                const int e = exponent_for(largest);
                u32x2 codes = {0u, 0u};
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    int w = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(v[i], -e), ldexpf(v[i + 1], -e), 0, false);
                    codes[i / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(v[i + 2], -e), ldexpf(v[i + 3], -e), w, true);
                }
                if (inside) *reinterpret_cast<u32x2 *>(at) = codes;
                if (chunk == 0) *exponent = (uint8_t)(e + 127);
            } else {
                if (inside) store8(at, v);
            }
        } else if (inside) {
            if (page >= 0) {
                if constexpr (CODES) {
                    const u32x2 codes = *reinterpret_cast<const u32x2 *>(at);
                    const int e = *exponent - 127;
                    decode4(codes[0], v);
                    decode4(codes[1], v + 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = ldexpf(v[i], e);
                } else {
                    load8(at, v);
                }
            }
            store8(x, v);
        }
    }
}

template <typename T, bool WRITE>
static hipError_t launch_cache_as(const CacheArgs &a, hipStream_t s) {
    int lanes = 2;
    while (lanes * 8 < a.cache.head_dim) lanes *= 2;
    const dim3 grid((unsigned)((a.tokens + kCacheWaves - 1) / kCacheWaves));
    if (a.cache.dtype == DT_E4M3) cache_kernel<T, unsigned char, WRITE><<<grid, 64 * kCacheWaves, 0, s>>>(a, lanes);
    else if (a.cache.dtype == DT_F16) cache_kernel<T, f16, WRITE><<<grid, 64 * kCacheWaves, 0, s>>>(a, lanes);
    else cache_kernel<T, bf16, WRITE><<<grid, 64 * kCacheWaves, 0, s>>>(a, lanes);
    return hipGetLastError();
}

template <bool WRITE>
static hipError_t launch_cache(const CacheArgs &a, hipStream_t s) {
    if (a.tokens < 1 || a.sequences < 1 || a.cache.head_dim % 16 != 0 || a.cache.head_dim > kAttendMostDim) return hipErrorInvalidValue;
    if (a.dtype == DT_F32) return launch_cache_as<float, WRITE>(a, s);
    return a.dtype == DT_F16 ? launch_cache_as<f16, WRITE>(a, s) : launch_cache_as<bf16, WRITE>(a, s);
}

hipError_t launch_cache_write(const CacheArgs &a, hipStream_t s) { return launch_cache<true>(a, s); }
hipError_t launch_cache_read(const CacheArgs &a, hipStream_t s) { return launch_cache<false>(a, s); }

}  // namespace cw
