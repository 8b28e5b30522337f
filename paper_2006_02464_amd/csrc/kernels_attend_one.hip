// Attention of one new token over a paged cache (cw_attend_one has the definition).
#include <cmath>

#include "attend_common.h"

namespace cw {

// The simplest form: a wave for each query head, four numbers of the head a lane, one token at a time with the running maximum and sum of its softmax.
template <typename T, typename CT>
__global__ __launch_bounds__(64) void attend_one_kernel(const AttendOneArgs a) {
    constexpr bool CODES = std::is_same<CT, unsigned char>::value;
    const CacheView &c = a.cache;
    const int lane = threadIdx.x, s = blockIdx.x / a.heads, h = blockIdx.x - s * a.heads, kvh = h / (a.heads / c.kv_heads);
    const bool inside = lane * 4 < c.head_dim;
    const T *q = static_cast<const T *>(a.q) + s * a.q_stride + h * a.q_head_stride + lane * 4;
    float qv[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    if (inside)
        for (int i = 0; i < 4; ++i) qv[i] = (float)q[i];
    const int len = a.lengths[s], from = a.window > 0 && len > a.window ? len - a.window : 0;
    for (int t = from; t < len; ++t) {
        const int page = page_of(c, a.table + s * a.table_stride, a.table_pages, t);
        if (t >> c.page_shift >= a.table_pages) break;
        if (page < 0) continue;
        const int in = t & ((1 << c.page_shift) - 1);
        const int64_t at = page * c.page_stride + kvh * c.head_stride + in * c.token_stride + lane * 4;
        float kv[4] = {0.f, 0.f, 0.f, 0.f}, vv[4] = {0.f, 0.f, 0.f, 0.f};
        if (inside) {
            if constexpr (CODES) {
                const int64_t e = page * c.exp_page_stride + kvh * c.exp_head_stride + in * c.exp_token_stride;
                decode4(*reinterpret_cast<const unsigned *>(static_cast<const unsigned char *>(c.k) + at), kv);
                decode4(*reinterpret_cast<const unsigned *>(static_cast<const unsigned char *>(c.v) + at), vv);
                for (int i = 0; i < 4; ++i) {
                    kv[i] = ldexpf(kv[i], c.k_exp[e] - 127);
                    vv[i] = ldexpf(vv[i], c.v_exp[e] - 127);
                }
            } else {
                for (int i = 0; i < 4; ++i) {
                    kv[i] = (float)static_cast<const CT *>(c.k)[at + i];
                    vv[i] = (float)static_cast<const CT *>(c.v)[at + i];
                }
            }
        }
        float x = 0.f;
        for (int i = 0; i < 4; ++i) x = fmaf(qv[i], kv[i], x);
        for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
        x *= a.scale;
        const float top = x > m || x != x ? x : m, ref = top == -INFINITY ? 0.f : top, f = expf(m - ref), p = expf(x - ref);
        m = top;
        l = l * f + p;
        for (int i = 0; i < 4; ++i) o[i] = o[i] * f + p * vv[i];
    }
    const float by = l == 0.f ? 0.f : 1.f / l;
    T *y = static_cast<T *>(a.y) + s * a.y_stride + h * a.y_head_stride + lane * 4;
    if (inside)
        for (int i = 0; i < 4; ++i) y[i] = (T)(l == 0.f ? 0.f : o[i] * by);
    if (a.lse && lane == 0) a.lse[(int64_t)s * a.heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

size_t attend_one_workspace_bytes() { return (size_t)32 << 20; }

hipError_t launch_attend_one(const AttendOneArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)a.sequences * a.heads);
    const bool half = a.dtype == DT_F16;
    if (a.cache.dtype == DT_E4M3) {
        if (half) attend_one_kernel<f16, unsigned char><<<grid, 64, 0, s>>>(a);
        else attend_one_kernel<bf16, unsigned char><<<grid, 64, 0, s>>>(a);
    } else if (half) attend_one_kernel<f16, f16><<<grid, 64, 0, s>>>(a);
    else attend_one_kernel<bf16, bf16><<<grid, 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cw
