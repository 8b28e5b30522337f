// Attention of packed prompts (cw_attend has the definition).
#include <cmath>

#include "attend_common.h"

namespace cw {

// The simplest form: a wave for each query and head, four numbers of the head a lane, one key at a time with the running maximum and sum of its softmax.
template <typename T>
__global__ __launch_bounds__(64) void attend_kernel(const AttendArgs a) {
    const int lane = threadIdx.x, row = blockIdx.x, h = blockIdx.y, kvh = h / (a.heads / a.kv_heads);
    if (row < a.first[0] || row >= a.first[a.sequences]) return;
    const int sq = last_not_above(a.sequences, row, [&](int i) { return (int64_t)a.first[i]; });
    const int ahead = a.first[sq + 1] - row;     // queries from this one to the end
    if (ahead < 1) return;
    const int k0 = a.first_k[sq] < 0 ? 0 : a.first_k[sq], k1 = a.first_k[sq + 1] > a.keys ? a.keys : a.first_k[sq + 1];
    const int last = a.causal ? k1 - ahead : k1 - 1;
    const int from = a.window > 0 && last + 1 - a.window > k0 ? last + 1 - a.window : k0;
    const bool inside = lane * 4 < a.head_dim;
    float qv[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    const T *q = static_cast<const T *>(a.q) + row * a.q_stride + h * a.q_head_stride + lane * 4;
    if (inside)
        for (int i = 0; i < 4; ++i) qv[i] = (float)q[i];
    for (int t = from; t <= last; ++t) {
        const T *k = static_cast<const T *>(a.k) + t * a.k_stride + kvh * a.k_head_stride + lane * 4;
        const T *v = static_cast<const T *>(a.v) + t * a.v_stride + kvh * a.v_head_stride + lane * 4;
        float x = 0.f, vv[4] = {0.f, 0.f, 0.f, 0.f};
        if (inside)
            for (int i = 0; i < 4; ++i) {
                x = fmaf(qv[i], (float)k[i], x);
                vv[i] = (float)v[i];
            }
        for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
        x *= a.scale;
        const float top = x > m || x != x ? x : m, ref = top == -INFINITY ? 0.f : top, f = expf(m - ref), p = expf(x - ref);
        m = top;
        l = l * f + p;
        for (int i = 0; i < 4; ++i) o[i] = o[i] * f + p * vv[i];
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride + h * a.y_head_stride + lane * 4;
    if (inside)
        for (int i = 0; i < 4; ++i) y[i] = (T)(l == 0.f ? 0.f : o[i] / l);
    if (a.lse && lane == 0) a.lse[(int64_t)row * a.heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

hipError_t launch_attend(const AttendArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)a.tokens, (unsigned)a.heads);
    if (a.dtype == DT_F16) attend_kernel<f16><<<grid, 64, 0, s>>>(a);
    else attend_kernel<bf16><<<grid, 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cw
