// The answer of a row of logits: log probability and rank of a given class, entropy, the likeliest classes (cw_answer has the definitions).
#include <cmath>

#include "common.h"

namespace cw {

__device__ static inline float logit(const AnswerArgs &a, int64_t i) {
    return a.dtype == DT_F32 ? static_cast<const float *>(a.x)[i] : a.dtype == DT_F16 ? (float)static_cast<const f16 *>(a.x)[i] : (float)static_cast<const bf16 *>(a.x)[i];
}

// The larger logit, and of equal ones the lower index, comes first.
__device__ static inline bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

// One workgroup a row, a pass for each question.
__global__ __launch_bounds__(256) void answer_kernel(const AnswerArgs a) {
    __shared__ float fs[256];
    __shared__ int is[256];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x, base = row * a.stride;
    float m = -INFINITY;
    int bad = 0;
    for (int i = t; i < a.classes; i += 256) {
        const float x = logit(a, base + i);
        bad |= !(x < INFINITY);
        m = fmaxf(m, x);
    }
    auto sum = [&](float v) {
        __syncthreads();
        fs[t] = v;
        __syncthreads();
        for (int n = 128; n; n >>= 1) {
            if (t < n) fs[t] += fs[t + n];
            __syncthreads();
        }
        return fs[0];
    };
    fs[t] = m; is[t] = bad;
    __syncthreads();
    for (int n = 128; n; n >>= 1) {
        if (t < n) { fs[t] = fmaxf(fs[t], fs[t + n]); is[t] |= is[t + n]; }
        __syncthreads();
    }
    m = fs[0]; bad = is[0];
    const int g = a.given ? a.given[row] : -1;
    const bool inside = g >= 0 && g < a.classes;
    const float xg = inside ? logit(a, base + g) : 0.f;
    float S = 0.f, T = 0.f, R = 0.f;
    for (int i = t; i < a.classes; i += 256) {
        const float x = logit(a, base + i);
        if (x > -INFINITY) {
            const float d = (x - m) * a.scale, e = expf(d);
            S += e;
            if (e > 0.f) T += e * d;
        }
        R += before(x, i, xg, g);   // exact: at most 2^24
    }
    S = sum(S); T = sum(T); R = sum(R);
    const bool empty = m == -INFINITY;
    const float ls = logf(S);
    if (t == 0) {
        float lp = bad ? NAN : !inside ? NAN : empty ? -INFINITY : (xg - m) * a.scale - ls;
        if (g < 0) lp = 0.f;
        if (a.logp) a.logp[row] = lp;
        if (a.rank) a.rank[row] = bad || !inside ? -1 : (int)R;
        if (a.entropy) a.entropy[row] = bad ? NAN : empty ? 0.f : ls - T / S;
    }
    float lx = INFINITY;
    int li = -1;
    for (int k = 0; k < a.top; ++k) {   // the first class behind the last one
        float bx = -INFINITY;
        int bi = 0x7fffffff;
        for (int i = t; i < a.classes; i += 256) {
            const float x = logit(a, base + i);
            if (before(lx, li, x, i) && before(x, i, bx, bi)) { bx = x; bi = i; }
        }
        __syncthreads();
        fs[t] = bx; is[t] = bi;
        __syncthreads();
        for (int n = 128; n; n >>= 1) {
            if (t < n && before(fs[t + n], is[t + n], fs[t], is[t])) { fs[t] = fs[t + n]; is[t] = is[t + n]; }
            __syncthreads();
        }
        lx = fs[0]; li = is[0];
        if (t == 0) {
            const bool none = bad || !(lx > -INFINITY);
            a.top_id[row * a.top + k] = none ? -1 : li;
            a.top_logp[row * a.top + k] = bad ? NAN : none ? -INFINITY : (lx - m) * a.scale - ls;
        }
    }
}

size_t answer_workspace_bytes() { return 1024; }

hipError_t launch_answer(const AnswerArgs &a, hipStream_t s) {
    if (a.rows < 1 || a.classes < 1 || a.classes > kAnswerMostClasses || a.top < 0 || a.top > kAnswerMostTop || (a.top > 0 && (!a.top_id || !a.top_logp))) return hipErrorInvalidValue;
    answer_kernel<<<dim3(a.rows), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cw
