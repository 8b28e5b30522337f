// Fully connected layer over 4-bit weights with group scales:
//   y[m][n] = bias[n] + sum_k x[m][k] * (q[n][k] - z[n][k / group]) * s[n][k / group]
#include "common.h"

namespace cw {

__device__ static inline float element(const void *p, int64_t i, DType t) {
    return t == DT_F32 ? static_cast<const float *>(p)[i] : t == DT_F16 ? (float)static_cast<const f16 *>(p)[i] : (float)static_cast<const bf16 *>(p)[i];
}
__device__ static inline void store(void *p, int64_t i, DType t, float v) {
    if (t == DT_F32) static_cast<float *>(p)[i] = v;
    else if (t == DT_F16) static_cast<f16 *>(p)[i] = (f16)v;
    else static_cast<bf16 *>(p)[i] = (bf16)v;
}

constexpr int kRows = 8;   // a workgroup of four waves: one weight row a wave, kRows rows of x

__global__ __launch_bounds__(256) void fc4_kernel(const Fc4Args a) {
    const int lane = threadIdx.x & 63, n = blockIdx.x * 4 + (threadIdx.x >> 6), m0 = blockIdx.y * kRows;
    if (n >= a.cout) return;
    const uint8_t *q = a.q + n * a.q_stride;
    float acc[kRows] = {};
    for (int k = lane; k < a.cin; k += 64) {
        const int j = k / a.group, b = q[k >> 1];
        const int v = ((k & 1) ? b >> 4 : b & 15) - (a.zeros ? a.zeros[n * a.zero_stride + j] & 15 : 8);
        const float w = (float)v * element(a.scales, n * a.scale_stride + j, a.scale_dtype);
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (m0 + i < a.rows) acc[i] += element(a.x, (m0 + i) * a.x_stride + k, a.x_dtype) * w;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
#pragma unroll
        for (int off = 32; off; off >>= 1) acc[i] += __shfl_xor(acc[i], off, 64);
        if (lane == 0 && m0 + i < a.rows) store(a.y, (m0 + i) * a.y_stride + n, a.y_dtype, acc[i] + (a.bias ? a.bias[n] : 0.f));
    }
}

void fc4_grid(const Fc4Args &a, dim3 *grid, int *block) {
    *grid = dim3((a.cout + 3) / 4, (a.rows + kRows - 1) / kRows);
    *block = 256;
}

hipError_t launch_fc4(const Fc4Args &a, hipStream_t s) {
    if (a.rows < 1 || a.rows > kFc4MostRows || a.cin < 1 || a.cout < 1 || a.group < 32) return hipErrorInvalidValue;
    for (int m = 0; m < a.rows; m += 65535 * kRows) {   // rows beyond the grid's y
        Fc4Args b = a;
        b.rows = a.rows - m < 65535 * kRows ? a.rows - m : 65535 * kRows;
        b.x = static_cast<const char *>(a.x) + m * a.x_stride * (a.x_dtype == DT_F32 ? 4 : 2);
        b.y = static_cast<char *>(a.y) + m * a.y_stride * (a.y_dtype == DT_F32 ? 4 : 2);
        dim3 grid;
        int block;
        fc4_grid(b, &grid, &block);
        fc4_kernel<<<grid, block, 0, s>>>(b);
    }
    return hipGetLastError();
}

// LOAD: the canonical parts, each a multiple of 2 bytes from an even address on, to the aligned places of fc4_layout, and the bias.  Bound: HBM.
__global__ __launch_bounds__(256) void pack_fc4_kernel(const uint16_t *src, char *dst, const float *bias_src, float *bias_dst, Fc4Layout l, int32_t cout) {
    const size_t q = ((size_t)cout * l.q_row + 1) / 2, s = (size_t)cout * l.groups;
    const size_t step = (size_t)gridDim.x * 256, first = (size_t)blockIdx.x * 256 + threadIdx.x;
    for (size_t i = first; i < q; i += step) reinterpret_cast<uint16_t *>(dst)[i] = src[i];
    for (size_t i = first; i < s; i += step) reinterpret_cast<uint16_t *>(dst + l.scales)[i] = src[q + i];
    const uint8_t *zeros = reinterpret_cast<const uint8_t *>(src + q + s);
    for (size_t i = first; i < s; i += step) reinterpret_cast<uint8_t *>(dst + l.zeros)[i] = zeros[i];
    for (size_t i = first; i < (size_t)cout; i += step) bias_dst[i] = bias_src[i];
}

hipError_t launch_pack_fc4(const char *src, char *dst, const float *bias_src, float *bias_dst, int32_t cin, int32_t cout, int32_t group, hipStream_t s) {
    if (!src || !dst || !bias_src || !bias_dst || reinterpret_cast<uintptr_t>(src) % 2 != 0 || reinterpret_cast<uintptr_t>(dst) % 256 != 0) return hipErrorInvalidValue;
    const Fc4Layout l = fc4_layout(cin, cout, group);
    const size_t wgs = ((size_t)cout * l.q_row / 2 + 255) / 256;
    pack_fc4_kernel<<<dim3((unsigned)(wgs < 1 ? 1 : wgs < kLoadGridCap ? wgs : kLoadGridCap)), 256, 0, s>>>(
        reinterpret_cast<const uint16_t *>(src), dst, bias_src, bias_dst, l, cout);
    return hipGetLastError();
}

}  // namespace cw
