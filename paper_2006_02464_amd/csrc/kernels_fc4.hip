// Fully connected layer over 4-bit weights: the choice of a form, rows of a few inputs, and LOAD's packing (fc4_body.h has the kernels).
#include "fc4_body.h"

namespace cw {

extern template hipError_t launch_fc4_x<X_F16>(const Fc4Args &, const Fc4Plan &, hipStream_t);
extern template hipError_t launch_fc4_x<X_BF16>(const Fc4Args &, const Fc4Plan &, hipStream_t);
extern template hipError_t launch_fc4_x<X_F32>(const Fc4Args &, const Fc4Plan &, hipStream_t);
extern template hipError_t launch_fc4_x<X_PLAIN>(const Fc4Args &, const Fc4Plan &, hipStream_t);

// Rows of fewer bytes than a load: one wave a weight row, eight rows of x.
constexpr int kShortRows = 8;
__global__ __launch_bounds__(256) void fc4_short_kernel(const Fc4Args a) {
    const int lane = threadIdx.x & 63, n = blockIdx.x * 4 + (threadIdx.x >> 6), m0 = blockIdx.y * kShortRows;
    if (n >= a.cout) return;
    auto element = [](const void *p, int64_t i, DType t) { return t == DT_F32 ? static_cast<const float *>(p)[i] : t == DT_F16 ? (float)static_cast<const f16 *>(p)[i] : (float)static_cast<const bf16 *>(p)[i]; };
    float w = 0.f;
    if (lane < a.cin) {   // one group
        const int b = a.q[n * a.q_stride + (lane >> 1)], z = a.zeros ? a.zeros[n * a.zero_stride] & 15 : 8;
        w = (float)((lane & 1 ? b >> 4 : b & 15) - z);
    }
    const float scale = element(a.scales, n * a.scale_stride, a.scale_dtype), bias = a.bias ? a.bias[n] : 0.f;
    for (int m = m0; m < m0 + kShortRows && m < a.rows; ++m) {
        float v = lane < a.cin ? element(a.x, m * a.x_stride + lane, a.x_dtype) * w : 0.f;
#pragma unroll
        for (int off = kShortIn / 2; off; off >>= 1) v += __shfl_xor(v, off, 64);
        if (lane == 0) fc4_store(a.y, m * a.y_stride + n, a.y_dtype, fmaf(v, scale, bias));
    }
}

static hipError_t launch_short(const Fc4Args &a, hipStream_t s) {
    for (int m = 0; m < a.rows; m += 65535 * kShortRows) {
        Fc4Args b = a;
        b.rows = a.rows - m < 65535 * kShortRows ? a.rows - m : 65535 * kShortRows;
        b.x = static_cast<const char *>(a.x) + m * a.x_stride * (a.x_dtype == DT_F32 ? 4 : 2);
        b.y = static_cast<char *>(a.y) + m * a.y_stride * (a.y_dtype == DT_F32 ? 4 : 2);
        fc4_short_kernel<<<dim3((a.cout + 3) / 4, (b.rows + kShortRows - 1) / kShortRows), 256, 0, s>>>(b);
    }
    return hipGetLastError();
}

// Measured in graphs of calls over several sets of weights, us a call (K = 4096, fp16, groups of 128, unless said otherwise):
//   up to 16 rows  x in LDS once a workgroup, which walks tiles of 16 weight rows; pairs of tiles where there are more than two for each CU
//                  (1 x 8192 bf16 to 32001: 31.0 in pairs, 32.3-37.7 one by one), but one by one up to that (4 x 4096 to 16384: 10.3 and 11.0)
//   more of x than LDS holds, or more rows: x in blocks.  64 or 128 weight rows a workgroup share a block of x, 16 make more workgroups:
//                  16 rows to 16384 11.5 us with 64, 19.6 with 16; 32 rows to 16384 16.6 and 16.9 (32), to 4096 14.5 and 10.0;
//                  64 rows to 16384 (groups of 64, zero points) 21-24 us with 64, 38 with 128; 512 rows to 4096 42.9 and 29.
//   32 or 64 rows  128 rows to 1000: 10.6 us with 32 rows and 16 weight rows a workgroup, 15.6 with 64 and 32.
Fc4Plan fc4_plan(const Fc4Args &a) {
    const bool two = a.x_dtype == DT_F32;
    auto wgs = [&](int rows, int cols) { return (int64_t)((a.rows + rows - 1) / rows) * ((a.cout + cols - 1) / cols); };
    if (a.cin < kShortIn) return {Fc4Plan::SHORT, kShortRows, 4, 256, 0};
    constexpr int enough = 200;   // workgroups that keep 256 CUs busy
    if (a.rows <= 16) {
        const int64_t blocks = (a.cin + kBlock - 1) / kBlock, fixed = (two ? 2 : 1) * a.rows * blocks * kBlock * 2 + 16 * 1024 + blocks * 64, scales = ((int64_t)fc4_groups(a) * 5 + 4) * 16;
        if (wgs(16, 16) > 1024 && fixed + 2 * scales <= few_lds(two, wgs(16, 32))) return {Fc4Plan::FEW_PAIRS, 16, 32, 512, 1024};
        if (fixed + scales <= few_lds(two, wgs(16, 16))) return {Fc4Plan::FEW, 16, 16, 512, 512};
        if (wgs(16, 64) >= enough) return {Fc4Plan::MANY1_64, 16, 64, 1024, 0};
        return {Fc4Plan::MANY1_16, 16, 16, 512, 0};
    }
    if (a.rows > 32) {
        if (wgs(64, 128) >= enough) return {Fc4Plan::MANY4_128, 64, 128, 512, 0};
        if (wgs(64, 64) >= enough) return {Fc4Plan::MANY4_64, 64, 64, two ? 512 : 1024, 0};
    }
    if (wgs(32, 64) >= enough) return {Fc4Plan::MANY2_64, 32, 64, two ? 512 : 1024, 0};
    return {Fc4Plan::MANY2_16, 32, 16, two ? 256 : 512, 0};
}

void fc4_grid(const Fc4Args &a, dim3 *grid, int *block) {
    const Fc4Plan p = fc4_plan(a);
    *grid = dim3((a.cout + p.cols - 1) / p.cols, (a.rows + p.rows - 1) / p.rows);
    if (p.most > 0 && (int)grid->x > p.most) {   // fewer workgroups walk all tiles, an even share of them each
        const unsigned own = (grid->x + p.most - 1) / p.most;
        grid->x = (grid->x + own - 1) / own;
    }
    *block = p.threads;
}

hipError_t launch_fc4(const Fc4Args &a, hipStream_t s) {
    if (a.rows < 1 || a.rows > kFc4MostRows || a.cin < 1 || a.cin > kFc4MostIn || a.cout < 1 || a.cout > kFc4MostOut || a.group < 32 || a.group % 32 != 0) return hipErrorInvalidValue;
    const Fc4Plan p = fc4_plan(a);
    if (p.form == Fc4Plan::SHORT) return launch_short(a, s);
    if (a.x_dtype == DT_BF16 && a.y_dtype != DT_F32 && p.form != Fc4Plan::FEW && p.form != Fc4Plan::FEW_PAIRS) return launch_fc4_x<X_PLAIN>(a, p, s);
    return a.x_dtype == DT_F16 ? launch_fc4_x<X_F16>(a, p, s) : a.x_dtype == DT_BF16 ? launch_fc4_x<X_BF16>(a, p, s) : launch_fc4_x<X_F32>(a, p, s);
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
