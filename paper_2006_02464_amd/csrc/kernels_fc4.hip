// Fully connected layer over 4-bit weights: the choice of a form, rows of a few inputs, and LOAD's packing (fc4_body.h has the kernels).
#include "fc4_body.h"

namespace cw {

extern template hipError_t launch_fc4_x<X_F16>(const Fc4Args &, const Fc4Plan &, hipStream_t);
extern template hipError_t launch_fc4_x<X_BF16>(const Fc4Args &, const Fc4Plan &, hipStream_t);
extern template hipError_t launch_fc4_x<X_F32>(const Fc4Args &, const Fc4Plan &, hipStream_t);

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

// Up to 16 rows whose x LDS holds: one workgroup keeps it and walks tiles of 16 weight rows; pairs of tiles, twice the loads under way, where there are more
// than two for each of 512 workgroups and they are long (us one by one and in pairs, 1 x 8192 bf16 to 32001: 36.1 and 32.4, 2 x 4096 fp16 to 60000: 36.5
// and 33.3; but 6 x 1536 fp32 to 31051: 11.7 and 14.7, 8 x 2048 bf16 to 20000, groups of 32: 14.2 and 15.9).
// More: x in blocks, and tiles of 16 x 16 to 128 x 256.  A larger tile reads x and converts weights less often for each product, and fewer of them fill
// the 256 CUs, so the tile is the one with the least  rounds of 256 workgroups x (2 us + a time for each block of 128 inputs), which were measured in graphs
// of calls over several sets of weights (fp16, groups of 128; us, rates in TFLOP/s):
//   tile          16x16  16x32  16x64  32x32  32x64  64x64  64x128  64x256  128x256
//   16 x 4096 to 4096     7.1    7.7    9.9
//   16 x 4096 to 16384   18.7   11.8   10.8
//   32 x 4096 to 8192                         10.9   12.6
//   64 x 4096 to 4096                         10.3   12.5   17.4    23.0
//   64 x 4096 to 16384                        38     24     20.7
//   256 x 2048 to 1000                         7.4    8.3   11.1    14.1
//   512 x 4096 to 4096                                      35      25-29   41       64
//   1024 x 4096 to 4096                                             56.7    45.5     64.8
//   2048 x 8192 to 8192                                     475     366     317      265 (1036; a library's product of 16-bit weights 1226)
// fp32, in two parts, takes about twice the time for a block, and 128 rows' two parts do not fit in the registers; nor do 128 rows of bf16 beside their conversion.
struct Fc4Tile {
    Fc4Plan::Form form;
    int rows, cols, threads, threads_two;   // threads_two: of activations in two parts
    float block;                            // us
};
constexpr Fc4Tile kFc4Tiles[] = {{Fc4Plan::MANY1_16, 16, 16, 512, 512, 0.15f},    {Fc4Plan::MANY1_32, 16, 32, 512, 512, 0.2f},    {Fc4Plan::MANY1_64, 16, 64, 1024, 1024, 0.27f},
                                 {Fc4Plan::MANY2_32, 32, 32, 512, 512, 0.25f},    {Fc4Plan::MANY2_64, 32, 64, 512, 1024, 0.33f},  {Fc4Plan::MANY4_64, 64, 64, 512, 512, 0.56f},
                                 {Fc4Plan::MANY4_128, 64, 128, 1024, 1024, 0.78f}, {Fc4Plan::MANY4_256, 64, 256, 512, 512, 1.36f}, {Fc4Plan::MANY8_256, 128, 256, 512, 512, 2.05f}};

Fc4Plan fc4_plan(const Fc4Args &a) {
    const bool two = a.x_dtype == DT_F32;
    const int64_t blocks = (a.cin + kBlock - 1) / kBlock;
    auto wgs = [&](int rows, int cols) { return (int64_t)((a.rows + rows - 1) / rows) * ((a.cout + cols - 1) / cols); };
    if (a.cin < kShortIn) return {Fc4Plan::SHORT, kShortRows, 4, 256, 0};
    if (a.rows <= 16) {
        if (wgs(16, 16) > 1024 && blocks >= 32 && fc4_few(a, 2, 1024).wgs) return {Fc4Plan::FEW_PAIRS, 16, 32, 64 * kFewWaves, 1024};
        if (fc4_few(a, 1, 512).wgs) return {Fc4Plan::FEW, 16, 16, 64 * kFewWaves, 512};
    }
    const Fc4Tile *best = nullptr;
    float least = 0.f;
    for (const Fc4Tile &t : kFc4Tiles) {
        if (t.form == Fc4Plan::MANY8_256 && a.x_dtype != DT_F16) continue;
        const float time = (float)((wgs(t.rows, t.cols) + 255) / 256) * (2.f + (two ? 2 : 1) * t.block * blocks);
        if (!best || time < least) best = &t, least = time;
    }
    return {best->form, best->rows, best->cols, two ? best->threads_two : best->threads, 0};
}

void fc4_grid(const Fc4Args &a, dim3 *grid, int *block) {
    const Fc4Plan p = fc4_plan(a);
    *grid = dim3((a.cout + p.cols - 1) / p.cols, (a.rows + p.rows - 1) / p.rows);
    if (p.most > 0) grid->x = fc4_few(a, p.cols / 16, p.most).wgs;
    *block = p.threads;
}

hipError_t launch_fc4(const Fc4Args &a, hipStream_t s) {
    if (a.rows < 1 || a.rows > kFc4MostRows || a.cin < 1 || a.cin > kFc4MostIn || a.cout < 1 || a.cout > kFc4MostOut || a.group < 32 || a.group % 32 != 0) return hipErrorInvalidValue;
    const Fc4Plan p = fc4_plan(a);
    if (p.form == Fc4Plan::SHORT) return launch_short(a, s);
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
