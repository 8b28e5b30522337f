// Fully connected layer over 4-bit weights with group scales:
//   y[m][n] = bias[n] + sum_k x[m][k] * (q[n][k] - z[n][k / group]) * s[n][k / group]
#include "conv_common.h"

namespace cw {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));     // a 16-byte load from any address (global memory takes them)

constexpr int kBlock = 128;   // inputs that a wave takes at a time: 16 bytes of weights a lane, four lanes a row

// How x becomes fp16 operands: as it is; bf16 and fp32 scaled by a power of two to each row's and block's largest value,
// fp32 in two parts.
enum XForm { X_F16, X_BF16, X_F32 };

struct Fc4Kernel {
    Fc4Args a;
    FastDiv group_div;   // of an input's number by `group`
    int32_t blocks;      // blocks of all waves along K in a phase
};

// A scale as it is stored, and its value: the load is waited for where the value is used.
__device__ static inline unsigned fc4_scale_bits(const char *p, int j, DType t) {
    return t == DT_F32 ? *reinterpret_cast<const unsigned *>(p + 4 * (int64_t)j) : *reinterpret_cast<const uint16_t *>(p + 2 * (int64_t)j);
}
__device__ static inline float fc4_scale(unsigned bits, DType t) {
    const float half = (float)__builtin_bit_cast(f16, (uint16_t)bits);
    return t == DT_F16 ? half : __builtin_bit_cast(float, bits << (t == DT_F32 ? 0 : 16));
}
__device__ static inline void fc4_store(void *p, int64_t i, DType t, float v) {
    if (t == DT_F32) static_cast<float *>(p)[i] = v;
    else if (t == DT_F16) static_cast<f16 *>(p)[i] = (f16)v;
    else static_cast<bf16 *>(p)[i] = (bf16)v;
}

// Sixteen bytes of a row of weights from byte `at` on, of which the row has `have` (the others: zeros).
__device__ static inline u32x4 fc4_weights(const uint8_t *row, int at, int have) {
    if (at + 16 <= have) return *reinterpret_cast<const u32x4_any *>(row + at);
    u32x4 v = {0, 0, 0, 0};
    for (int i = 0; i < 16 && at + i < have; ++i) v[i >> 2] |= (unsigned)row[at + i] << ((i & 3) * 8);
    return v;
}

// Eight activations from k on as fp16, in the order (0 4) (1 5) (2 6) (3 7) in which the weights' nibbles come out.
template <int X>
__device__ static inline void fc4_take_x(const void *row, int k, int cin, float (&v)[8]) {
    typedef typename std::conditional<X == X_F16, f16, typename std::conditional<X == X_BF16, bf16, float>::type>::type T;
    const T *p = static_cast<const T *>(row) + k;
    if (k + 8 <= cin) {
        u32x4 raw[sizeof(T) / 2];
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const u32x4_any *>(p)[i];
        const T *e = reinterpret_cast<const T *>(raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)e[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < cin ? (float)p[i] : 0.f;
    }
}

// MT, NT: tiles of 16 rows of x and of 16 weight rows that a wave multiplies; NW x KW: waves along the weight rows and along K;
// GM: matrix steps of 32 inputs between two scales; D: blocks whose weights are under way.
template <int X, int MT, int NT, int NW, int KW, int GM, int D, bool Z>
__global__ __launch_bounds__(64 * NW * KW) void fc4_kernel(const Fc4Kernel f) {
    constexpr int THREADS = 64 * NW * KW, PARTS = X == X_F32 ? 2 : 1;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Fc4Args &a = f.a;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), nw = wave % NW, kw = wave / NW;
    const int c = lane & 15, kq = lane >> 4;
    const int m0 = blockIdx.y * (16 * MT), rows = a.rows - m0 < 16 * MT ? a.rows - m0 : 16 * MT;
    const int n0 = (blockIdx.x * NW + nw) * (16 * NT);
    const int per_wave = f.blocks / KW, have = (a.cin + 1) >> 1;
    const int slices = f.blocks * (kBlock / 32), part_bytes = slices * rows * 64;
    float *xs = reinterpret_cast<float *>(lds + PARTS * part_bytes);   // [block][16 MT]: what x was divided by

    const uint8_t *q[NT], *zp[NT];
    const char *sp[NT];
    const int ssize = a.scale_dtype == DT_F32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int n = n0 + i * 16 + c < a.cout ? n0 + i * 16 + c : a.cout - 1;
        q[i] = a.q + n * a.q_stride;
        sp[i] = static_cast<const char *>(a.scales) + n * a.scale_stride * ssize;
        if (Z) zp[i] = a.zeros + n * a.zero_stride;
    }
    u32x4 w[D][NT];
    unsigned s[D][NT][4 / GM], z[D][NT][4 / GM];
    auto load = [&](int u, int block) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            if (block * kBlock >= a.cin) continue;
            if ((block + 1) * kBlock <= a.cin) w[u][i] = *reinterpret_cast<const u32x4_any *>(q[i] + block * 64 + kq * 16);
            else w[u][i] = fc4_weights(q[i], block * 64 + kq * 16, have);
#pragma unroll
            for (int g = 0; g < 4 / GM; ++g) {
                const int k = block * kBlock + g * GM * 32;
                const int j = (int)fast_div(k < a.cin ? k : a.cin - 1, f.group_div);
                s[u][i][g] = fc4_scale_bits(sp[i], j, a.scale_dtype);
                if (Z) z[u][i][g] = zp[i][j];
            }
        }
    };
    f32x4 total[MT][NT] = {};
    unsigned magic = 0x64006400u;
    asm("" : "+v"(magic));

    const int phases = (a.cin + f.blocks * kBlock - 1) / (f.blocks * kBlock);
    int first = kw * per_wave;   // this wave's first block of the phase
#pragma unroll
    for (int u = 0; u < D; ++u)
        if (u < per_wave) load(u, first + u);
    for (int phase = 0; phase < phases; ++phase, first += f.blocks) {
        // x of this phase: [part][slice of 32 inputs][row][32]
        if (phase > 0) __syncthreads();
        const int k0 = phase * f.blocks * kBlock;
        const int staged = (a.cin - k0 + kBlock - 1) / kBlock < f.blocks ? (a.cin - k0 + kBlock - 1) / kBlock : f.blocks;
        for (int item = t; item < rows * staged * 16; item += THREADS) {
            const int piece = item & 15, rb = item >> 4, row = rb % rows, block = rb / rows, kk = block * kBlock + piece * 8;
            const int es = X == X_F32 ? 4 : 2;
            float v[8];
            fc4_take_x<X>(static_cast<const char *>(a.x) + (m0 + row) * a.x_stride * es, k0 + kk, a.cin, v);
            if (X != X_F16) {
                float most = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));
#pragma unroll
                for (int off = 8; off; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, 16));
                int e = (int)(__builtin_bit_cast(unsigned, most) >> 23) - 127;
                e = e > 127 ? 127 : e < -113 ? -113 : e;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = ldexpf(v[i], 14 - e);
                if (piece == 0) xs[block * (16 * MT) + row] = ldexpf(1.f, e - 14);
            }
            f16x8 hi, lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = i < 4 ? 2 * i : 2 * (i - 4) + 1;
                hi[at] = (f16)v[i];
                if (X == X_F32) lo[at] = (f16)(__builtin_isinf(v[i]) ? 0.f : v[i] - (float)hi[at]);
            }
            const int to = ((kk >> 5) * rows + row) * 64 + (piece & 3) * 16;
            *reinterpret_cast<f16x8 *>(lds + to) = hi;
            if (X == X_F32) *reinterpret_cast<f16x8 *>(lds + part_bytes + to) = lo;
        }
        __syncthreads();
        int rowoff[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) rowoff[i] = (i * 16 + c < rows ? i * 16 + c : rows - 1) * 64 + kq * 16;
        for (int b = 0; b < per_wave; b += D) {
#pragma unroll
            for (int u = 0; u < D; ++u) {
                const int block = first + b + u;
                if (b + u < per_wave && block * kBlock < a.cin) {
                    const int slice = (kw * per_wave + b + u) * (kBlock / 32);
#pragma unroll
                    for (int i = 0; i < NT; ++i) {   // word j of lane group kq becomes word kq of lane group j: step j then has inputs 32 j + 8 kq + 0..7
                        u32x4 &v = w[u][i];
                        auto r = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
                        v[0] = r[0]; v[2] = r[1];
                        r = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
                        v[1] = r[0]; v[3] = r[1];
                        r = __builtin_amdgcn_permlane16_swap(v[0], v[1], false, false);
                        v[0] = r[0]; v[1] = r[1];
                        r = __builtin_amdgcn_permlane16_swap(v[2], v[3], false, false);
                        v[2] = r[0]; v[3] = r[1];
                    }
                    f32x4 block_total[MT][NT];
                    if (X != X_F16)
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int j = 0; j < NT; ++j) block_total[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                    f32x4 p[MT][NT];
#pragma unroll
                    for (int step = 0; step < 4; ++step) {
                        f16x8 x[PARTS][MT];
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
#pragma unroll
                            for (int i = 0; i < MT; ++i)
                                x[part][i] = *reinterpret_cast<const f16x8 *>(lds + part * part_bytes + (slice + step) * rows * 64 + rowoff[i]);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            // Nibbles as the low bits of fp16 numbers of exponent 10: 1024 + q and 1024 + 16 q, from which q - z follows exactly.
                            const float scale = fc4_scale(s[u][j][step / GM], a.scale_dtype);
                            const unsigned v = w[u][j][step], v8 = v >> 8;
                            unsigned zlo = 0xE408E408u, zhi = 0xD480D480u;   // -(1024 + 8), -(64 + 8)
                            if (Z) {
                                const unsigned zz = (z[u][j][step / GM] & 15) * 0x10001u;
                                zlo = 0xE400E400u | zz;
                                zhi = 0xD400D400u | (zz << 4);
                            }
                            const f16x2 sixteenth = {(f16)0.0625f, (f16)0.0625f};
                            const f16x2 clo = __builtin_bit_cast(f16x2, zlo), chi = __builtin_bit_cast(f16x2, zhi);
                            const f16x2 w0 = __builtin_bit_cast(f16x2, (v & 0x000F000Fu) | magic) + clo;
                            const f16x2 w1 = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00F000F0u) | magic), sixteenth, chi);
                            const f16x2 w2 = __builtin_bit_cast(f16x2, (v8 & 0x000F000Fu) | magic) + clo;
                            const f16x2 w3 = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v8 & 0x00F000F0u) | magic), sixteenth, chi);
                            const f16x8 ww = {w0[0], w0[1], w1[0], w1[1], w2[0], w2[1], w3[0], w3[1]};
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                                p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[0][i], ww, step % GM == 0 ? zero : p[i][j], 0, 0, 0);
                                if (X == X_F32) p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[PARTS - 1][i], ww, p[i][j], 0, 0, 0);
                                if (step % GM == GM - 1) {
                                    f32x4 &to = X == X_F16 ? total[i][j] : block_total[i][j];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) to[e] = fmaf(p[i][j][e], scale, to[e]);
                                }
                            }
                        }
                    }
                    if (X != X_F16)
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            const f32x4 back = *reinterpret_cast<const f32x4 *>(xs + (kw * per_wave + b + u) * (16 * MT) + i * 16 + kq * 4);
#pragma unroll
                            for (int j = 0; j < NT; ++j)
#pragma unroll
                                for (int e = 0; e < 4; ++e) total[i][j][e] = fmaf(block_total[i][j][e], back[e], total[i][j][e]);
                        }
                }
                // the next block of these registers
                const int next = b + u + D;
                if (next < per_wave) load(u, first + next);

            }
        }
        if (phase + 1 < phases)
#pragma unroll
            for (int u = 0; u < D; ++u)
                if (u < per_wave) load(u, first + f.blocks + u);
    }
    // The waves along K meet in LDS: [kw][nw][tile][4][64]
    __syncthreads();
    float *part = reinterpret_cast<float *>(lds);
    constexpr int TILES = MT * NT;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[(((wave * MT + i) * NT + j) * 4 + e) * 64 + lane] = total[i][j][e];
    __syncthreads();
    for (int o = t; o < NW * TILES * 256; o += THREADS) {   // o = ((nw, i, j), e, lane)
        const int l = o & 63, e = (o >> 6) & 3, tile = (o >> 8) % TILES, ow = (o >> 8) / TILES;
        const int m = (tile / NT) * 16 + (l >> 4) * 4 + e, n = (blockIdx.x * NW + ow) * (16 * NT) + (tile % NT) * 16 + (l & 15);
        if (m >= rows || n >= a.cout) continue;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < KW; ++k) v += part[k * (NW * TILES * 256) + o];
        fc4_store(a.y, (m0 + m) * a.y_stride + n, a.y_dtype, v + (a.bias ? a.bias[n] : 0.f));
    }
}

constexpr int kLdsBytes = 160 * 1024;

template <int X, int MT, int NT, int NW, int KW, int GM, bool Z>
static hipError_t launch_form(const Fc4Args &a, hipStream_t s) {
    constexpr int D = 4;
    Fc4Kernel f{a, make_fast_div((uint32_t)a.group), 0};
    const int blocks = (a.cin + kBlock - 1) / kBlock, rows = a.rows < 16 * MT ? a.rows : 16 * MT;
    const int per_block = rows * kBlock * 2 * (X == X_F32 ? 2 : 1) + 16 * MT * 4;   // bytes of LDS
    int per_wave = (blocks + KW - 1) / KW;
    const int budget = 64 * 1024;
    if (per_wave * KW * per_block > budget) {
        per_wave = budget / (KW * per_block);
        per_wave = per_wave < 1 ? 1 : per_wave;
    }
    f.blocks = per_wave * KW;
    int bytes = f.blocks * per_block;
    const int meet = NW * KW * MT * NT * 1024;
    bytes = bytes > meet ? bytes : meet;
    if (bytes > kLdsBytes) return hipErrorInvalidValue;
    auto kernel = fc4_kernel<X, MT, NT, NW, KW, GM, D, Z>;
    const int per_y = 16 * MT;
    for (int m = 0; m < a.rows; m += 65535 * per_y) {   // rows beyond the grid's y
        Fc4Kernel part = f;
        part.a.rows = a.rows - m < 65535 * per_y ? a.rows - m : 65535 * per_y;
        part.a.x = static_cast<const char *>(a.x) + m * a.x_stride * (a.x_dtype == DT_F32 ? 4 : 2);
        part.a.y = static_cast<char *>(a.y) + m * a.y_stride * (a.y_dtype == DT_F32 ? 4 : 2);
        kernel<<<dim3((a.cout + 16 * NT * NW - 1) / (16 * NT * NW), (part.a.rows + per_y - 1) / per_y), 64 * NW * KW, bytes, s>>>(part);
    }
    return hipGetLastError();
}

template <int X, int MT, int NT, int NW, int KW>
static hipError_t launch_groups(const Fc4Args &a, hipStream_t s) {
    if (a.group % 128 == 0) return a.zeros ? launch_form<X, MT, NT, NW, KW, 4, true>(a, s) : launch_form<X, MT, NT, NW, KW, 4, false>(a, s);
    if (a.group % 64 == 0) return a.zeros ? launch_form<X, MT, NT, NW, KW, 2, true>(a, s) : launch_form<X, MT, NT, NW, KW, 2, false>(a, s);
    return a.zeros ? launch_form<X, MT, NT, NW, KW, 1, true>(a, s) : launch_form<X, MT, NT, NW, KW, 1, false>(a, s);
}

template <int X>
static hipError_t launch_x(const Fc4Args &a, hipStream_t s) {
    if (a.rows <= 16) return launch_groups<X, 1, 1, 1, 8>(a, s);
    return launch_groups<X, 4, 2, 4, 2>(a, s);
}

void fc4_grid(const Fc4Args &a, dim3 *grid, int *block) {
    if (a.rows <= 16) *grid = dim3((a.cout + 15) / 16, 1);
    else *grid = dim3((a.cout + 127) / 128, (a.rows + 63) / 64);
    *block = 512;
}

hipError_t launch_fc4(const Fc4Args &a, hipStream_t s) {
    if (a.rows < 1 || a.rows > kFc4MostRows || a.cin < 1 || a.cin > kFc4MostIn || a.cout < 1 || a.cout > kFc4MostOut || a.group < 32 || a.group % 32 != 0) return hipErrorInvalidValue;
    return a.x_dtype == DT_F16 ? launch_x<X_F16>(a, s) : a.x_dtype == DT_BF16 ? launch_x<X_BF16>(a, s) : launch_x<X_F32>(a, s);
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
