// Fully connected layer over 4-bit weights with group scales:
//   y[m][n] = bias[n] + sum_k x[m][k] * (q[n][k] - z[n][k / group]) * s[n][k / group]
#pragma once
#include "conv_common.h"

namespace cw {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));     // a 16-byte load from any address (global memory takes them)

constexpr int kBlock = 128;   // inputs that a wave takes at a time: 16 bytes of weights a lane, four lanes a row

// How x becomes operands: fp16 as it is; bf16 and fp32 as fp16, scaled by a power of two to each row's and block's largest value, fp32 in two parts.
// Weights are q - z exactly, whatever the type: a sum of (16 + q) x less (16 + z) sum x, which bf16 numbers would need no conversion for (512 x 4096 to 4096:
// 33 us for 37; 2048 x 8192 to 8192: 300 for 394), rounds with 16 to 31 times every |x|, that of an input whose weights are zero among them.
enum XForm { X_F16, X_BF16, X_F32 };
constexpr int kShortIn = 32;   // rows of fewer inputs have fewer bytes than a load: a kernel of their own

struct Fc4Kernel {
    Fc4Args a;
    FastDiv group_div;   // of an input's number by `group`
    FastDiv lots_div;    // by a row's groups in sixteens
};

__device__ static inline void fc4_store(void *p, int64_t i, DType t, float v) {
    if (t == DT_F32) static_cast<float *>(p)[i] = v;
    else if (t == DT_F16) static_cast<f16 *>(p)[i] = (f16)v;
    else static_cast<bf16 *>(p)[i] = (bf16)v;
}

// v[0..N) as one number, shifted down by `bits` (a multiple of 8, less than 32 N; of 32 N and more: zero).
template <int N>
__device__ static inline void fc4_shift_down(u32x4 (&v)[N / 4], unsigned bits) {
    auto at = [&](int i) -> unsigned { return i < N ? v[i / 4][i % 4] : 0u; };
#pragma unroll
    for (int i = 0; i < N; ++i) v[i / 4][i % 4] = __builtin_amdgcn_alignbit(at(i + 1), at(i), bits & 31);
#pragma unroll
    for (int s = 1; s < N; s *= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i / 4][i % 4] = bits & (32 * s) ? at(i + s) : at(i);
    if (bits >= 32 * N)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i / 4][i % 4] = 0;
}

// What a lane reads of the weights: 32 nibbles a block of each of NT rows.  No load stands in a branch: the wait for earlier loads behind it would be for all
// of them.
template <int NT>
struct Fc4Weights {
    u32x4 w[NT];
    // The sixteen bytes of a lane, or where the row ends among them or before, its last sixteen (see shift).
    __device__ void load(const Fc4Kernel &f, const uint8_t *const (&q)[NT], int block, int kq) {
        const int at = block * (kBlock / 2) + kq * 16, last = ((f.a.cin + 1) >> 1) - 16, from = at < last ? at : last;
#pragma unroll
        for (int i = 0; i < NT; ++i) w[i] = *reinterpret_cast<const u32x4_any *>(q[i] + from);
    }
    // The last block, where it is not whole: bytes to their places (what then stands behind the row is multiplied by zeros).
    __device__ void shift(const Fc4Kernel &f, int block, int kq) {
        const int at = block * (kBlock / 2) + kq * 16, last = ((f.a.cin + 1) >> 1) - 16;
        const unsigned bits = at > last ? (unsigned)(at - last) * 8 : 0;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            u32x4 v[1] = {w[i]};
            fc4_shift_down<4>(v, bits);
            w[i] = v[0];
        }
    }
};
template <int NT>
__device__ static inline void fc4_rows(const uint8_t *(&q)[NT], const Fc4Args &a, int n0, int c) {   // rows behind the last: the last
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int n = n0 + i * 16 + c < a.cout ? n0 + i * 16 + c : a.cout - 1;
        q[i] = a.q + n * a.q_stride;
    }
}

// Scales and zero points in LDS, as fp32 [tile][group][ROWS] and bytes [tile][group][ROWS], of groups j0 .. j0 + groups of `count` tiles of ROWS weight rows,
// every wgs-th from `tile` on: read from memory by the lanes that need them, a scale of each of sixteen rows would bring a line of each of them from the XCD's
// L2 to the CU for every use.
template <int ROWS, int THREADS, int U, bool Z>   // U: loads of a thread under way
__device__ static inline void fc4_scales(const Fc4Kernel &f, int tile, int wgs, int count, int j0, int groups, float *scale, uint8_t *zero, int t) {
    const Fc4Args &a = f.a;
    const int lots = (groups + 15) / 16, total = count * lots * (16 * ROWS);   // sixteen groups of each row
    struct Place { int tile, row, j; };
    auto place = [&](int i) {
        i = i < total ? i : total - 1;
        const int lot = i / (16 * ROWS), mine = count == 1 ? 0 : (int)fast_div(lot, f.lots_div);
        return Place{mine, i / 16 % ROWS, (lot - mine * lots) * 16 + i % 16};
    };
    auto take = [&](auto *p, auto value) {
        for (int base = 0; base < total; base += U * THREADS) {
            unsigned v[U], z[U];   // words: 16-bit values packed two to a register would be waited for one by one
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Place to = place(base + u * THREADS + t);
                const int at = (tile + to.tile * wgs) * ROWS + to.row, n = at < a.cout ? at : a.cout - 1, j = j0 + (to.j < groups ? to.j : groups - 1);
                v[u] = p[n * a.scale_stride + j];
                if (Z) z[u] = a.zeros[n * a.zero_stride + j];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = base + u * THREADS + t;
                const Place at = place(i);
                const int to = (at.tile * groups + at.j) * ROWS + at.row;
                if (i < total && at.j < groups) {
                    scale[to] = value(v[u]);
                    if (Z) zero[to] = (uint8_t)z[u];
                }
            }
        }
    };
    if (a.scale_dtype == DT_F32) take(static_cast<const unsigned *>(a.scales), [](unsigned v) { return __builtin_bit_cast(float, v); });
    else if (a.scale_dtype == DT_F16) take(static_cast<const uint16_t *>(a.scales), [](unsigned v) { return (float)__builtin_bit_cast(f16, (uint16_t)v); });
    else take(static_cast<const uint16_t *>(a.scales), [](unsigned v) { return __builtin_bit_cast(float, v << 16); });
    __builtin_amdgcn_s_waitcnt(0);   // said once here, or the compiler waits in every turn of a loop behind this for loads that lanes without a place may have left
}

// The bias of the same rows, [tile][ROWS]: where a tile ends, a load would wait for the weights under way.
template <int ROWS>
__device__ static inline float fc4_bias(const Fc4Args &a, int tile, int wgs, int count, int i) {
    const int n = (tile + i / ROWS * wgs) * ROWS + i % ROWS;
    return a.bias && i < count * ROWS && n < a.cout ? a.bias[n] : 0.f;
}

// A lane has 32 inputs of its row, 8 a word; a matrix step takes 8 inputs of each of the four lanes of a row.  Word j of lane group kq becomes word kq of
// lane group j: step j then has inputs 32 j + 8 kq + 0..7, and all of a step are of one group.
__device__ static inline void fc4_turn(u32x4 &v) {
    auto r = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
    v[0] = r[0]; v[2] = r[1];
    r = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
    v[1] = r[0]; v[3] = r[1];
    r = __builtin_amdgcn_permlane16_swap(v[0], v[1], false, false);
    v[0] = r[0]; v[1] = r[1];
    r = __builtin_amdgcn_permlane16_swap(v[2], v[3], false, false);
    v[2] = r[0]; v[3] = r[1];
}

// The eight weights of a word, less their zero point, in the order (0 4) (1 5) (2 6) (3 7).  Nibbles as the low bits of fp16 numbers of exponent 10 are
// 1024 + q and 1024 + 16 q, from which q - z follows exactly.
template <bool Z>
__device__ static inline f16x8 fc4_operand(unsigned v, unsigned z, unsigned magic) {
    unsigned zlo = 0xE408E408u, zhi = 0xD480D480u;   // -(1024 + 8), -(64 + 8)
    if (Z) {
        const unsigned zz = (z & 15) * 0x10001u;
        zlo = 0xE400E400u | zz;
        zhi = 0xD400D400u | (zz << 4);
    }
    const unsigned v8 = v >> 8;
    const f16x2 sixteenth = {(f16)0.0625f, (f16)0.0625f}, clo = __builtin_bit_cast(f16x2, zlo), chi = __builtin_bit_cast(f16x2, zhi);
    const f16x2 w0 = __builtin_bit_cast(f16x2, (v & 0x000F000Fu) | magic) + clo;
    const f16x2 w1 = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00F000F0u) | magic), sixteenth, chi);
    const f16x2 w2 = __builtin_bit_cast(f16x2, (v8 & 0x000F000Fu) | magic) + clo;
    const f16x2 w3 = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v8 & 0x00F000F0u) | magic), sixteenth, chi);
    return f16x8{w0[0], w0[1], w1[0], w1[1], w2[0], w2[1], w3[0], w3[1]};
}

constexpr float kFc4LeastPower = 0x1p-113f;   // fc4_power's for blocks whose largest magnitude is 2^127 or more

// Eight activations as they are stored, from input k on (zeros behind cin).
template <int X>
struct Fc4X {
    static constexpr int WORDS = X == X_F32 ? 2 : 1;
    u32x4 raw[WORDS];
    static constexpr int SIZE = X == X_F32 ? 4 : 2;
    // From input k on, or where the row ends among them or before, its last eight (see shift).
    __device__ void load(const void *row, int k, int cin) {
        const u32x4_any *p = reinterpret_cast<const u32x4_any *>(static_cast<const char *>(row) + (int64_t)(k + 8 <= cin ? k : cin - 8) * SIZE);
#pragma unroll
        for (int i = 0; i < WORDS; ++i) raw[i] = p[i];
    }
    __device__ void shift(int k, int cin) { fc4_shift_down<4 * WORDS>(raw, k + 8 <= cin ? 0u : (unsigned)(k + 8 - cin) * (8 * SIZE)); }
    __device__ float value(int i) const {
        const unsigned word = raw[i / 4 % WORDS][i % 4];   // a bit_cast of a vector's element itself takes the first one
        if (X == X_F32) return __builtin_bit_cast(float, word);
        return __builtin_bit_cast(float, i % 2 ? raw[0][i / 2] & 0xffff0000u : raw[0][i / 2] << 16);   // bf16
    }
    // The largest magnitude, as the bits of its exponent and below.
    __device__ unsigned most() const {
        if (X == X_F32) {   // without the sign, which costs this instruction nothing; a NaN beside a number is passed over and stays one in its product
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 8; i += 2) asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(m) : "v"(m), "v"(value(i)), "v"(value(i + 1)));
            return __builtin_bit_cast(unsigned, m);
        }
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 m = __builtin_bit_cast(u16x2, raw[0][0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, raw[0][i] & 0x7fff7fffu));
        return (unsigned)(m[0] > m[1] ? m[0] : m[1]) << 16;
    }
    // In the order in which the weights come, times `by`: the rounded value and, of fp32, what the rounding left.
    __device__ void operands(float by, f16x8 &hi, f16x8 &lo) const {
        if (X == X_F16) {
            const u32x4 v = raw[0];
            const u32x4 o = {__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                             __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
            hi = __builtin_bit_cast(f16x8, o);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v0 = value(i) * by, v1 = value(i + 4) * by;
            if (X == X_BF16) {   // eight bits fit: only what is below 2^-24 of the scaled range is cut off
                const auto p = __builtin_amdgcn_cvt_pkrtz(v0, v1);
                hi[2 * i] = (f16)p[0];
                hi[2 * i + 1] = (f16)p[1];
            } else {
                typedef float f32x2 __attribute__((ext_vector_type(2)));
                f16x2 p = __builtin_convertvector((f32x2{v0, v1}), f16x2);
                asm("" : "+v"(p));   // products and halves are made once: again for each use they would be mixed fmas, which take longer than two instructions
                hi[2 * i] = p[0];
                hi[2 * i + 1] = p[1];
                lo[2 * i] = (f16)fmaf((float)p[0], -1.f, v0);
                lo[2 * i + 1] = (f16)fmaf((float)p[1], -1.f, v1);
            }
        }
        // What an infinity leaves is no number.  Half a step of a number below 2^15 is 8 at most; 16 is what the infinity outweighs.
        if (X == X_F32 && __builtin_expect(by == kFc4LeastPower, 0)) lo = __builtin_elementwise_min(lo, (f16x8)(f16)16.f);
    }
};
// 2^(14 - e) for a largest magnitude of 2^e..2^(e+1): its numbers stay below 2^15; and 2^(e - 14).  Neither leaves fp32's range.
__device__ static inline void fc4_power(unsigned most, float &by, float &back) {
    int e = (int)(most >> 23) - 127;
    e = e > 127 ? 127 : e < -112 ? -112 : e;
    by = __builtin_bit_cast(float, (unsigned)(14 - e + 127) << 23);
    back = __builtin_bit_cast(float, (unsigned)(e - 14 + 127) << 23);
}

// The largest of 16 lanes' numbers.
__device__ static inline unsigned fc4_max_row(unsigned v) {
    auto join = [&](int o) { v = v > (unsigned)o ? v : (unsigned)o; };
    join(__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));    // lanes 1 0 3 2
    join(__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));    // lanes 2 3 0 1
    join(__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // mirrored in 8
    join(__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));   // mirrored in 16
    return v;
}

// ---- few rows: up to 16 of x, which LDS holds -----------------------------------------------------------
// x lies in LDS as fp16 operands, [part][block][row][128], made once a workgroup, and so do the scales of all its weight rows.  The workgroup walks tiles
// of 16 NT weight rows; its eight waves take the blocks of K in turn and two blocks a wave are under way all the time, also from one tile to the next.
// Bound: the weights' way from HBM.  1 x 8192 to 32001 in groups of 128: 135 MB in 32-33 us, 4.1 TB/s (a copy of 1 GiB: 5.0); 1 x 4096 to 4096 4.8 us, of
// which an empty launch is 2.1 and the trip to HBM and the meeting of the waves the most of the others.
constexpr int kFewWaves = 8;
template <int X, int NT, int GM, bool Z>
__global__ __launch_bounds__(64 * kFewWaves) void fc4_few_kernel(const Fc4Kernel f, int tiles, int wgs, int groups, int own) {   // own: tiles of a workgroup at most
    constexpr int KW = kFewWaves, D = 2, THREADS = 64 * KW, PARTS = X == X_F32 ? 2 : 1, MEET = KW * NT * 256, ROWS = 16 * NT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Fc4Args &a = f.a;
    const int t = threadIdx.x, lane = t & 63, kw = __builtin_amdgcn_readfirstlane(t >> 6);
    const int c = lane & 15, kq = lane >> 4;
    const int rows = a.rows, blocks = (a.cin + kBlock - 1) / kBlock, part_bytes = blocks * rows * (kBlock * 2);
    float *meet = reinterpret_cast<float *>(lds + PARTS * part_bytes), *xs = meet + 2 * MEET;           // xs: [block][16], what x was divided by
    float *bias = xs + (X == X_F16 ? 0 : blocks * 16), *scales = bias + own * ROWS;                         // [tile][ROWS], [tile][group][ROWS]
    uint8_t *zeros = reinterpret_cast<uint8_t *>(scales + own * groups * ROWS);
    const int mine = (blocks - kw + KW - 1) / KW;   // blocks of a tile: kw, kw + KW, ...
    const int todo_tiles = (tiles - (int)blockIdx.x + wgs - 1) / wgs, todo = todo_tiles * mine;

    // The next block to ask for.
    const uint8_t *q[NT];
    Fc4Weights<NT> w[D];
    int at_tile = blockIdx.x, at = kw;
    fc4_rows<NT>(q, a, at_tile * ROWS, c);
    auto ask = [&](Fc4Weights<NT> &to) {
        to.load(f, q, at, kq);
        at += KW;
        if (at >= blocks) {   // behind the last tile: its last block again
            const bool more = at_tile + wgs < tiles;
            at = more ? kw : at - KW;
            if (more) {
                at_tile += wgs;
                fc4_rows<NT>(q, a, at_tile * ROWS, c);
            }
        }
    };
    if (todo > 0)
#pragma unroll
        for (int u = 0; u < D; ++u) ask(w[u]);

    const float first_bias = fc4_bias<ROWS>(a, blockIdx.x, wgs, todo_tiles, t);
    constexpr int U = 4;   // pieces of eight inputs a thread has under way; sixteen threads a row and block
    const int piece = t & 15;
    for (int base = 0; base < rows * blocks * 16; base += U * THREADS) {
        Fc4X<X> x[U];
        int row[U], block[U];
        const int item = base + t;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (base + u * THREADS >= rows * blocks * 16) break;
            const int at = (item + u * THREADS) >> 4, rb = at < rows * blocks ? at : rows * blocks - 1;
            block[u] = rows == 1 ? rb : rb / rows;
            row[u] = rb - block[u] * rows;
            x[u].load(static_cast<const char *>(a.x) + row[u] * a.x_stride * (X == X_F32 ? 4 : 2), block[u] * kBlock + piece * 8, a.cin);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (item + u * THREADS >= rows * blocks * 16) break;
            const int k = block[u] * kBlock + piece * 8;
            if (k + 8 > a.cin) x[u].shift(k, a.cin);
            float by = 1.f, back;
            if (X != X_F16) {
                fc4_power(fc4_max_row(x[u].most()), by, back);
                if (piece == 0) xs[block[u] * 16 + row[u]] = back;
            }
            f16x8 hi, lo;
            x[u].operands(by, hi, lo);
            char *to = lds + (block[u] * rows + row[u]) * (kBlock * 2) + ((piece ^ row[u]) << 4);
            *reinterpret_cast<f16x8 *>(to) = hi;
            if (X == X_F32) *reinterpret_cast<f16x8 *>(to + part_bytes) = lo;
        }
    }
    fc4_scales<ROWS, THREADS, 2, Z>(f, blockIdx.x, wgs, todo_tiles, 0, groups, scales, zeros, t);
    for (int i = t; i < todo_tiles * ROWS; i += THREADS) bias[i] = i == t ? first_bias : fc4_bias<ROWS>(a, blockIdx.x, wgs, todo_tiles, i);
    __syncthreads();

    // A row's sixteen pieces of a block change places with the row's number: every sixteen lanes write, and read, 256 different bytes of the 256 that LDS serves at a time.
    const int xrow = c < rows ? c : rows - 1;
    int xat[4];
#pragma unroll
    for (int step = 0; step < 4; ++step) xat[step] = xrow * (kBlock * 2) + (((step * 4 + kq) ^ xrow) << 4);
    unsigned magic = 0x64006400u;
    asm("" : "+v"(magic));   // in a register
    f32x4 total[NT] = {};
    int tile = blockIdx.x, side = 0, block = kw, slot = c;   // slot: this lane's first row among the scales
    auto work = [&](Fc4Weights<NT> &v) {
        const f32x4 back = X != X_F16 ? *reinterpret_cast<const f32x4 *>(xs + block * 16 + kq * 4) : f32x4{};
        if ((block + 1) * kBlock > a.cin) v.shift(f, block, kq);
#pragma unroll
        for (int j = 0; j < NT; ++j) fc4_turn(v.w[j]);
        f32x4 p[NT];
        int at[4 / GM];
#pragma unroll
        for (int g = 0; g < 4 / GM; ++g) {
            const int k = block * kBlock + g * GM * 32;
            at[g] = slot + (int)fast_div(k < a.cin ? k : a.cin - 1, f.group_div) * ROWS;
        }
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            f16x8 x[PARTS];
#pragma unroll
            for (int part = 0; part < PARTS; ++part) x[part] = *reinterpret_cast<const f16x8 *>(lds + part * part_bytes + block * rows * (kBlock * 2) + xat[step]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const f16x8 ww = fc4_operand<Z>(v.w[j][step], Z ? zeros[at[step / GM] + j * 16] : 0u, magic);
                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                p[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[0], ww, step % GM == 0 ? zero : p[j], 0, 0, 0);
                if (X == X_F32) p[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[PARTS - 1], ww, p[j], 0, 0, 0);
                if (step % GM == GM - 1) {
                    const float scale = scales[at[step / GM] + j * 16];
#pragma unroll
                    for (int e = 0; e < 4; ++e) total[j][e] = X == X_F16 ? fmaf(p[j][e], scale, total[j][e]) : fmaf(p[j][e] * scale, back[e], total[j][e]);
                }
            }
        }
        block += KW;
    };
    // The end of a tile: the sums of the waves in LDS, [kw][tile][4][64], on the two sides in turn.
    auto finish = [&]() {
        float *part = meet + side * MEET;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                part[((kw * NT + j) * 4 + e) * 64 + lane] = total[j][e];
                total[j][e] = 0.f;
            }
        __syncthreads();
        for (int o = t; o < NT * 256; o += THREADS) {   // o = (tile of 16, e, lane)
            const int l = o & 63, m = (l >> 4) * 4 + ((o >> 6) & 3), n = tile * ROWS + (o >> 8) * 16 + (l & 15);
            if (m >= rows || n >= a.cout) continue;
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < KW; ++k) v += part[k * (NT * 256) + o];
            fc4_store(a.y, m * a.y_stride + n, a.y_dtype, v + bias[(o >> 8) * 16 + (l & 15)]);
        }
        tile += wgs;
        side ^= 1;
        block = kw;
        slot += groups * ROWS;
        bias += ROWS;
    };
    if (todo == 0) {   // fewer blocks than waves
        while (tile < tiles) finish();
        return;
    }
    int done = 0;
    for (; done + D < todo; done += D)
#pragma unroll
        for (int u = 0; u < D; ++u) {
            work(w[u]);
            ask(w[u]);
            if (block >= blocks) finish();
        }
#pragma unroll
    for (int u = 0; u < D; ++u)
        if (done + u < todo) {
            work(w[u]);
            if (block >= blocks) finish();
        }
}

// ---- many rows --------------------------------------------------------------------------------------
// A workgroup computes 16 MT rows by 16 NT NW weight rows; its KW groups of waves take the blocks of K in turn.  The NW waves of a group stage the group's
// phase, PB blocks of x, in one of two LDS buffers while they multiply the other one, from registers that were loaded two blocks before; weights go straight
// to the registers of the wave that multiplies them, as early.
// Bound: vector instructions, next to which the matrix cores run: of a block's 16 weight rows and 64 rows of x about 90 to make operands and scale sums and
// 16 on the matrix cores, which twice the rows share (fp16, 64 x 4096 to 16384: vector units 52% of the time, matrix cores 18%; 2048 x 8192 to 8192: 52% and 46%; bf16, 512 x 4096 to 4096: 80% and 23%).
// Two blocks between barriers: 512 x 4096 to 4096 fp16 26.1 -> 25.2 us; 32 x 4096 to 16384 14.3 -> 13.2.
template <int X, int MT, int NT, int NW, int KW, int PB>
struct Fc4Many {
    static constexpr int ROWS = 16 * MT, COLS = 16 * NT * NW, THREADS = 64 * NW * KW, PARTS = X == X_F32 ? 2 : 1, ITEMS = ROWS / 4 / NW;   // ITEMS of a wave: four rows of a block each
    static constexpr int PART = 4 * ROWS * 64, BUFFER = PARTS * PART + (X == X_F16 ? 0 : ROWS * 4);   // bytes of a block: operands, and what a row was divided by
    static constexpr int STAGED = KW * 2 * PB * BUFFER, MEET = NW * (KW - 1) * MT * NT * 1024, FIXED = (STAGED > MEET ? STAGED : MEET) + COLS * 4;   // LDS: x, where later the groups meet; the bias; the scales
};

template <int X, int MT, int NT, int NW, int KW, int PB, int GM, bool Z>
__global__ __launch_bounds__(64 * NW * KW) void fc4_many_kernel(const Fc4Kernel f, int chunk, int chunk_groups) {   // chunk: phases whose scales LDS holds, in chunk_groups groups
    typedef Fc4Many<X, MT, NT, NW, KW, PB> S;
    constexpr int ROWS = S::ROWS, COLS = S::COLS, PARTS = S::PARTS, ITEMS = S::ITEMS, PART = S::PART, BUFFER = S::BUFFER;
    static_assert(ROWS / 4 % NW == 0, "rows in fours, evenly");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Fc4Args &a = f.a;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), nw = wave % NW, kw = wave / NW;
    const int c = lane & 15, kq = lane >> 4;
    const int m0 = blockIdx.y * ROWS, rows = a.rows - m0 < ROWS ? a.rows - m0 : ROWS;
    const uint8_t *q[NT];
    fc4_rows<NT>(q, a, (blockIdx.x * NW + nw) * (16 * NT), c);
    char *const mine = lds + kw * (2 * PB * BUFFER);
    float *bias = reinterpret_cast<float *>(lds + S::FIXED - COLS * 4), *scales = reinterpret_cast<float *>(lds + S::FIXED);
    uint8_t *zeros = reinterpret_cast<uint8_t *>(scales + chunk_groups * COLS);
    f32x4 total[MT][NT] = {};
    unsigned magic = 0x64006400u;
    asm("" : "+v"(magic));   // in a register

    // Staging: sixteen lanes a row, whose sixteen pieces of a block change places with the row's number (modulo 16): every sixteen lanes write, and read, 256
    // different bytes of the 256 that LDS serves at a time.
    Fc4X<X> x[2][ITEMS];
    const int piece = lane & 15;
    const char *xrow[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int row = (nw * ITEMS + i) * 4 + (lane >> 4);
        xrow[i] = static_cast<const char *>(a.x) + (m0 + (row < rows ? row : rows - 1)) * a.x_stride * (X == X_F32 ? 4 : 2);
    }
    const int whole = a.cin / kBlock, phases = (whole + PB * KW - 1) / (PB * KW);
    auto place_of = [&](int phase, int u) { return (phase * KW + kw) * PB + u; };
    auto block_of = [&](int phase, int u) {   // behind the last whole block: that one again
        const int block = place_of(phase, u);
        return block < whole ? block : whole - 1;
    };
    auto ask_x = [&](int block, Fc4X<X> (&to)[ITEMS]) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) to[i].load(xrow[i], block * kBlock + piece * 8, a.cin);
    };
    auto stage = [&](Fc4X<X> (&v)[ITEMS], char *to) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int row = (nw * ITEMS + i) * 4 + (lane >> 4);
            float by = 1.f, back;
            if (X != X_F16) {
                fc4_power(fc4_max_row(v[i].most()), by, back);
                if (piece == 0) reinterpret_cast<float *>(to + PARTS * PART)[row] = back;
            }
            f16x8 hi, lo;
            v[i].operands(by, hi, lo);
            char *at = to + row * (kBlock * 2) + (((piece ^ row) & 15) << 4);
            *reinterpret_cast<f16x8 *>(at) = hi;
            if (X == X_F32) *reinterpret_cast<f16x8 *>(at + PART) = lo;
        }
    };
    Fc4Weights<NT> w[2];
    const int slot = nw * (16 * NT) + c;
    int xat[4];
#pragma unroll
    for (int step = 0; step < 4; ++step) xat[step] = c * (kBlock * 2) + (((step * 4 + kq) ^ c) << 4);
    int j0 = 0;   // first group of the chunk
    auto multiply = [&](Fc4Weights<NT> &v, int block, const char *from) {
#pragma unroll
        for (int j = 0; j < NT; ++j) fc4_turn(v.w[j]);
        f32x4 p[MT][NT];
        int at[4 / GM];
#pragma unroll
        for (int g = 0; g < 4 / GM; ++g) {
            const int k = block * kBlock + g * GM * 32;
            at[g] = slot + ((int)fast_div(k < a.cin ? k : a.cin - 1, f.group_div) - j0) * COLS;
        }
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            f16x8 xx[PARTS][MT];
#pragma unroll
            for (int part = 0; part < PARTS; ++part)
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    xx[part][i] = *reinterpret_cast<const f16x8 *>(from + part * PART + i * (16 * kBlock * 2) + xat[step]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const f16x8 ww = fc4_operand<Z>(v.w[j][step], Z ? zeros[at[step / GM] + j * 16] : 0u, magic);
                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xx[0][i], ww, step % GM == 0 ? zero : p[i][j], 0, 0, 0);
                    if (X == X_F32) p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xx[PARTS - 1][i], ww, p[i][j], 0, 0, 0);
                }
            }
            if (step % GM == GM - 1) {
                float scale[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) scale[j] = scales[at[step / GM] + j * 16];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const f32x4 back = X != X_F16 ? *reinterpret_cast<const f32x4 *>(from + PARTS * PART + (i * 16 + kq * 4) * 4) : f32x4{};
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            total[i][j][e] = X != X_F16 ? fmaf(p[i][j][e] * scale[j], back[e], total[i][j][e]) : fmaf(p[i][j][e], scale[j], total[i][j][e]);
                }
            }
        }
    };
    auto take_scales = [&](int phase) {   // of the next `chunk` phases
        const int k0 = phase * PB * KW * kBlock, k1 = k0 + chunk * PB * KW * kBlock;
        j0 = (int)fast_div(k0, f.group_div);
        fc4_scales<COLS, S::THREADS, 4, Z>(f, blockIdx.x, 1, 1, j0, (int)fast_div((k1 < a.cin ? k1 : a.cin) - 1, f.group_div) - j0 + 1, scales, zeros, t);
    };
    const float my_bias = fc4_bias<COLS>(a, blockIdx.x, 1, 1, t);
    if (phases > 0) {
        // Of a group's two blocks under way, PB are a phase's: one of each of two phases, or both of one.
        auto ahead = [&](int phase, int u, int by) { return block_of(phase + (PB == 2 ? by / 2 : by), PB == 2 ? u : 0); };
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            w[u].load(f, q, ahead(PB == 2 ? 0 : u, u, 0), kq);
            ask_x(ahead(PB == 2 ? 0 : u, u, 0), x[u]);
        }
        take_scales(0);
#pragma unroll
        for (int u = 0; u < PB; ++u) {
            stage(x[u], mine + u * BUFFER);
            ask_x(ahead(0, u, 2), x[u]);
        }
        for (int from = 0; from < phases; from += chunk) {   // chunks of an even number of phases, or one
            if (from > 0) {
                __syncthreads();
                take_scales(from);
            }
            const int to = from + chunk < phases ? from + chunk : phases;
            if constexpr (PB == 1) {
                for (int phase = from; phase < to; phase += 2) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        __syncthreads();
                        const int block = place_of(phase + u, 0);
                        if (block < whole) multiply(w[u], block, mine + u * BUFFER);   // an odd last phase has a second one with nothing to multiply
                        w[u].load(f, q, ahead(phase + u, 0, 2), kq);
                        stage(x[1 - u], mine + (1 - u) * BUFFER);
                        ask_x(ahead(phase + u, 0, 3), x[1 - u]);
                    }
                }
            } else {
                for (int phase = from; phase < to; ++phase) {
                    __syncthreads();
                    char *const here = mine + (phase & 1) * (2 * BUFFER), *const there = mine + (~phase & 1) * (2 * BUFFER);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int block = place_of(phase, u);
                        if (block < whole) multiply(w[u], block, here + u * BUFFER);
                        w[u].load(f, q, ahead(phase, u, 2), kq);
                        stage(x[u], there + u * BUFFER);
                        ask_x(ahead(phase, u, 4), x[u]);
                    }
                }
            }
        }
    }
    if (whole * kBlock < a.cin) {   // the rest of K is one group's
        __syncthreads();
        if (whole % (PB * KW * chunk) == 0) take_scales(phases);
        if (kw == 0) {
            ask_x(whole, x[0]);
            w[0].load(f, q, whole, kq);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) x[0][i].shift(whole * kBlock + piece * 8, a.cin);
            w[0].shift(f, whole, kq);
            stage(x[0], mine);
        }
        __syncthreads();
        if (kw == 0) multiply(w[0], whole, mine);
    }
    // The groups of waves meet in LDS: [kw > 0][nw][tile][4][64]; the first group adds its own and stores.
    __syncthreads();
    if (t < COLS) bias[t] = my_bias;
    float *part = reinterpret_cast<float *>(lds) + nw * (MT * NT * 256) + lane;
    constexpr int GROUP = NW * MT * NT * 256;
    if (kw > 0)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[(kw - 1) * GROUP + ((i * NT + j) * 4 + e) * 64] = total[i][j][e];
    __syncthreads();
    if (kw > 0) return;
    auto put = [&](auto *y) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int col = (nw * NT + j) * 16 + c, n = blockIdx.x * COLS + col;
            const float add = bias[col];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int m = i * 16 + kq * 4 + e;
                    float v = total[i][j][e];
#pragma unroll
                    for (int k = 1; k < KW; ++k) v += part[(k - 1) * GROUP + ((i * NT + j) * 4 + e) * 64];
                    if (m < rows && n < a.cout) y[(m0 + m) * a.y_stride + n] = (typename std::remove_pointer<decltype(y)>::type)(v + add);
                }
        }
    };
    if (a.y_dtype == DT_F32) put(static_cast<float *>(a.y));
    else if (a.y_dtype == DT_F16) put(static_cast<f16 *>(a.y));
    else put(static_cast<bf16 *>(a.y));
}

// ---- the choice of a form ----------------------------------------------------------------------------
struct Fc4Plan {
    enum Form { SHORT, FEW, FEW_PAIRS, MANY1_16, MANY1_32, MANY1_64, MANY2_32, MANY2_64, MANY4_64, MANY4_128, MANY4_256, MANY8_256 } form;
    int rows, cols, threads;   // of a workgroup; FEW and FEW_PAIRS: `cols` at a time
    int most;                  // workgroups of those
};
Fc4Plan fc4_plan(const Fc4Args &a);

constexpr int kLdsBytes = 160 * 1024;
// LDS of a workgroup of few rows: two share a CU.  fp32 activations may have all of it where there is a workgroup for each CU at most: 16 x 2048 to
// 1000 7.0 us, in the form for many rows, which converts them as often, 7.4; but fp16 16 x 4096 to 4096 8.6 us, and 7.1 in that form.
constexpr int few_lds(bool fp32, int64_t tiles) { return fp32 && tiles <= 256 ? kLdsBytes : kLdsBytes / 2; }

static int fc4_groups(const Fc4Args &a) { return (int)fc4_layout(a.cin, a.cout, a.group).groups; }   // `group` may be anything up to 2^31 - 32
static Fc4Kernel fc4_kernel_args(const Fc4Args &a) { return {a, make_fast_div((uint32_t)a.group), make_fast_div((uint32_t)(fc4_groups(a) + 15) / 16)}; }

// How fc4_few_kernel walks tiles of 16 NT weight rows: at most `most` workgroups, an even share of the tiles each, as far as LDS has room for
// their scales (a place for zero points is counted where there are none too).
struct Fc4Few {
    int tiles, own, wgs;    // wgs 0: x does not fit
    int64_t fixed, tile;    // LDS without the scales, and of the scales of a tile
};
static Fc4Few fc4_few(const Fc4Args &a, int nt, int most) {
    const int64_t blocks = (a.cin + kBlock - 1) / kBlock;
    Fc4Few f;
    f.tiles = (a.cout + 16 * nt - 1) / (16 * nt);
    f.fixed = (a.x_dtype == DT_F32 ? 2 : 1) * a.rows * blocks * kBlock * 2 + 2 * kFewWaves * nt * 1024 + (a.x_dtype == DT_F16 ? 0 : blocks * 64);
    f.tile = ((int64_t)fc4_groups(a) * 5 + 4) * (16 * nt);
    const int64_t fit = (few_lds(a.x_dtype == DT_F32, f.tiles) - f.fixed) / f.tile;
    f.own = (f.tiles + most - 1) / most;
    f.own = f.own < fit ? f.own : (int)fit;
    f.wgs = f.own > 0 ? (f.tiles + f.own - 1) / f.own : 0;
    return f;
}

template <int X, int NT, int GM, bool Z>
static hipError_t launch_few(const Fc4Args &a, const Fc4Plan &p, hipStream_t s) {
    const Fc4Few f = fc4_few(a, NT, p.most);
    if (a.rows > 16 || a.cin < kShortIn || f.wgs < 1 || p.cols != 16 * NT || p.threads != 64 * kFewWaves) return hipErrorInvalidValue;
    fc4_few_kernel<X, NT, GM, Z><<<dim3(f.wgs), 64 * kFewWaves, (size_t)(f.fixed + f.own * f.tile), s>>>(fc4_kernel_args(a), f.tiles, f.wgs, fc4_groups(a), f.own);
    return hipGetLastError();
}

template <int X, int MT, int NT, int NW, int KW, int PB, int GM, bool Z>
static hipError_t launch_many(const Fc4Args &a, const Fc4Plan &p, hipStream_t s) {
    typedef Fc4Many<X, MT, NT, NW, KW, PB> S;
    static_assert(S::FIXED + (2 * KW * 4 / GM + 1) * S::COLS * 5 <= kLdsBytes, "LDS");
    if (a.cin < kShortIn || p.rows != S::ROWS || p.cols != S::COLS || p.threads != S::THREADS) return hipErrorInvalidValue;
    // The scales of as many phases as fit.  Inputs that begin anywhere touch a group more than they fill.
    const int phases = (a.cin + PB * KW * kBlock - 1) / (PB * KW * kBlock), most = (kLdsBytes - S::FIXED) / (S::COLS * (Z ? 5 : 4));
    int chunk = phases, groups = fc4_groups(a);
    while (groups > most && chunk > 2 / PB) {   // an even number of them with one block each
        chunk = PB == 2 ? (chunk + 1) / 2 : (chunk + 3) / 4 * 2;
        groups = (int)(((int64_t)chunk * PB * KW * kBlock + a.group - 1) / a.group) + 1;
    }
    if (groups > most) return hipErrorInvalidValue;
    const int bytes = S::FIXED + groups * S::COLS * (Z ? 5 : 4);
    for (int m = 0; m < a.rows; m += 65535 * S::ROWS) {   // rows beyond the grid's y
        Fc4Kernel f = fc4_kernel_args(a);
        f.a.rows = a.rows - m < 65535 * S::ROWS ? a.rows - m : 65535 * S::ROWS;
        f.a.x = static_cast<const char *>(a.x) + m * a.x_stride * (a.x_dtype == DT_F32 ? 4 : 2);
        f.a.y = static_cast<char *>(a.y) + m * a.y_stride * (a.y_dtype == DT_F32 ? 4 : 2);
        fc4_many_kernel<X, MT, NT, NW, KW, PB, GM, Z><<<dim3((a.cout + S::COLS - 1) / S::COLS, (f.a.rows + S::ROWS - 1) / S::ROWS), S::THREADS, bytes, s>>>(f, chunk, groups);
    }
    return hipGetLastError();
}

template <int X>
hipError_t launch_fc4_x(const Fc4Args &a, const Fc4Plan &p, hipStream_t s);

template <int X, int GM, bool Z>
static hipError_t launch_fc4_form(const Fc4Args &a, const Fc4Plan &p, hipStream_t s) {
    constexpr bool two = X == X_F32;   // operands in two parts: twice the LDS
    switch (p.form) {
        case Fc4Plan::FEW: return launch_few<X, 1, GM, Z>(a, p, s);
        case Fc4Plan::FEW_PAIRS: return launch_few<X, 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY1_16: return launch_many<X, 1, 1, 1, 8, 1, GM, Z>(a, p, s);
        case Fc4Plan::MANY1_32: return launch_many<X, 1, 1, 2, 4, 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY1_64: return launch_many<X, 1, 1, 4, 4, 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY2_32: return launch_many<X, 2, 1, 2, 4, two ? 1 : 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY2_64: return launch_many<X, 2, 1, 4, two ? 4 : 2, two ? 1 : 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY4_64: return launch_many<X, 4, 1, 4, 2, two ? 1 : 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY4_128: return launch_many<X, 4, 1, 8, 2, two ? 1 : 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY4_256: return launch_many<X, 4, 2, 8, 1, two ? 1 : 2, GM, Z>(a, p, s);
        case Fc4Plan::MANY8_256:
            if constexpr (X == X_F16) return launch_many<X, 8, 2, 8, 1, 1, GM, Z>(a, p, s);
        default: return hipErrorInvalidValue;
    }
}

template <int X>
hipError_t launch_fc4_x(const Fc4Args &a, const Fc4Plan &p, hipStream_t s) {
    if (a.group % 128 == 0) return a.zeros ? launch_fc4_form<X, 4, true>(a, p, s) : launch_fc4_form<X, 4, false>(a, p, s);
    if (a.group % 64 == 0) return a.zeros ? launch_fc4_form<X, 2, true>(a, p, s) : launch_fc4_form<X, 2, false>(a, p, s);
    return a.zeros ? launch_fc4_form<X, 1, true>(a, p, s) : launch_fc4_form<X, 1, false>(a, p, s);
}

}  // namespace cw
