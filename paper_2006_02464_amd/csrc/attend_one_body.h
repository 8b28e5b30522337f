// The attention kernel of single tokens over a paged cache (cw_attend_one has the definition), a type of queries and of pages to a source file.
#pragma once
#include <cmath>

#include "attend_common.h"
#include "lds_loads.h"

namespace cw {

// Reading keys and values is what this costs: everything serves to keep enough of their bytes under way.  A workgroup takes up to 16 of the query heads that share a key head, and a part of a
// sequence's tokens; its waves walk shares of that by themselves, 32 tokens a step, K and V of the next step on their way straight to the wave's own LDS while this one is worked on.
// Products are transposed, on 16 x 16 tiles of the matrix cores: S^T = K Q^T, whose lanes have a query and tokens 4 (lane / 16) + 0..3 of each half of the step, just what the second product,
// O^T = V^T P^T, wants of P^T with its tokens in that order; V is transposed by the reads of LDS that do that.  Tokens that are not seen come from a line of zeros.
// Codes of 8 bits become numbers of the queries' type for the first product and fp16 for the second, exactly; a key's exponent goes to its score, a value's to its weight before that is rounded:
// weights refer to a maximum of their own.  bf16 weights go into the second product in two parts.
constexpr int kOneTokens = 32;
constexpr int kOneHeads = 16;
constexpr float kOneSlack = 8.f;   // maxima follow beyond 2^8
constexpr int kOneMostParts = 64;
constexpr int kOneCounters = 65536 / 4;

struct AttendOneKernel {
    AttendOneArgs a;
    int32_t group, blocks;   // query heads of a key head, blocks of kOneHeads of them
    int32_t parts;
    float c;                 // |scale| / ln 2
};

constexpr int one_waves(int row_bytes) { return row_bytes > 256 ? 2 : 4; }
// Where 16-byte chunk c of row r lies: what is read at once lies in different banks.  K: 16 rows, one chunk; V: 8 rows, two chunks (16 bits) or rows 0..7 and 16..23, one (codes).
template <int RB>
__device__ static inline int k_key(int r) { return RB >= 256 ? r & 15 : RB == 128 ? (r >> 1) & 7 : (r >> 2) & 3; }
template <int RB, bool CODES>
__device__ static inline int v_key(int r) {
    if (CODES) return RB == 256 ? (r & 7) | (r >> 4 & 1) << 3 : RB == 128 ? (r >> 1 & 3) | (r >> 4 & 1) << 2 : (r >> 2 & 1) | (r >> 4 & 1) << 1;
    return RB >= 256 ? (r & 7) << 1 : (r >> 1 & 3) << 1;
}

// Eight codes as numbers.
template <typename T>
__device__ static inline typename Mfma<T>::v8 decode8(unsigned lo, unsigned hi) {
    auto two = [](unsigned codes, auto upper) {
        if constexpr (std::is_same<T, f16>::value) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, decltype(upper)::value));
        else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, decltype(upper)::value));
    };
    return __builtin_bit_cast(typename Mfma<T>::v8, u32x4{two(lo, std::false_type{}), two(lo, std::true_type{}), two(hi, std::false_type{}), two(hi, std::true_type{})});
}

static __device__ const unsigned __attribute__((aligned(16))) one_zeros[4] = {0u, 0u, 0u, 0u};

// The largest of lanes l, l + 16, l + 32, l + 48, and their sum.
template <typename F>
__device__ static inline float of_four(float v, F f) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = f(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
    const unsigned w = __builtin_bit_cast(unsigned, v);
    r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return f(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}

// T: queries; CODES: pages of e4m3, else of T.  RB: bytes of a row in LDS, at least those of a head.
template <typename T, bool CODES, int RB>
__global__ __launch_bounds__(64 * one_waves(RB)) void attend_one_kernel(const AttendOneKernel f) {
    typedef typename std::conditional<CODES, f16, T>::type VT;    // of the second product
    typedef typename Mfma<T>::v8 v8;
    typedef typename Mfma<VT>::v8 w8;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) unsigned char lds_char;
    constexpr int WAVES = one_waves(RB), THREADS = 64 * WAVES, SIZE = CODES ? 1 : 2, DP = RB / SIZE;
    constexpr int PART = kOneTokens * RB, EXPS = CODES ? 256 : 0, STAGE = 2 * PART + EXPS, LOADS = PART / 1024;
    constexpr bool TWO = std::is_same<VT, bf16>::value;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * WAVES * STAGE];
    __shared__ float tops[WAVES][kOneHeads], sums[WAVES][kOneHeads];
    __shared__ int last;
    const AttendOneArgs &a = f.a;
    const CacheView &c = a.cache;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
    int b = blockIdx.x;
    const int part = b % f.parts;
    b /= f.parts;
    const int item = b, kvh = b % c.kv_heads;
    b /= c.kv_heads;
    const int block = b % f.blocks, s = b / f.blocks;
    const int heads = min(kOneHeads, f.group - block * kOneHeads), head0 = kvh * f.group + block * kOneHeads;

    const int full = max(a.lengths[s], 0), from = a.window > 0 ? max(0, full - a.window) : 0, len = min(full, a.table_pages << c.page_shift);
    const int step0 = from / kOneTokens, steps = len > from ? (len + kOneTokens - 1) / kOneTokens - step0 : 0;
    const int parts = max(1, min(f.parts, steps / (2 * WAVES)));   // as many as have two steps for every wave
    if (part >= parts) return;
    const int unit = part * WAVES + wave, units = parts * WAVES;
    int step = step0 + (int)((int64_t)steps * unit / units);
    const int end = step0 + (int)((int64_t)steps * (unit + 1) / units);

    // Q as the second operand of the first product: with codes 16 numbers of a head in a row, whose halves two steps of the product take.
    v8 q[DP / 32];
    {
        const T *at = static_cast<const T *>(a.q) + s * a.q_stride + (int64_t)(head0 + col) * a.q_head_stride;
        const unsigned sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            const int d = CODES ? (i >> 1) * 64 + quad * 16 + (i & 1) * 8 : i * 32 + quad * 8;
            u32x4 w = {0u, 0u, 0u, 0u};
            if (col < heads && d < c.head_dim) w = *reinterpret_cast<const u32x4 *>(at + d);
            w ^= sign;
            q[i] = __builtin_bit_cast(v8, w);
        }
    }

    lds_char *const mine = (lds_char *)lds + wave * 2 * STAGE;
    const unsigned mine_at = (unsigned)(size_t)mine;
    const int32_t *table = a.table + s * a.table_stride;
    const char *k_head = static_cast<const char *>(c.k) + kvh * c.head_stride * SIZE, *v_head = static_cast<const char *>(c.v) + kvh * c.head_stride * SIZE;
    int table_base = 0, entries = -1;    // a lane's page of the sequence's pages table_base..table_base + 63
    bool have_table = false;
    unsigned seen = 0, seen_next = 0;    // tokens of the step at hand and of the next one, a bit each
    auto load = [&](int st) {
        const int t0 = st * kOneTokens, token = t0 + (lane & 31);
        if (!have_table || ((t0 + kOneTokens - 1) >> c.page_shift) - table_base >= 64) {
            have_table = true;
            table_base = t0 >> c.page_shift;
            const int at = table_base + lane;
            const int page = at < a.table_pages ? table[at] : -1;
            entries = (unsigned)page < (unsigned)c.pages ? page : -1;
        }
        const int page = __shfl(entries, (token >> c.page_shift) - table_base), in = token & ((1 << c.page_shift) - 1);
        const bool ok = page >= 0 && token >= from && token < len;
        seen_next = (unsigned)__ballot(ok);
        const int64_t row = ok ? (page * c.page_stride + in * c.token_stride) * SIZE : -1;
        const int row_lo = (int)row, row_hi = (int)(row >> 32);
        const unsigned to = mine_at + (st & 1) * STAGE;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int r = (j * 64 + lane) * 16 / RB, pos = lane & (RB / 16 - 1);
            const int kc = pos ^ k_key<RB>(r), vc = pos ^ v_key<RB, CODES>(r);
            const int64_t at = (int64_t)__shfl(row_hi, r) << 32 | (unsigned)__shfl(row_lo, r);
            const char *zero = reinterpret_cast<const char *>(one_zeros);
            load_to_lds(at >= 0 && kc * 16 < c.head_dim * SIZE ? k_head + at + kc * 16 : zero, to + j * 1024);
            load_to_lds(at >= 0 && vc * 16 < c.head_dim * SIZE ? v_head + at + vc * 16 : zero, to + PART + j * 1024);
        }
        if constexpr (CODES) {
            const char *e = reinterpret_cast<const char *>(lane < 32 ? c.k_exp : c.v_exp) + page * c.exp_page_stride + kvh * c.exp_head_stride + in * c.exp_token_stride;
            load_byte_to_lds(ok ? e : reinterpret_cast<const char *>(one_zeros), to + 2 * PART);
        }
    };

    f32x4 o[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, sum = 0.f, top_w = -INFINITY;   // maxima in units of ln 2: of the scores, and of what the weights refer to
    const auto larger = [](float p, float q) { return fmaxf(p, q); };
    if (step < end) load(step);
    for (; step < end; ++step) {
        seen = seen_next;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the reads of the step before, whose place the next one takes, are over
        if (step + 1 < end) {
            load(step + 1);
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LOADS + CODES) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const lds_char *stage = mine + (step & 1) * STAGE;
        f32x4 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int r = h * 16 + col;
            if constexpr (CODES) {
#pragma unroll
                for (int i = 0; i < DP / 64; ++i) {
                    const u32x4 w = *reinterpret_cast<const __attribute__((address_space(3))) u32x4 *>(stage + r * RB + (((i * 4 + quad) ^ k_key<RB>(r)) << 4));
                    x[h] = MfmaTile<T, 16>::mma(decode8<T>(w[0], w[1]), q[2 * i], x[h]);
                    x[h] = MfmaTile<T, 16>::mma(decode8<T>(w[2], w[3]), q[2 * i + 1], x[h]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < DP / 32; ++i)
                    x[h] = MfmaTile<T, 16>::mma(*reinterpret_cast<const __attribute__((address_space(3))) v8 *>(stage + r * RB + (((i * 4 + quad) ^ k_key<RB>(r)) << 4)), q[i], x[h]);
            }
        }
        // Scores in units of ln 2, those of codes with their key's exponent; z[h]: with the value's too.
        f32x4 z[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (CODES) {
                const i32x4 ke = *reinterpret_cast<const __attribute__((address_space(3))) i32x4 *>(stage + 2 * PART + (h * 16 + quad * 4) * 4);
                const i32x4 ve = *reinterpret_cast<const __attribute__((address_space(3))) i32x4 *>(stage + 2 * PART + 128 + (h * 16 + quad * 4) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[h][e] = ldexpf(x[h][e] * f.c, ke[e] - 127);
                    z[h][e] = x[h][e] + (float)(ve[e] - 127);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[h][e] *= f.c;
            }
        }
        if (seen != 0xffffffffu) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(seen >> (h * 16 + quad * 4 + e) & 1)) {
                        x[h][e] = -INFINITY;
                        if constexpr (CODES) z[h][e] = -INFINITY;
                    }
        }
        const float most = of_four(fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3]))), larger);
        bool follow = most > top + kOneSlack || (top == -INFINITY && most > top);
        float most_w = most;
        if constexpr (CODES) {
            most_w = of_four(fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3]))), larger);
            follow |= most_w > top_w + kOneSlack || (top_w == -INFINITY && most_w > top_w);
        }
        if (__any(follow)) {
            const float now = fmaxf(top, most), by = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.f : now));
            top = now;
            sum *= by;
            float by_w = by;
            if constexpr (CODES) {
                const float now_w = fmaxf(top_w, most_w);
                by_w = __builtin_amdgcn_exp2f(top_w - (now_w == -INFINITY ? 0.f : now_w));
                top_w = now_w;
            }
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) o[i] *= by_w;
        }
        const float ref = top == -INFINITY ? 0.f : top, ref_w = top_w == -INFINITY ? 0.f : top_w;
        w8 w, rest;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(x[h][e] - ref);
                sum += p;
                const float by = CODES ? __builtin_amdgcn_exp2f(z[h][e] - ref_w) : p;
                if constexpr (TWO) {
                    // A part below the weight, and what is left, above 0 and at most 2^-7 of it: both times an infinite value are that.
                    const unsigned u = __builtin_bit_cast(unsigned, by), upper = ((u > 1u ? u : 1u) - 1u) & 0xffff0000u;
                    w[h * 4 + e] = __builtin_bit_cast(VT, (unsigned short)(upper >> 16));
                    rest[h * 4 + e] = (VT)(by - __builtin_bit_cast(float, upper));
                } else {
                    w[h * 4 + e] = (VT)by;
                }
            }
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            w8 v;
            if constexpr (CODES) {
                const int slot = col >> 1, r = (slot & 3) + quad * 4 + (slot >> 2) * 16;
                const i32x2 codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(stage + PART + r * RB + ((i ^ v_key<RB, true>(r)) << 4) + (col & 1) * 8));
                v = decode8<f16>(codes[0], codes[1]);
            } else {
                s16x4 t[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = h * 16 + quad * 4 + (col >> 2);
                    t[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4 *)(stage + PART + r * RB + (((i * 2 + (col >> 1 & 1)) ^ v_key<RB, false>(r)) << 4) + (col & 1) * 8));
                }
                v = __builtin_bit_cast(w8, __builtin_shufflevector(t[0], t[1], 0, 1, 2, 3, 4, 5, 6, 7));
            }
            o[i] = MfmaTile<VT, 16>::mma(v, w, o[i]);
            if constexpr (TWO) o[i] = MfmaTile<VT, 16>::mma(v, rest, o[i]);
        }
    }
    sum = of_four(sum, [](float p, float q) { return p + q; });

    // The waves meet in LDS, each in its own part of it.
    if constexpr (CODES) {
        const float by = __builtin_amdgcn_exp2f(top_w == -INFINITY ? 0.f : top_w - top);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) o[i] *= by;
    }
    if (quad == 0) {
        tops[wave][col] = top;
        sums[wave][col] = sum;
    }
    static_assert(kOneHeads * DP * 4 <= 2 * STAGE, "a wave's results fit where its tokens were");
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)   // [head][DP], chunks of 16 bytes exchanged by the head
        *reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(mine + col * (DP * 4) + (((i * 4 + quad) ^ (col & 7)) << 4)) = o[i];
    __syncthreads();

    const int chunks = c.head_dim / 4;     // of 16 bytes a head
    T *const y = static_cast<T *>(a.y) + s * a.y_stride;
    auto store = [&](int h, int d4, f32x4 v, float total) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        T4 r;
        const float by = 1.f / total;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (T)(total == 0.f ? 0.f : v[e] * by);
        *reinterpret_cast<T4 *>(y + (int64_t)(head0 + h) * a.y_head_stride + d4 * 4) = r;
    };
    auto store_lse = [&](int h, float m, float total) {
        if (a.lse) a.lse[(int64_t)s * a.heads + head0 + h] = total == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(total)) * 0.693147181f;
    };
    // Of head h: the waves' maximum and sum, and what each wave's results count.
    auto of_waves = [&](int h, float &m, float &total, float (&by)[WAVES]) {
        m = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w][h]);
        const float r = m == -INFINITY ? 0.f : m;
        total = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            by[w] = __builtin_amdgcn_exp2f(tops[w][h] - r);
            total += sums[w][h] * by[w];
        }
    };
    const int record = heads * (c.head_dim + 2);   // numbers: results, then a maximum and a sum for each head
    float *const records = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + kOneCounters * 4) + ((int64_t)item * f.parts) * (min(f.group, kOneHeads) * (c.head_dim + 2));
    for (int i = tid; i < heads * chunks; i += THREADS) {
        const int h = i / chunks, d4 = i - h * chunks;
        float m, total, by[WAVES];
        of_waves(h, m, total, by);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            v += by[w] * *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>((lds_char *)lds + w * 2 * STAGE + h * (DP * 4) + ((d4 ^ (h & 7)) << 4));
        if (parts == 1) {
            store(h, d4, v, total);
            if (d4 == 0) store_lse(h, m, total);
        } else {
            float *to = records + (int64_t)part * record;
            auto put = [&](int at, float p, float q) {
                const uint64_t two = (uint64_t)__builtin_bit_cast(unsigned, q) << 32 | __builtin_bit_cast(unsigned, p);
                __hip_atomic_store(reinterpret_cast<uint64_t *>(to + at), two, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            };
            put(h * c.head_dim + d4 * 4, v[0], v[1]);
            put(h * c.head_dim + d4 * 4 + 2, v[2], v[3]);
            if (d4 == 0) put(heads * c.head_dim + 2 * h, m, total);
        }
    }
    if (parts == 1) return;

    // Parts meet in memory: each stores past its XCD's own L2, then counts; the last one to come joins them in their order.  A store counts as outstanding until it is where loads of that
    // scope look, which is what makes the relaxed accesses enough, as in the answer over logits.
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __syncthreads();
    int *counter = static_cast<int *>(a.workspace) + item;
    if (tid == 0) last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    auto get = [&](int p, int at) {
        return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<uint64_t *>(records + (int64_t)p * record + at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    };
    for (int i = tid; i < heads * chunks; i += THREADS) {
        const int h = i / chunks, d4 = i - h * chunks;
        float m = -INFINITY, total = 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            const f32x2 ms = get(p, heads * c.head_dim + 2 * h), lo = get(p, h * c.head_dim + d4 * 4), hi = get(p, h * c.head_dim + d4 * 4 + 2);
            const float pm = ms[0], pt = ms[1];
            const f32x4 pv = {lo[0], lo[1], hi[0], hi[1]};
            const float now = fmaxf(m, pm), r = now == -INFINITY ? 0.f : now, bo = __builtin_amdgcn_exp2f(m - r), bn = __builtin_amdgcn_exp2f(pm - r);
            m = now;
            total = total * bo + pt * bn;
            v = v * bo + pv * bn;
        }
        store(h, d4, v, total);
        if (d4 == 0) store_lse(h, m, total);
    }
}

template <typename T, bool CODES, int RB>
hipError_t launch_attend_one_as(const AttendOneArgs &a, hipStream_t s) {
    constexpr int WAVES = one_waves(RB);
    AttendOneKernel f{a, a.heads / a.cache.kv_heads, 0, 1, fminf(fmaxf(fabsf(a.scale) * 1.44269504f, 1e-37f), 3e38f)};
    f.blocks = (f.group + kOneHeads - 1) / kOneHeads;
    const int64_t items = (int64_t)a.sequences * f.blocks * a.cache.kv_heads;
    // Parts: one round of workgroups where the items are few, several where they are many, so that long sequences do not end alone.
    const int64_t slots = 256 * (kOneTokens * RB * 2 * 2 * WAVES > 64 * 1024 ? 1 : 2);
    const int64_t steps = (((int64_t)a.table_pages << a.cache.page_shift) + kOneTokens - 1) / kOneTokens;
    if (items < 8 * slots && items <= kOneCounters) {
        int64_t parts = items <= slots ? slots / items : (8 * slots + items - 1) / items;
        parts = std::min({parts, (int64_t)kOneMostParts, steps / (2 * WAVES)});
        const int64_t record = (int64_t)std::min(f.group, kOneHeads) * (a.cache.head_dim + 2) * 4;
        if (a.workspace_bytes > kOneCounters * 4) parts = std::min(parts, (int64_t)((a.workspace_bytes - kOneCounters * 4) / (record * items)));
        else parts = 1;
        f.parts = (int)std::max<int64_t>(parts, 1);
    }
    if (items * f.parts > INT32_MAX) return hipErrorInvalidValue;
    attend_one_kernel<T, CODES, RB><<<dim3((unsigned)(items * f.parts)), 64 * WAVES, 0, s>>>(f);
    return hipGetLastError();
}

template <typename T, bool CODES>
hipError_t launch_attend_one_typed(const AttendOneArgs &a, hipStream_t s) {
    const int bytes = a.cache.head_dim * (CODES ? 1 : 2);
    if (a.cache.head_dim % 16 != 0 || a.cache.head_dim > kAttendMostDim) return hipErrorInvalidValue;
    if constexpr (CODES) {
        if (bytes <= 64) return launch_attend_one_as<T, CODES, 64>(a, s);
        if (bytes <= 128) return launch_attend_one_as<T, CODES, 128>(a, s);
        return launch_attend_one_as<T, CODES, 256>(a, s);
    } else {
        if (bytes <= 128) return launch_attend_one_as<T, CODES, 128>(a, s);
        if (bytes <= 256) return launch_attend_one_as<T, CODES, 256>(a, s);
        return launch_attend_one_as<T, CODES, 512>(a, s);
    }
}

}  // namespace cw
