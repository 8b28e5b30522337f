// The attention kernel of single tokens over a paged cache (cw_attend_one has the definition), a type of queries and of pages to a source file.
#pragma once
#include <cmath>

#include "attend_common.h"
#include "lds_loads.h"

namespace cw {

// Reading keys and values is what this costs: everything serves to keep enough of their bytes under way.  A workgroup takes up to 16 of the query heads that share a key head, and a part of a
// sequence's tokens; its waves walk shares of that by themselves, 32 tokens a step (16 of large rows), K and V of the next step on their way straight to the wave's own LDS while this one is worked on.
// Products are transposed, on 16 x 16 tiles of the matrix cores: S^T = K Q^T, whose lanes have a query and tokens 4 (lane / 16) + 0..3 of each half of the step, just what the second product,
// O^T = V^T P^T, wants of P^T with its tokens in that order; V is transposed by the reads of LDS that do that.  Tokens that are not seen come from a line of zeros.
// Codes of 8 bits become numbers of the queries' type for the first product and fp16 for the second, exactly; a key's exponent goes to its score, a value's to its weight before that is rounded:
// weights refer to a maximum of their own, which follows where one is 2^kSlack times above it.  bf16 weights go into the second product in two parts, 15 bits, which their loads hide; fp16 weights in one of 11 bits: a second
// one leaves an error that is a tenth less and costs a call 8 to 18 % where little is read (one sequence of 1000 tokens, 32 heads over 8 of 128 fp16, 8.4 us and 9.3, of 300 6.2 and 7.3), 200 of up to 4096 in e4m3 173 us and 177.
// fp16 ends early, so its weights refer to 2^11 below the maximum: what the type cannot hold of a weight is at most 2^-36 of the largest.
// 64 sequences of 133 to 8192 tokens, 32 heads over 8 of 128 bf16, take 196 to 204 us, 5.4 TB/s, where reading GiBs and nothing else reaches 7.1; 200 of up to 4096, 64 heads over 8 in e4m3, 164 to 176; one of 32001 31, 4.2 TB/s, of
// which about 12 go to the launch, the first bytes and the meeting.  More loads under way (four steps, smaller ones) gave nothing.
constexpr int kOneMostParts = 64;   // a lane each where they meet
constexpr int kOneCounters = 65536 / 4;

struct AttendOneKernel {
    AttendOneArgs a;
    int32_t group, blocks;   // query heads of a key head, blocks of kOneHeads of them
    int32_t items;           // of a sequence: key heads times blocks
    int32_t inner, parts_outer;   // of the grid: what follows within the other, items within parts or parts within items
    FastDiv by_inner, by_kv_heads, by_items, by_chunks;   // chunks: 16 bytes of a head's results in fp32
    int32_t parts, fewest, from;   // of a sequence at most; steps of a part at least; steps of a sequence that is worth parts
    float c;                 // |scale| / ln 2
    int32_t most;            // EVEN: parts of all sequences together
};

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

__device__ static inline float max3(float a, float b, float c) {   // as the instruction has it: a NaN loses
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The tokens of a sequence that are looked at, and the steps that they take.
struct OneRange {
    int from, len, step0, steps;
};
template <int TOKENS>
__device__ static inline OneRange one_range(const AttendOneArgs &a, int length) {
    const int full = max(length, 0), from = a.window > 0 ? max(0, full - a.window) : 0, len = min(full, a.table_pages << a.cache.page_shift), step0 = from / TOKENS;
    return {from, len, step0, len > from ? (len + TOKENS - 1) / TOKENS - step0 : 0};
}

// What a workgroup keeps in LDS.
template <bool CODES, int RB, int WAVES>
struct OneShared {
    static constexpr int TOKENS = one_tokens(RB), STAGES = 2, STAGE = 2 * TOKENS * RB + (CODES ? 256 : 0);
    __attribute__((aligned(1024))) unsigned char lds[STAGES * WAVES * STAGE];
    float tops[WAVES][kOneHeads], sums[WAVES][kOneHeads];
    int last;
};

// Part `part` of `parts` of the attention of sequence s and heads hh: this wave's steps of it are step..end - 1 of the range.  Part p leaves its record at first + p.
// T: queries; CODES: pages of e4m3, else of T.  RB: bytes of a row in LDS, at least those of a head.
template <typename T, bool CODES, int RB, int WAVES>
__device__ static __forceinline__ void attend_one_part(const AttendOneKernel &f, OneShared<CODES, RB, WAVES> &shared, int s, int hh, const OneRange range, int step, int end, int part, int parts, int first) {
    typedef typename std::conditional<CODES, f16, T>::type VT;    // of the second product
    typedef typename Mfma<T>::v8 v8;
    typedef typename Mfma<VT>::v8 w8;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) unsigned char lds_char;
    typedef OneShared<CODES, RB, WAVES> Shared;
    constexpr int THREADS = 64 * WAVES, SIZE = CODES ? 1 : 2, DP = RB / SIZE, TOKENS = Shared::TOKENS, HALVES = TOKENS / 16, STAGES = Shared::STAGES;
    constexpr int PART = TOKENS * RB, STAGE = Shared::STAGE, LOADS = PART / 1024;
    constexpr unsigned ALL = TOKENS == 32 ? 0xffffffffu : (1u << TOKENS) - 1u;
    static_assert(!CODES || TOKENS == 32, "codes' exponents: a lane each of keys and of values");
    constexpr bool TWO = std::is_same<VT, bf16>::value;
    constexpr float kSlack = TWO ? 8.f : 4.f, kShift = TWO ? 0.f : 11.f;   // in units of ln 2
    auto &lds = shared.lds;
    auto &tops = shared.tops;
    auto &sums = shared.sums;
    const AttendOneArgs &a = f.a;
    const CacheView &c = a.cache;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
    const int block = fast_div(hh, f.by_kv_heads), kvh = hh - block * c.kv_heads;
    const int heads = min(kOneHeads, f.group - block * kOneHeads), head0 = kvh * f.group + block * kOneHeads;
    const int from = range.from, len = range.len;
    const bool whole = WAVES == 1 || parts == 1;   // a single wave has all of a sequence

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

    lds_char *const mine = (lds_char *)lds + wave * STAGES * STAGE;
    const unsigned mine_at = (unsigned)(size_t)mine;
    const int32_t *table = a.table + s * a.table_stride;
    const char *k_head = static_cast<const char *>(c.k) + kvh * c.head_stride * SIZE, *v_head = static_cast<const char *>(c.v) + kvh * c.head_stride * SIZE;
    int table_base = 0, entries = -1;    // a lane's page of the sequence's pages table_base..table_base + 63
    bool have_table = false;
    constexpr int LOAD_ROWS = 1024 / RB;    // that a load covers
    const bool regular = c.head_dim * SIZE == RB && c.page_shift >= 4 && c.token_stride <= (1 << 24);   // 16 rows lie in a page
    unsigned k_off[LOADS], v_off[LOADS];    // of this lane's 16 bytes behind the first row of the 16 that its load is among
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int r = (j * 64 + lane) * 16 / RB, pos = lane & (RB / 16 - 1);
        const unsigned row = (unsigned)(r & 15) * (unsigned)c.token_stride * SIZE;
        k_off[j] = row + (pos ^ k_key<RB>(r)) * 16;
        v_off[j] = row + (pos ^ v_key<RB, CODES>(r)) * 16;
    }
    // Loads the tokens of a step, tells which of them are seen.
    auto load = [&](int st, int place) {
        const int t0 = st * TOKENS, token = t0 + (lane & (TOKENS - 1));
        if (!have_table || ((t0 + TOKENS - 1) >> c.page_shift) - table_base >= 64) {
            have_table = true;
            table_base = t0 >> c.page_shift;
            const int at = table_base + lane;
            const int page = at < a.table_pages ? table[at] : -1;
            entries = (unsigned)page < (unsigned)c.pages ? page : -1;
        }
        const int in = token & ((1 << c.page_shift) - 1), page = __shfl(entries, (token >> c.page_shift) - table_base);
        const bool ok = page >= 0 && token >= from && token < len;
        const unsigned bits = (unsigned)__ballot(ok) & ALL, to = mine_at + place * STAGE;
        if (bits == ALL && regular) {
            // One address for all lanes.
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const int t = t0 + h * 16, first = __builtin_amdgcn_readlane(page, h * 16);
                const int64_t at = ((int64_t)(unsigned)first * c.page_stride + (t & ((1 << c.page_shift) - 1)) * c.token_stride) * SIZE;
#pragma unroll
                for (int j = h * LOADS / HALVES; j < (h + 1) * LOADS / HALVES; ++j) {
                    load_to_lds(k_head + at, k_off[j], to + j * 1024);
                    load_to_lds(v_head + at, v_off[j], to + PART + j * 1024);
                }
            }
        } else {
            const int64_t row = ok ? (page * c.page_stride + in * c.token_stride) * SIZE : -1;
            const int row_lo = (int)row, row_hi = (int)(row >> 32);
            int64_t at[LOADS];
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int r = (j * 64 + lane) * 16 / RB;
                at[j] = (int64_t)__shfl(row_hi, r) << 32 | (unsigned)__shfl(row_lo, r);
            }
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int r = (j * 64 + lane) * 16 / RB, pos = lane & (RB / 16 - 1), kc = pos ^ k_key<RB>(r), vc = pos ^ v_key<RB, CODES>(r);
                const char *zero = reinterpret_cast<const char *>(one_zeros);
                load_to_lds(at[j] >= 0 && kc * 16 < c.head_dim * SIZE ? k_head + at[j] + kc * 16 : zero, to + j * 1024);
                load_to_lds(at[j] >= 0 && vc * 16 < c.head_dim * SIZE ? v_head + at[j] + vc * 16 : zero, to + PART + j * 1024);
            }
        }
        if constexpr (CODES) {
            const char *e = reinterpret_cast<const char *>(lane < 32 ? c.k_exp : c.v_exp) + page * c.exp_page_stride + kvh * c.exp_head_stride + in * c.exp_token_stride;
            load_byte_to_lds(ok ? e : reinterpret_cast<const char *>(one_zeros), to + 2 * PART);
        }
        return bits;
    };

    f32x4 o[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, sum = 0.f, top_w = -INFINITY;   // maxima in units of ln 2: of the scores, and with codes of the scores with their values' exponents
    const auto larger = [](float p, float q) { return max3(p, q, q); };
    unsigned seen_next = step < end ? load(step, step & 1) : 0u;    // of the next step's tokens, a bit each
    for (; step < end; ++step) {
        const unsigned seen = seen_next;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the reads of the step before, whose place the next one takes, are over
        if (step + 1 < end) {
            seen_next = load(step + 1, (step + 1) & 1);
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LOADS + CODES) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const lds_char *stage = mine + (step & 1) * STAGE;
        f32x4 x[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
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
        f32x4 z[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
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
        if (__builtin_expect(seen != ALL, 0)) {
            asm volatile("");   // a branch: few steps take it
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(seen >> (h * 16 + quad * 4 + e) & 1)) {
                        x[h][e] = -INFINITY;
                        if constexpr (CODES) z[h][e] = -INFINITY;
                    }
        }
        auto most_of = [&](const f32x4 (&v)[HALVES]) {
            float m = max3(v[0][0], v[0][1], v[0][2]);
            if constexpr (HALVES == 2) m = max3(max3(m, v[0][3], v[1][0]), max3(v[1][1], v[1][2], v[1][3]), m);
            else m = max3(m, v[0][3], m);
            return of_four(m, larger);
        };
        const float most = most_of(x);
        bool follow = most > top + kSlack || (top == -INFINITY && most > top);
        float most_w = most;
        if constexpr (CODES) {
            most_w = most_of(z);
            follow |= most_w > top_w + kSlack || (top_w == -INFINITY && most_w > top_w);
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
        const float ref = top == -INFINITY ? 0.f : top - (CODES ? 0.f : kShift), ref_w = top_w == -INFINITY ? 0.f : top_w - kShift;
        w8 w = {}, rest = {};
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
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
                s16x4 t[2] = {};
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
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

    // Results and their sum, both relative to `top`.
    if constexpr (CODES) {
        // In two steps: the power may lie beyond fp32's where the result does not, and the instruction gives 0 below 2^-126.
        const float by = __builtin_amdgcn_exp2f(top_w == -INFINITY ? 0.f : (top_w - kShift - top) * 0.5f);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) o[i] = o[i] * by * by;
    } else {
        top -= kShift;
    }

    // The waves meet in LDS, each in its own part of it.
    if (quad == 0) {
        tops[wave][col] = top;
        sums[wave][col] = sum;
    }
    static_assert(kOneHeads * DP * 4 <= STAGES * STAGE, "a wave's results fit where its tokens were");
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
    const int items = heads * chunks;
    // A part's record: results, then a maximum and a sum for each head.
    auto record_of = [&](int p) {
        return reinterpret_cast<float *>(static_cast<char *>(a.workspace) + kOneCounters * 4) + (int64_t)(first + p) * (min(f.group, kOneHeads) * (c.head_dim + 2));
    };
    for (int i = tid; i < items; i += THREADS) {
        const int h = fast_div(i, f.by_chunks), d4 = i - h * chunks;
        float m, total, by[WAVES];
        of_waves(h, m, total, by);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            v += by[w] * *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>((lds_char *)lds + w * STAGES * STAGE + h * (DP * 4) + ((d4 ^ (h & 7)) << 4));
        if (whole) {
            store(h, d4, v, total);
            if (d4 == 0) store_lse(h, m, total);
        } else {
            float *to = record_of(part);
            auto put = [&](int at, float p, float q) {
                const uint64_t two = (uint64_t)__builtin_bit_cast(unsigned, q) << 32 | __builtin_bit_cast(unsigned, p);
                __hip_atomic_store(reinterpret_cast<uint64_t *>(to + at), two, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            };
            put(h * c.head_dim + d4 * 4, v[0], v[1]);
            put(h * c.head_dim + d4 * 4 + 2, v[2], v[3]);
            if (d4 == 0) put(heads * c.head_dim + 2 * h, m, total);
        }
    }
    if (whole) return;

    // Parts meet in memory: each stores past its XCD's own L2, then counts; the last one to come joins them in their order.  A store counts as outstanding until it is where loads of that
    // scope look, which is what makes the relaxed accesses enough, as in the answer over logits.
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __syncthreads();
    int *counter = static_cast<int *>(a.workspace) + s * (f.blocks * c.kv_heads) + hh;
    if (tid == 0) shared.last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!shared.last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    auto get = [&](int p, int at) {
        return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<uint64_t *>(record_of(p) + at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    };
    // A trip to memory takes longer than all the arithmetic: where a head's results are fewer than the threads, groups of these take every so manieth part, and the first
    // four of each thread are under way while the parts' weights are made, a lane a part.  Eight at a time load more than there is where the parts are few, past the L2 and so slowly, and their code is longer: one sequence of 1000,
    // 32 heads over 8 of 128, 8.6 us for 8.2, 25 of 100 to 4000 25.7 for 25.1; but one of 65000, 64 heads over 4 in e4m3 (64 parts), 33.3 for 37.5.
    constexpr int BATCH = 4;
    const int groups = items < THREADS ? (int)((THREADS + 0.5f) * __builtin_amdgcn_rcpf((float)items)) : 1;
    const int g = groups > 1 ? (int)((tid + 0.5f) * __builtin_amdgcn_rcpf((float)items)) : 0, i0 = tid - g * items * (groups > 1);
    f32x2 lo[BATCH], hi[BATCH];
    auto fetch = [&](int i, int from) {
        const int h = fast_div(i, f.by_chunks), at = h * c.head_dim + (i - h * chunks) * 4;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const int p = min(from + j * groups, parts - 1);
            lo[j] = get(p, at);
            hi[j] = get(p, at + 2);
        }
    };
    const bool some = i0 < items && g < groups;
    if (some) fetch(i0, g);
    typedef __attribute__((address_space(3))) float lds_float;
    lds_float *const weights = (lds_float *)(lds_char *)lds;           // [head][kOneMostParts]
    lds_float *const heads_of = weights + kOneHeads * kOneMostParts;   // a maximum and a sum for each head
    static_assert((kOneHeads * kOneMostParts + 2 * kOneHeads + 4 * THREADS) * 4 <= STAGES * WAVES * STAGE, "weights and sums fit where the tokens were");
#pragma unroll 4
    for (int h = wave; h < heads; h += WAVES) {
        const f32x2 ms = get(min(lane, parts - 1), heads * c.head_dim + 2 * h);
        float m = lane < parts ? ms[0] : -INFINITY;
        const float mine_m = m;
#pragma unroll
        for (int j = 1; j < 64; j *= 2) m = fmaxf(m, __shfl_xor(m, j));
        const float w = __builtin_amdgcn_exp2f(mine_m - (m == -INFINITY ? 0.f : m));
        float total = lane < parts ? ms[1] * w : 0.f;
#pragma unroll
        for (int j = 1; j < 64; j *= 2) total += __shfl_xor(total, j);
        weights[h * kOneMostParts + lane] = w;
        if (lane == 0) {
            heads_of[2 * h] = m;
            heads_of[2 * h + 1] = total;
        }
    }
    __syncthreads();
    for (int i = i0; i < items; i += THREADS) {
        if (!some) break;
        const int h = fast_div(i, f.by_chunks), d4 = i - h * chunks;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int from = g; from < parts; from += BATCH * groups) {
            if (i != i0 || from != g) fetch(i, from);
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int p = from + j * groups;
                if (p < parts) v += weights[h * kOneMostParts + p] * f32x4{lo[j][0], lo[j][1], hi[j][0], hi[j][1]};   // 0 times what is no number is none, as within a part
            }
        }
        if (groups > 1) {
            *reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(heads_of + 2 * kOneHeads + 4 * tid) = v;
            break;
        }
        store(h, d4, v, heads_of[2 * h + 1]);
        if (d4 == 0) store_lse(h, heads_of[2 * h], heads_of[2 * h + 1]);
    }
    if (groups == 1) return;
    __syncthreads();
    if (tid >= items) return;
    const int h = fast_div(tid, f.by_chunks), d4 = tid - h * chunks;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < groups; ++j) v += *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(heads_of + 2 * kOneHeads + 4 * (j * items + tid));
    store(h, d4, v, heads_of[2 * h + 1]);
    if (d4 == 0) store_lse(h, heads_of[2 * h], heads_of[2 * h + 1]);
}

constexpr int one_waves(bool codes, int rb) { return rb / (codes ? 1 : 2) <= 128 ? 2 : 1; }   // of a SIMD, at least

// A grid of parts of items, items being sequences and their heads.  EVEN: parts of up to 64 sequences, of the same steps whatever these have; a kernel of its own, as small calls feel the code that they skip (0.1 us of 4.6).
template <typename T, bool CODES, int RB, int WAVES, bool EVEN>
__global__ __launch_bounds__(64 * WAVES, one_waves(CODES, RB)) void attend_one_kernel(const AttendOneKernel f) {
    __shared__ OneShared<CODES, RB, WAVES> shared;
    int s, hh, part, parts, first;
    OneRange range;
    if constexpr (EVEN) {
        // The steps of a part are the fewest with which all parts run at once, found by halving: a lane a sequence.
        const int lane = threadIdx.x & 63, outer = fast_div(blockIdx.x, f.by_items);
        const int mine = lane < f.a.sequences ? one_range<one_tokens(RB)>(f.a, f.a.lengths[lane]).steps : 0;
        auto reduce = [&](int v, auto op) {
            auto dpp = [](int x, auto control, auto mask) { return __builtin_amdgcn_update_dpp(0, x, decltype(control)::value, decltype(mask)::value, 0xf, false); };
            v = op(v, dpp(v, std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{}));
            v = op(v, dpp(v, std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{}));
            v = op(v, dpp(v, std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{}));
            v = op(v, dpp(v, std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{}));
            v = op(v, dpp(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}));
            return op(v, dpp(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}));   // lane i: of lanes 0..i where op is a sum
        };
        auto sum = [](int p, int q) { return p + q; };
        auto parts_of = [&](int steps) { return lane >= f.a.sequences ? 0 : mine < f.from ? 1 : min(kOneMostParts, (int)ceilf((float)mine / (float)steps)); };   // rounded, the quotient is not above the next whole number
        const int longest = __builtin_amdgcn_readlane(reduce(mine, [](int p, int q) { return max(p, q); }), 63);
        int low = f.fewest - 1, high = max(longest, f.fewest);   // too few, and enough
        for (int i = 0; i < 8 && high - low > 1; ++i) {
            const int mid = i == 0 ? low + 1 : low + (high - low) / 2;
            if (__builtin_amdgcn_readlane(reduce(parts_of(mid), sum), 63) <= f.most) high = mid;
            else low = mid;
        }
        const int of_lane = parts_of(high), up = reduce(of_lane, sum);
        const uint64_t here = __ballot(up - of_lane <= outer && outer < up);
        if (!here) return;
        s = __builtin_ctzll(here);
        parts = __builtin_amdgcn_readlane(of_lane, s);
        const int base = __builtin_amdgcn_readlane(up, s) - parts;
        hh = blockIdx.x - outer * f.items;
        part = outer - base;
        first = base * f.items + hh * parts;
        range = one_range<one_tokens(RB)>(f.a, f.a.lengths[s]);
    } else {
        const int outer = fast_div(blockIdx.x, f.by_inner), inner = blockIdx.x - outer * f.inner, item = f.parts_outer ? inner : outer;
        part = f.parts_outer ? outer : inner;
        s = fast_div(item, f.by_items);
        hh = item - s * f.items;
        first = item * f.parts;
        range = one_range<one_tokens(RB)>(f.a, f.a.lengths[s]);
        parts = WAVES == 1 || range.steps < f.from ? 1 : max(1, min(f.parts, range.steps / f.fewest));
        if (part >= parts) return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int each = (int)((unsigned)(range.steps + parts * WAVES - 1) / (unsigned)(parts * WAVES));   // steps of a wave
    const int step = range.step0 + (part * WAVES + wave) * each;
    attend_one_part<T, CODES, RB, WAVES>(f, shared, s, hh, range, step, min(step + each, range.step0 + range.steps), part, parts, first);
}

inline AttendOneKernel one_kernel(const AttendOneArgs &a, int64_t parts, int fewest, int from, bool parts_outer) {
    AttendOneKernel f{};
    f.a = a;
    f.group = a.heads / a.cache.kv_heads;
    f.blocks = (f.group + kOneHeads - 1) / kOneHeads;
    f.items = f.blocks * a.cache.kv_heads;
    f.parts = (int)std::max<int64_t>(parts, 1);
    f.fewest = fewest;
    f.from = from;
    f.parts_outer = parts_outer;
    f.inner = parts_outer ? (int)std::min<int64_t>((int64_t)a.sequences * f.items, INT32_MAX) : f.parts;   // more items are refused
    f.by_inner = make_fast_div((uint32_t)f.inner);
    f.by_kv_heads = make_fast_div((uint32_t)a.cache.kv_heads);
    f.by_items = make_fast_div((uint32_t)f.items);
    f.by_chunks = make_fast_div((uint32_t)a.cache.head_dim / 4);
    f.c = fabsf(a.scale) * 1.44269504f;
    return f;
}

// Records that the workspace has room for; of more than attend_one_workspace_bytes() no use is made.  Two parts of up to 2047 items of 16 heads of 128 and more would take more, and gain nothing: 254 sequences of 4096, 128 heads
// over 8 of 128 in e4m3, 409 us whole and 444 in two, of 1 to 8192 454 and 459.
inline int64_t one_records(const AttendOneArgs &a, int64_t items) {
    const size_t bytes = std::min(a.workspace_bytes, attend_one_workspace_bytes());
    if (items > kOneCounters || bytes <= kOneCounters * 4) return 0;
    return (int64_t)(bytes - kOneCounters * 4) / ((int64_t)std::min(a.heads / a.cache.kv_heads, kOneHeads) * (a.cache.head_dim + 2) * 4);
}

template <typename T, bool CODES, int RB, int WAVES>
hipError_t launch_attend_one_as(const AttendOneArgs &a, int64_t items, int64_t steps, int64_t parts, int fewest, int from, bool parts_outer, hipStream_t s) {
    parts = steps < from ? 1 : std::min({parts, (int64_t)kOneMostParts, steps / fewest, one_records(a, items) / items});
    const AttendOneKernel f = one_kernel(a, parts, fewest, from, parts_outer);
    if (items * f.parts * 64 * WAVES > kMostThreads) return hipErrorInvalidValue;
    attend_one_kernel<T, CODES, RB, WAVES, false><<<dim3((unsigned)(items * f.parts)), 64 * WAVES, 0, s>>>(f);
    return hipGetLastError();
}

template <typename T, bool CODES, int RB>
hipError_t launch_attend_one_row(const AttendOneArgs &a, const OneForm &form, hipStream_t s) {
    constexpr int TOKENS = one_tokens(RB), WAVES = kOneWaves;
    const int64_t items = form.items, steps = form.steps, slots = form.slots;
    // Up to as many items as workgroups run at once: parts fill them, of 256 tokens at least (4 sequences of 810 to 1999, 4 heads of 80 bf16 11.4 us, of 512 tokens 15.0; but
    // 2 of 1486 and 5604, 64 heads over 4 in e4m3, 17.3 and 16.8), of sequences from 704 on (one of 600, 32 heads over 8 of 128 fp16, 8.3 us whole, 9.6 in two; one of 1000 11.6 whole, 8.2 in three), an item's behind one another: neighbours go to different XCDs (9 of 100 to 9000, 16 heads of 64 40.5 us, with all items' parts p behind one another 45.2).
    // Parts of the same steps whatever the lengths, no more than run at once, an item's neighbours those of the other heads: 6 of 9661 to 38277, 64 heads over 8 of 256 bf16, 218 us, as many parts of every sequence 240;
    // 5 of 100 to 20000, 32 heads over 8 of 128 42.7 and 50.5, 12 of 30 to 5000 29.7 and 36.2; 14 of 3726 to 4520, 80 over 5 of 256, 73.5 and 71.3. Where a record is large a part is too: 7 of 2441 to 6183, 32 heads over 2 of 128,
    // 23.8 us with parts of 256 tokens, 18.9 of 512.
    if (items <= slots && a.sequences > 1 && a.sequences <= 64 && form.tokens >= 704) {
        const int64_t grid = std::max(items, std::min(slots, one_records(a, items)));
        AttendOneKernel f = one_kernel(a, 1, (std::min(a.heads / a.cache.kv_heads, kOneHeads) * a.cache.head_dim > 1024 ? 512 : 256) / TOKENS, 704 / TOKENS, false);
        f.most = (int)(grid / f.items);
        attend_one_kernel<T, CODES, RB, WAVES, true><<<dim3((unsigned)grid), 64 * WAVES, 0, s>>>(f);
        return hipGetLastError();
    }
    if (items <= slots) return launch_attend_one_as<T, CODES, RB, WAVES>(a, items, steps, slots / items, 256 / TOKENS, 704 / TOKENS, false, s);
    if (form.wave_each) return launch_attend_one_as<T, CODES, RB, 1>(a, items, steps, 1, 1, 0, true, s);
    // Of more items, what a workgroup spends before its tokens, behind them and on meeting others is made up for by long parts only: 200 of up to 4096 in e4m3, 8 heads, 175 us, in parts of 256 tokens 187; 36 of up to 16000 219, whole
    // 239.  All items' first parts come first: of two parts behind one another the second is empty for all but the longest, which leaves every other XCD without work (64 of up to 8192 284 us for 228).
    return launch_attend_one_as<T, CODES, RB, WAVES>(a, items, steps, (4 * slots + items - 1) / items, 2048 / TOKENS, 0, true, s);
}

template <typename T, bool CODES>
hipError_t launch_attend_one_typed(const AttendOneArgs &a, hipStream_t s) {
    const OneForm form = one_form(a);
    if (a.cache.head_dim % 16 != 0 || a.cache.head_dim > kAttendMostDim) return hipErrorInvalidValue;
    if constexpr (CODES) {
        if (form.row_bytes == 64) return launch_attend_one_row<T, CODES, 64>(a, form, s);
        if (form.row_bytes == 128) return launch_attend_one_row<T, CODES, 128>(a, form, s);
        return launch_attend_one_row<T, CODES, 256>(a, form, s);
    } else {
        if (form.row_bytes == 128) return launch_attend_one_row<T, CODES, 128>(a, form, s);
        if (form.row_bytes == 256) return launch_attend_one_row<T, CODES, 256>(a, form, s);
        return launch_attend_one_row<T, CODES, 512>(a, form, s);
    }
}

}  // namespace cw
