// The attention kernel of packed prompts (cw_attend has the definition), a type of numbers to a source file.
#pragma once
#include <cmath>

#include "attend_common.h"
#include "lds_loads.h"

namespace cw {

// A workgroup takes up to 128 rows of one key head, a row being a query of one of the `each` heads that share it (query row / each): heads share the keys that a workgroup loads, and few
// queries of many heads fill it.  Its waves take 32 rows each and walk the keys that any of these sees, a tile at a time.  Both products are transposed,
// S^T = K Q^T and O^T = V^T P^T: in an accumulator of the matrix cores a lane has one row of the attention and 4 (lane / 32) + 8 j + 0..3 of the other side, so
// maxima and sums of the softmax are a lane's own but for one exchange, and the eight numbers that a lane holds of S^T are those that the second product wants of P^T once it
// takes its keys in that order.  K lies in LDS as it is, V too and is transposed by the reads of LDS that do that.
// The running maximum follows the scores only where one is more than kSlack above it, so that most tiles rescale nothing.  Weights go into the second product in the values' type, half a step
// of each, which leaves the result about a quarter further from the formula than its own rounding does: weights of two parts take half as many matrix instructions again and a third more time (8192 tokens of 32 heads over
// 8 of 128 fp16 564 us and 757, 16 prompts of 33 to 2048 bf16 267 and 338).  fp16 ends early, so its weights refer to kShift below the maximum: the largest is 2^11 to 2^15, and what the type cannot hold
// of a weight is at most 2^-36 of the largest, where it would be 2^-25 with the maximum itself.
// The matrix cores and the card's power bound it: 8192 tokens of 32 heads over 8 of 128 fp16, causal, in 530 to 565 us, 970 to 1040 TFLOP/s at 1.5 to 1.8 GHz, where a library's product of 8192^3 random numbers reaches 1365, with its
// right operand transposed 1600; short prompts what comes before and behind the tiles: 16 prompts of 33 to 2048 tokens, bf16, in 246 to 265 us, 725 to 780 TFLOP/s.  Heads beyond 192 numbers do not fit a wave's registers where tiles
// have masks: 132 bytes a lane lie in scratch, 76 where waves share rows, and nine prompts of three tokens, 16 heads of 256, take 11 us, of 64 numbers 4.7.  A third tile under way in LDS is no faster (9 prompts of 1737 to 2121, 40 heads over 5 of 80 352 us and 353, one of 2468 and one head 33 and 42), nor are
// three waves a SIMD, whose registers spill (44 and 78 us for 60 prompts of 99 to 167, 32 heads over 8 of 80).
// Where the rows do not fill the GPU, SPLIT waves share 32 of them and take parts of each tile: their results meet in LDS at the end.
constexpr int kAttendKeys = 64;   // of a tile: two of them and their successors fit a CU's LDS up to 128 numbers a head
template <typename T>
struct AttendWeights {   // in units of ln 2
    static constexpr float kSlack = std::is_same<T, f16>::value ? 4.f : 8.f, kShift = std::is_same<T, f16>::value ? 11.f : 0.f;
};

struct AttendKernel {
    AttendArgs a;
    FastDiv each, kv_heads;
    int32_t group;     // heads that share a key head
    int32_t tiles;     // workgroups of a key head
    float c;           // |scale| / ln 2, above 0
};

template <typename T, int DP, int SPLIT>
__global__ __launch_bounds__(64 * kAttendWaves, DP <= 128 ? 2 : 1) void attend_kernel(const AttendKernel f) {
    typedef typename Mfma<T>::v8 v8;
    typedef AttendWeights<T> Weights;
    typedef T T2 __attribute__((ext_vector_type(2)));
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) unsigned char lds_char;
    constexpr int ROWS = attend_rows(SPLIT), KEYS = kAttendKeys, BLOCKS = KEYS / (32 * SPLIT);   // BLOCKS of 32 keys of each tile are a wave's
    constexpr int PANELS = DP / 32, PANEL = KEYS * 64, PART = PANELS * PANEL, STAGE = 2 * PART;   // bytes; a panel: 32 numbers of every key, 64 bytes each
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
    const AttendArgs &a = f.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
    const int block = fast_div(blockIdx.x, f.kv_heads), kvh = blockIdx.x - block * a.kv_heads, tile_id = f.tiles - 1 - block;   // the last queries, which see the most keys, first

    // The tile's sequence.  Tile tile_of(s) is the first of sequence s: tiles are counted as if the sequences' rows were one behind the other, and one more a sequence.
    int s, q0, q1, k0, k1;
    auto clamped = [](int r, int most) { return r < 0 ? 0 : r > most ? most : r; };
    if (a.sequences < 64) {
        const int at = min(lane, a.sequences), mine = clamped(a.first[at], a.tokens), mine_k = clamped(a.first_k[at], a.keys);
        s = max(0, __popcll(__ballot(lane < a.sequences && mine * f.group / ROWS + lane <= tile_id)) - 1);
        q0 = __builtin_amdgcn_readlane(mine, s);
        q1 = __builtin_amdgcn_readlane(mine, s + 1);
        k0 = __builtin_amdgcn_readlane(mine_k, s);
        k1 = __builtin_amdgcn_readlane(mine_k, s + 1);
    } else {
        s = last_not_above(a.sequences, tile_id, [&](int i) { return (int64_t)(clamped(a.first[i], a.tokens) * f.group / ROWS + i); });
        q0 = clamped(a.first[s], a.tokens);
        q1 = clamped(a.first[s + 1], a.tokens);
        k0 = clamped(a.first_k[s], a.keys);
        k1 = clamped(a.first_k[s + 1], a.keys);
    }
    const int n = q1 - q0, m = max(0, k1 - k0), row0 = (tile_id - (q0 * f.group / ROWS + s)) * ROWS;
    if (n <= 0 || row0 < 0 || row0 >= n * f.group) return;
    const int rows = min(ROWS, n * f.group - row0), behind = m - n;
    auto query_of = [&](int r) { return (int)fast_div((unsigned)(row0 + min(r, rows - 1)), f.each); };   // of row r of the tile
    auto high_of = [&](int i) { return a.causal ? max(0, i + behind + 1) : m; };                         // keys [low, high) are what query i sees
    auto low_of = [&](int i) { return a.window > 0 ? max(0, i + behind + 1 - a.window) : 0; };
    const int row_group = wave % (kAttendWaves / SPLIT), key_group = wave / (kAttendWaves / SPLIT);
    const int my_row = row_group * 32 + l32, my_query = query_of(my_row), my_head = kvh * f.group + row0 + min(my_row, rows - 1) - my_query * f.group;
    const int my_low = low_of(my_query), my_high = high_of(my_query);
    const int wg_low = low_of(query_of(0)), wg_high = high_of(query_of(ROWS - 1));
    const int tiles = wg_high > wg_low ? (wg_high - wg_low + KEYS - 1) / KEYS : 0;
    // Of this wave: tiles [begin, end) hold keys that some row sees, [all_begin, all_end) of them only such that all rows see.
    const int first_query = query_of(row_group * 32), last_query = query_of(row_group * 32 + 31);
    const int begin = (low_of(first_query) - wg_low) / KEYS, end = (high_of(last_query) - wg_low + KEYS - 1) / KEYS;
    const int all_begin = (low_of(last_query) - wg_low + KEYS - 1) / KEYS, all_end = (high_of(first_query) - wg_low) / KEYS;

    // Q as the second operand; a negative scale is taken by its sign.
    const bool inside = my_row < rows;
    v8 q[DP / 16];
    {
        const T *from = static_cast<const T *>(a.q) + (int64_t)(q0 + my_query) * a.q_stride + (int64_t)my_head * a.q_head_stride + half * 8;
        const unsigned sign = a.scale < 0.f ? 0x80008000u : 0u;
        u32x4 w[DP / 16];
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) w[i] = *reinterpret_cast<const u32x4 *>(from + (i * 16 + half * 8 < a.head_dim ? i * 16 : -half * 8));
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) q[i] = __builtin_bit_cast(v8, i * 16 + half * 8 < a.head_dim ? w[i] ^ sign : u32x4{0u, 0u, 0u, 0u});
    }

    // Loads: a wave takes 16 rows of a panel at a time, a KB.  K's 16-byte chunks are exchanged within a panel's row by (row / 4) % 4, so that the 16 rows
    // that a read of an operand takes at once lie in different banks; four rows of V, 256 bytes, are read at once as they are.
    const unsigned lds_base = (unsigned)(size_t)(lds_char *)lds + wave * 1024;   // loads follow one another through the panels, a KB each
    static_assert(KEYS == 16 * kAttendWaves, "a wave loads the same rows of every panel");
    const int ld_row = wave * 16 + (lane >> 2), ld_chunk = lane & 3, key_chunk = ld_chunk ^ ((ld_row >> 2) & 3);
    const unsigned k_off = (unsigned)ld_row * (unsigned)(a.k_stride * 2) + key_chunk * 16, v_off = (unsigned)ld_row * (unsigned)(a.v_stride * 2) + ld_chunk * 16;
    const char *k_at = reinterpret_cast<const char *>(static_cast<const T *>(a.k) + (int64_t)(k0 + wg_low) * a.k_stride + kvh * a.k_head_stride);
    const char *v_at = reinterpret_cast<const char *>(static_cast<const T *>(a.v) + (int64_t)(k0 + wg_low) * a.v_stride + kvh * a.v_head_stride);
    auto load = [&](int t) {   // tiles one after the other
        const int left = min(KEYS, m - wg_low - t * KEYS);   // rows beyond the last key are out of the buffers: zeros
        const u32x4 dk = make_desc(k_at, ((unsigned)(left - 1) * (unsigned)a.k_stride + a.head_dim) * 2u);
        const u32x4 dv = make_desc(v_at, ((unsigned)(left - 1) * (unsigned)a.v_stride + a.head_dim) * 2u);
        k_at += (unsigned)a.k_stride * (KEYS * 2u);
        v_at += (unsigned)a.v_stride * (KEYS * 2u);
        const unsigned to = lds_base + (t & 1) * STAGE;
#pragma unroll
        for (int p = 0; p < PANELS; ++p) load_to_lds(dk, p * 32 + key_chunk * 8 < a.head_dim ? k_off : kOob, p * 64, to + p * PANEL);
#pragma unroll
        for (int p = 0; p < PANELS; ++p) load_to_lds(dv, p * 32 + ld_chunk * 8 < a.head_dim ? v_off : kOob, p * 64, to + PART + p * PANEL);
    };
    auto next = [&](int t) {
        wait_lds_loads_and_barrier<0>();   // tile t is there, and the reads of the one before, whose place the next one takes, are over
        if (t + 1 < tiles) load(t + 1);
    };

    f32x16 o[PANELS];
#pragma unroll
    for (int p = 0; p < PANELS; ++p)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[p][e] = 0.f;
    float top = -INFINITY, sum = 0.f;   // the maximum, in units of ln 2, and the sum of this lane's weights, which refer to kShift less
    const int key_swz = (l32 >> 2) & 3;
    const unsigned mine = key_group * BLOCKS * 2048;   // this wave's keys in a panel
    const unsigned k_read[2] = {mine + (unsigned)(l32 * 64 + ((half ^ key_swz) << 4)), mine + (unsigned)(l32 * 64 + (((2 + half) ^ key_swz) << 4))};
    const unsigned v_read = PART + mine + (4 * half + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;

    unsigned odd_left = 0, odd_right = 0;   // of the tiles with masks before and behind those without: 32 rows see at most two such on a side
    auto work = [&](int t, auto masked) {
        const lds_char *stage = (const lds_char *)lds + (t & 1) * STAGE;
        f32x16 x[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[b][e] = 0.f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
                x[b] = Mfma<T>::mma(*reinterpret_cast<const __attribute__((address_space(3))) v8 *>(stage + k_read[i & 1] + (i >> 1) * PANEL + b * 2048), q[i], x[b]);
        }
        if constexpr (decltype(masked)::value) {
            const int base = wg_low + t * KEYS + key_group * BLOCKS * 32;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                auto below = [&](int key) { return (unsigned)((1ull << min(max(key - base - b * 32, 0), 32)) - 1); };   // of the block's keys those below one, a bit each
                const unsigned seen = (below(my_high) & ~below(my_low)) >> (4 * half);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const unsigned all = __builtin_amdgcn_sbfe(seen, 8 * (e / 4) + e % 4, 1), bits = __builtin_bit_cast(unsigned, (float)x[b][e]);
                    x[b][e] = __builtin_bit_cast(float, (bits & all) | (0xff800000u & ~all));
                }
            }
        }
        float most = x[0][0];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, x[b][e]);
        {
            const unsigned u = __builtin_bit_cast(unsigned, most);
            const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            most = fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])) * f.c;
        }
        if (__any(most > top + Weights::kSlack || (top == -INFINITY && most > top))) {
            const float now = fmaxf(top, most), by = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.f : now));
            top = now;
            sum *= by;
#pragma unroll
            for (int p = 0; p < PANELS; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[p][e] *= by;
        }
        const float ref = top == -INFINITY ? 0.f : top - Weights::kShift;
        v8 w[2 * BLOCKS];   // P^T, sixteen keys each
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(x[b][e], f.c, -ref));
                sum += p;
                w[b * 2 + e / 8][e % 8] = (T)p;
            }
        auto values = [&](int i, int p) {   // keys 16 i + 4 half + 0..3 and 8 further of panel p, transposed
            const lds_char *at = stage + v_read + p * PANEL + i * 1024;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 512));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if constexpr (decltype(masked)::value) {
            // A value that is no number, times a weight of 0, is none either: 0 times all of them tells.  A tile that has some is left for later.
            float odd = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * BLOCKS; ++i)
#pragma unroll
                for (int p = 0; p < PANELS; ++p) {
                    const u32x4 v = __builtin_bit_cast(u32x4, values(i, p));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned two = v[e];   // not v[e] itself: of an element of a vector __builtin_bit_cast takes the first
                        if constexpr (std::is_same<T, f16>::value) odd = __builtin_amdgcn_fdot2(__builtin_bit_cast(T2, two), T2{0, 0}, odd, false);
                        else odd = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(T2, two), T2{0, 0}, odd, false);
                    }
                }
            asm volatile("" ::: "memory");   // the values are read again where they are needed: as many registers are not there
            if (__builtin_expect(__any(odd != 0.f), 0)) {
                if (t < all_begin) odd_left |= 1u << (t - begin);
                else odd_right |= 1u << (end - 1 - t);
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < 2 * BLOCKS; ++i)
#pragma unroll
            for (int p = 0; p < PANELS; ++p) o[p] = Mfma<T>::mma(__builtin_bit_cast(v8, values(i, p)), w[i], o[p]);
    };

    if (tiles > 0) load(0);
    // The loop over tiles without masks has no other in it: what shares registers with it over a branch costs copies of them in every tile.
    for (int t = 0; t < tiles;) {
        if (t >= all_begin && t < all_end) {
            do {
                next(t);
                if constexpr (DP > 128) {   // what the vector registers do not hold stays in the others over the loop
#pragma unroll
                    for (int p = 0; p < PANELS; ++p) asm volatile("" : "+a"(o[p]));
                }
                work(t, std::false_type{});
            } while (++t < all_end);
        } else {
            next(t);
            if (t >= begin && t < end) work(t, std::true_type{});
            ++t;
        }
    }

    // What was left: weights once more, from memory, and the values key by key, into the rows that see it only.
    for (int side = 0; side < 2; ++side) {
        for (unsigned odd = side ? odd_right : odd_left; odd; odd &= odd - 1) {
            const int at = __builtin_ctz(odd), t = side ? end - 1 - at : begin + at, base = wg_low + t * KEYS + key_group * BLOCKS * 32;
            f32x16 x[BLOCKS];
            v8 w[2 * BLOCKS];
            const float ref = top == -INFINITY ? 0.f : top - Weights::kShift;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const int key = base + b * 32 + l32;
                const T *from = static_cast<const T *>(a.k) + (int64_t)(k0 + min(key, m - 1)) * a.k_stride + kvh * a.k_head_stride + half * 8;
#pragma unroll
                for (int e = 0; e < 16; ++e) x[b][e] = 0.f;
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    u32x4 v = {0u, 0u, 0u, 0u};
                    if (i * 16 + half * 8 < a.head_dim) v = *reinterpret_cast<const u32x4 *>(from + i * 16);
                    x[b] = Mfma<T>::mma(__builtin_bit_cast(v8, v), q[i], x[b]);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int mine = base + 4 * half + b * 32 + 8 * (e / 4) + e % 4;
                    w[b * 2 + e / 8][e % 8] = (T)(mine < my_low || mine >= my_high ? 0.f : __builtin_amdgcn_exp2f(fmaf(x[b][e], f.c, -ref)));
                }
            }
            for (int j = 0; j < BLOCKS * 32 && base + j < m; ++j) {
                const int slot = (j & 3) + ((j >> 3) & 1) * 4;
                const bool seen = base + j >= my_low && base + j < my_high, here = ((j >> 2) & 1) == half;
                v8 weights = w[0];
#pragma unroll
                for (int i = 1; i < 2 * BLOCKS; ++i)
                    if (j >> 4 == i) weights = w[i];
                const T *from = static_cast<const T *>(a.v) + (int64_t)(k0 + base + j) * a.v_stride + kvh * a.v_head_stride + l32;
#pragma unroll
                for (int p = 0; p < PANELS; ++p) {
                    const T value = here && p * 32 + l32 < a.head_dim ? from[p * 32] : (T)0.f;
                    v8 v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = e == slot ? value : (T)0.f;
                    f32x16 one;
#pragma unroll
                    for (int e = 0; e < 16; ++e) one[e] = 0.f;
                    one = Mfma<T>::mma(v, weights, one);
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[p][e] += seen ? one[e] : 0.f;
                }
            }
        }
    }

    {
        const unsigned u = __builtin_bit_cast(unsigned, sum);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        sum = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    if constexpr (SPLIT > 1) {
        // The waves that share rows meet: all but the first group leave theirs in LDS, lane by lane.
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        constexpr int BOX = (PANELS * 4 * 16 + 8) * 64;
        static_assert((kAttendWaves - kAttendWaves / SPLIT) * BOX <= 2 * STAGE, "results fit where the tiles were");
        auto box = [&](int group, int at) { return (__attribute__((address_space(3))) f32x4 *)((lds_char *)lds + ((group - 1) * (kAttendWaves / SPLIT) + row_group) * BOX + (at * 64 + lane) * 16); };
        auto tail = [&](int group) { return (__attribute__((address_space(3))) float *)((lds_char *)lds + ((group - 1) * (kAttendWaves / SPLIT) + row_group) * BOX + PANELS * 4 * 1024 + lane * 8); };
        wait_lds_loads_and_barrier<0>();
        if (key_group > 0) {
#pragma unroll
            for (int p = 0; p < PANELS; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) *box(key_group, p * 4 + e) = f32x4{o[p][4 * e], o[p][4 * e + 1], o[p][4 * e + 2], o[p][4 * e + 3]};
            tail(key_group)[0] = top;
            tail(key_group)[1] = sum;
        }
        wait_lds_and_barrier();
        if (key_group > 0) return;
        for (int g = 1; g < SPLIT; ++g) {
            const float other = tail(g)[0], now = fmaxf(top, other), ref = now == -INFINITY ? 0.f : now;
            const float by = __builtin_amdgcn_exp2f(top - ref), by_other = __builtin_amdgcn_exp2f(other - ref);
            top = now;
            sum = sum * by + tail(g)[1] * by_other;
#pragma unroll
            for (int p = 0; p < PANELS; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 v = *box(g, p * 4 + e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[p][4 * e + i] = o[p][4 * e + i] * by + v[i] * by_other;
                }
        }
    }
    const bool empty = sum == 0.f;
    const float by = empty ? 0.f : 1.f / sum;
    if (!inside) return;
    if (a.lse && half == 0) a.lse[(int64_t)(q0 + my_query) * a.heads + my_head] = empty ? -INFINITY : (top - Weights::kShift + __builtin_amdgcn_logf(sum)) * 0.693147181f;
    T *to = static_cast<T *>(a.y) + (int64_t)(q0 + my_query) * a.y_stride + (int64_t)my_head * a.y_head_stride;
#pragma unroll
    for (int p = 0; p < PANELS; ++p)
#pragma unroll
        for (int g = 0; g < 2; ++g) {   // numbers 16 g + 0..15 of the panel, 16 bytes a half
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 lo, hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = (T)(empty ? 0.f : o[p][8 * g + e] * by);
                hi[e] = (T)(empty ? 0.f : o[p][8 * g + 4 + e] * by);
            }
            const u32x2 lo2 = __builtin_bit_cast(u32x2, lo), hi2 = __builtin_bit_cast(u32x2, hi);
            const auto first2 = __builtin_amdgcn_permlane32_swap(lo2[0], hi2[0], false, false);
            const auto second2 = __builtin_amdgcn_permlane32_swap(lo2[1], hi2[1], false, false);
            const int d = p * 32 + g * 16 + half * 8;
            if (d < a.head_dim) *reinterpret_cast<u32x4 *>(to + d) = u32x4{(unsigned)first2[0], (unsigned)second2[0], (unsigned)first2[1], (unsigned)second2[1]};
        }
}

template <typename T, int DP, int SPLIT>
hipError_t launch_attend_as(const AttendArgs &a, hipStream_t s) {
    const int group = a.heads / a.kv_heads, tiles = (int)((int64_t)a.tokens * group / attend_rows(SPLIT) + a.sequences);
    const AttendKernel f{a, make_fast_div((uint32_t)group), make_fast_div((uint32_t)a.kv_heads), group, tiles, fmaxf(fabsf(a.scale) * 1.44269504f, 0x1p-149f)};   // not 0: it is multiplied with the -inf of masks, too
    attend_kernel<T, DP, SPLIT><<<dim3((unsigned)tiles * a.kv_heads), dim3(64 * kAttendWaves), 0, s>>>(f);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_attend_dim(const AttendArgs &a, hipStream_t s) {
    // Waves share rows where there are few workgroups of 128 rows: 500 queries of 32 heads over 8 of 128 bf16 (133 workgroups) 15.0 -> 11.8 us, eight prompts of 290 to 680 behind 215 keys, 8 heads (306)
    // 33.2 -> 27.2; but four of 301 to 1024 behind 2500, 16 heads over 4 of 96 (347) 58 -> 65, 39 of 80 to 149, 8 heads over 4 (434) 13.5 -> 16.4.
    return attend_workgroups(a) <= 320 ? launch_attend_as<T, DP, 2>(a, s) : launch_attend_as<T, DP, 1>(a, s);
}

template <typename T>
hipError_t launch_attend_typed(const AttendArgs &a, hipStream_t s) {
    if (a.head_dim % 16 != 0 || a.head_dim > kAttendMostDim || !attend_fits(a)) return hipErrorInvalidValue;
    if (a.head_dim <= 64) return launch_attend_dim<T, 64>(a, s);
    if (a.head_dim <= 96) return launch_attend_dim<T, 96>(a, s);
    if (a.head_dim <= 128) return launch_attend_dim<T, 128>(a, s);
    if (a.head_dim <= 192) return launch_attend_dim<T, 192>(a, s);
    return launch_attend_dim<T, 256>(a, s);
}

}  // namespace cw
