// The answer of a row of logits: log probability and rank of a given class, entropy, the likeliest classes (cw_answer has the definitions).
#include <cfloat>
#include <cmath>

#include "conv_common.h"

namespace cw {

// One pass.  A workgroup takes a row, or a run of its segments, 32 logits a thread at a time in registers, 16 bytes a load.  Every thread keeps a
// maximum m, S = sum 2^d and T = sum d 2^d with d = (x - m) scale / ln 2 of its own (a new maximum rescales both once a segment), the
// threads meet at the end.  A segment's 32 terms are added in fp32, segment to segment in fp64: one by one in fp32 equal terms round alike (error of S, one workgroup a
// row: 6.5e-6 of it at 2^17 classes, 8.7e-4 at 2^24).  For the top classes a segment gives those of its logits that can still be among them to a list in LDS.
constexpr int kEach = 32, kThreads = 256, kFewest = 64, kRowsOfAWave = 512;
constexpr int kSegment = kThreads * kEach;
constexpr int kParts = 32;                         // workgroups a row at most
constexpr int kRecords = 1024;                     // of rows that are shared
constexpr int kRecordBytes = 16 + 8 * kAnswerMostTop;
constexpr int kCounterSlots = 256;                 // rows that can be shared
// Logits above the k-th largest of the threads' maxima lie with fewer than k threads; those equal to it are taken eight a thread at a time.
constexpr int list_keys(int threads) { return kAnswerMostTop + (kAnswerMostTop - 1) * kEach + kAnswerMostTop + threads * 8; }
constexpr int few_threads(int threads) { return (list_keys(threads) - kAnswerMostTop) / kEach; }   // whose logits the list holds, all of them
constexpr int kPad = 8;   // keys that first_of reads at a time

template <typename T>
struct Vec { static constexpr int N = 16 / sizeof(T); };

// Of all 64 lanes, in all of them.
template <typename V, typename F>
__device__ static inline V wave_all(V v, F f) {
    static_assert(sizeof(V) == 4, "a register");
    auto dpp = [](V x, auto control) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(control)::value, 0xf, 0xf, false));
    };
    v = f(v, dpp(v, std::integral_constant<int, 0xB1>{}));    // lanes 1 0 3 2
    v = f(v, dpp(v, std::integral_constant<int, 0x4E>{}));    // lanes 2 3 0 1
    v = f(v, dpp(v, std::integral_constant<int, 0x141>{}));   // mirrored in 8
    v = f(v, dpp(v, std::integral_constant<int, 0x140>{}));   // mirrored in 16
    const unsigned u = __builtin_bit_cast(unsigned, v);
    auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = f(__builtin_bit_cast(V, (unsigned)r[0]), __builtin_bit_cast(V, (unsigned)r[1]));
    const unsigned w = __builtin_bit_cast(unsigned, v);
    r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return f(__builtin_bit_cast(V, (unsigned)r[0]), __builtin_bit_cast(V, (unsigned)r[1]));
}

// Larger numbers for larger floats (the zeros are equal).
__device__ static inline unsigned order_of(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x + 0.f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ static inline float of_order(unsigned o) { return __builtin_bit_cast(float, o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }
// Larger for what comes first: the larger logit, of equal ones the lower class.
__device__ static inline uint64_t key_of(float x, int i) { return (uint64_t)order_of(x) << 32 | (unsigned)~i; }

// m, S and T of two sets of logits.
struct Soft { float m, s, t; };
__device__ static inline Soft join(const Soft &a, const Soft &b, float c2) {
    const float m = fmaxf(a.m, b.m), base = m == -INFINITY ? 0.f : m;
    const float da = fmaxf((a.m - base) * c2, -1e30f), db = fmaxf((b.m - base) * c2, -1e30f);   // -inf times 0 is no number
    const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
    return {m, a.s * ea + b.s * eb, (a.t + a.s * da) * ea + (b.t + b.s * db) * eb};
}

// 2^d for d <= 0, near 1 with the bits of what it is less: a row that rises slowly rescales its sums in every segment.  The series' next term is 2^-21 of its sum at -1/2.
__device__ static inline double fall(float d) {
    const float y = d * 0.693147181f;
    const float less = y * fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 720, 1.f / 120), 1.f / 24), 1.f / 6), 0.5f), 1.f);
    return d > -0.5f ? 1.0 + (double)less : (double)__builtin_amdgcn_exp2f(d);
}

// Of all 64 lanes.
__device__ static inline Soft meet(const Soft &v, float c2) {
    const auto plus = [](float p, float q) { return p + q; };
    const float m = wave_all(v.m, [](float p, float q) { return fmaxf(p, q); }), ref = m == -INFINITY ? 0.f : m;
    const float d = fmaxf((v.m - ref) * c2, -1e30f), e = __builtin_amdgcn_exp2f(d);
    return {m, wave_all(v.s * e, plus), wave_all((v.t + v.s * d) * e, plus)};
}

template <int THREADS>
struct AnswerLds {
    static constexpr int WAVES = THREADS / 64, KEYS = THREADS == kFewest ? kFewest * kEach : list_keys(THREADS);   // of a wave's only segment no more can be listed
    __attribute__((aligned(16))) uint64_t list[KEYS + kPad];
    uint64_t best[kAnswerMostTop];
    unsigned order[2][THREADS];
    float m[WAVES], s[WAVES], t[WAVES];
    int rank[WAVES];
    int n, last;
};

// The k first of list[0..n) in order; returns how many there are.  All threads, behind a barrier behind the last write.
template <int THREADS>
__device__ static inline int first_of(AnswerLds<THREADS> &l, int n, int k) {
    const int t = threadIdx.x;
    if (t < kPad) l.list[n + t] = 0;
    __syncthreads();
    for (int at = t; at < n; at += THREADS) {
        const uint64_t mine = l.list[at];
        int rank = 0;
        for (int o = 0; o < n; o += kPad) {
            uint64_t other[kPad];
#pragma unroll
            for (int i = 0; i < kPad; ++i) other[i] = l.list[o + i];
#pragma unroll
            for (int i = 0; i < kPad; ++i) rank += other[i] > mine;
        }
        if (rank < k) l.best[rank] = mine;
    }
    __syncthreads();
    const int have = n < k ? n : k;
    if (t < have) l.list[t] = l.best[t];
    return have;
}

// A number that at least k of the threads' orders reach, or `low` where fewer are above it; `many`: how many reach it, or are above `low`.  A wave by itself.
// Cheapest the k-th largest of the largest of 64 groups, or of 16; where the threads that reach that are too many for the list, the
// k-th largest order itself, bit by bit.
template <int THREADS>
__device__ static inline unsigned kth_of(const unsigned *order, int k, int lane, unsigned low, int &many) {
    constexpr int EACH = THREADS / 64;
    unsigned o[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) o[i] = order[i * 64 + lane];
    auto reach = [&](unsigned q) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) c += __popcll(__ballot(o[i] >= q));
        return c;
    };
    auto larger = [](unsigned p, unsigned q) { return p > q ? p : q; };
    auto smaller = [](unsigned p, unsigned q) { return p < q ? p : q; };
    unsigned g = o[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) g = larger(g, o[i]);
    int above = 0;   // groups above this lane's
    if (k <= 16) {
        g = larger(g, (unsigned)__builtin_amdgcn_update_dpp(0, (int)g, 0xB1, 0xf, 0xf, false));   // of the four lanes
        g = larger(g, (unsigned)__builtin_amdgcn_update_dpp(0, (int)g, 0x4E, 0xf, 0xf, false));
#pragma unroll
        for (int i = 0; i < 64; i += 4) above += (unsigned)__builtin_amdgcn_readlane((int)g, i) > g;
    } else {
#pragma unroll
        for (int i = 0; i < 64; ++i) above += (unsigned)__builtin_amdgcn_readlane((int)g, i) > g;
    }
    const unsigned kth = wave_all(above < k ? g : 0xffffffffu, smaller);
    unsigned tau = kth > low ? kth : low;
    many = reach(tau + (tau == low));
    if (many <= few_threads(THREADS)) return tau;
    if (reach(low + 1) < k) return low;
    tau = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const unsigned q = tau | 1u << bit;
        const int c = reach(q);
        if (c >= k) { tau = q; many = c; }
        if (c == k) break;
    }
    return tau;
}

// Four waves a SIMD, as many workgroups of four as LDS holds lists for: two registers too many cost 254 x 64741 bf16 22 -> 31 us.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == kThreads ? 4 : 1) void answer_kernel(const AnswerArgs a, int parts) {
    constexpr int N = Vec<T>::N, CHUNKS = kEach / N, CHUNK = THREADS * N, SEGMENT = THREADS * kEach;
    typedef T TN __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    __shared__ AnswerLds<THREADS> l;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int row = blockIdx.x / parts, part = blockIdx.x - row * parts, k = a.top;
    const T *x = static_cast<const T *>(a.x) + row * a.stride;
    const int segments = (a.classes + SEGMENT - 1) / SEGMENT;
    const int seg0 = (int)((int64_t)segments * part / parts), seg1 = (int)((int64_t)segments * (part + 1) / parts);
    const float c2 = fminf(a.scale * 1.44269504f, FLT_MAX);   // 0 times infinity would be no number
    int g = -1;
    bool inside = false;
    float xg = INFINITY;

    float max_yet = -INFINITY;
    double s_yet = 0.0, t_yet = 0.0;
    int before = 0;       // logits that come before the given one
    int have = 0;         // classes in the list, the first `have` of it in order
    float bar = -INFINITY;   // the k-th of them: later ones have to be larger
    auto look_up = [&]() {   // behind the first logits' loads: these two wait for one another
        if (!a.given) return;
        g = a.given[row];
        inside = g >= 0 && g < a.classes;
        if (inside) xg = (float)x[g];
    };
    // Of 16 bits the next segment's logits are under way beside this one's 32 numbers (2000 x 20000, five top classes: 36.5 -> 33.9 us; 946 x 69207, none:
    // 44 -> 40; but rows in four parts of two segments, 254 x 64741: 20.2 -> 21.4); of fp32 they take registers from the other waves (860 x 23898: 32.1 -> 34.7).
    constexpr bool AHEAD = sizeof(T) == 2;
    TN raw[CHUNKS];
    auto fetch = [&](int seg) {
        const T *from = x + (int64_t)seg * SEGMENT;
        const int count = a.classes - seg * SEGMENT;
        if (count >= SEGMENT) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) raw[j] = *reinterpret_cast<const TN *>(from + j * CHUNK + t * N);
            return;
        }
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int at = j * CHUNK + t * N;
            if (at + N <= count) {
                raw[j] = *reinterpret_cast<const TN *>(from + at);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) raw[j][e] = at + e < count ? from[at + e] : (T)-INFINITY;
            }
        }
    };
    if constexpr (AHEAD) {
        fetch(seg0);
        look_up();
    }
    for (int seg = seg0; seg < seg1; ++seg) {
        float v[kEach];
        const int base = seg * SEGMENT, count = a.classes - base < SEGMENT ? a.classes - base : SEGMENT;
        if constexpr (AHEAD) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
                for (int e = 0; e < N; ++e) v[j * N + e] = (float)raw[j][e];
            if (seg + 1 < seg1) fetch(seg + 1);
        } else {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                const int at = j * CHUNK + t * N;
                if (at + N <= count) {
                    const TN now = *reinterpret_cast<const TN *>(x + base + at);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[j * N + e] = (float)now[e];
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) v[j * N + e] = at + e < count ? (float)x[base + at + e] : -INFINITY;
                }
            }
            if (seg == seg0) look_up();
        }
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (j * CHUNK >= count) break;
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, v[j * N + e]);
        }
        {
            const float m = fmaxf(max_yet, most), ref = m == -INFINITY ? 0.f : m;
            const float d0 = fmaxf((max_yet - ref) * c2, -1e30f);
            const double e0 = fall(d0);
            max_yet = m;
            float s1 = 0.f, t1 = 0.f;
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                if (j * CHUNK >= count) break;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = (v[j * N + e] - ref) * c2, p = __builtin_amdgcn_exp2f(d);
                    s1 += p;
                    t1 = fmaf(p, fmaxf(d, -1000.f), t1);   // p is 0 long before
                }
            }
            t_yet = fma(fma(s_yet, (double)d0, t_yet), e0, (double)t1);
            s_yet = fma(s_yet, e0, (double)s1);
        }
        if (inside) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                if (j * CHUNK >= count) break;
                const int from = base + j * CHUNK + t * N;
                if (from + N <= g) {
#pragma unroll
                    for (int e = 0; e < N; ++e) before += v[j * N + e] >= xg;
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) before += v[j * N + e] > xg;
                    if (from < g) {
#pragma unroll
                        for (int e = 0; e < N; ++e) before += from + e < g && v[j * N + e] == xg;
                    }
                }
            }
        }
        if (k > 0) {
            // What is above the bar, and of that not much more than the k-th largest of the threads' maxima reach.
            unsigned *order = l.order[(seg - seg0) & 1];
            order[t] = order_of(most);
            if (t == 0) l.n = have;
            __syncthreads();
            int many = 0;
            const unsigned low = order_of(bar), tau = kth_of<THREADS>(order, k, lane, low, many);
            const bool equal = tau != low, all_equal = equal && many <= few_threads(THREADS);   // then those equal to it too, as far as they are needed
            const float from = equal ? of_order(tau) : bar;
            auto put = [&](float value, int i) { l.list[atomicAdd(&l.n, 1)] = key_of(value, base + i); };
            if (most > from || (all_equal && most == from)) {
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) {
                    if (j * CHUNK >= count) break;
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (v[j * N + e] > from || (all_equal && v[j * N + e] == from)) put(v[j * N + e], j * CHUNK + t * N + e);
                }
            }
            __syncthreads();
            int n = l.n;
            if (equal && !all_equal)   // at least k logits are as large as `from`: of those equal to it the first ones are needed, chunk by chunk
                for (int j = 0; n - have < k && j * CHUNK < count; ++j) {
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < kEach; ++i)
                        if (i / N == j && v[i] == from) put(v[i], (i / N) * CHUNK + t * N + i % N);
                    __syncthreads();
                    n = l.n;
                }
            if (n > have) {
                have = first_of(l, n, k);
                __syncthreads();
                if (have == k) bar = of_order((unsigned)(l.list[k - 1] >> 32));
            }
        }
    }

    // The threads meet.
    const auto plus = [](auto p, auto q) { return p + q; };
    const Soft soft = meet({max_yet, (float)s_yet, (float)t_yet}, c2);
    before = wave_all(before, plus);
    Soft all = soft;
    if constexpr (THREADS == 256) {
        if (lane == 0) { l.m[wave] = soft.m; l.s[wave] = soft.s; l.t[wave] = soft.t; l.rank[wave] = before; }
        __syncthreads();
        all = join(join({l.m[0], l.s[0], l.t[0]}, {l.m[1], l.s[1], l.t[1]}, c2), join({l.m[2], l.s[2], l.t[2]}, {l.m[3], l.s[3], l.t[3]}, c2), c2);
        before = l.rank[0] + l.rank[1] + l.rank[2] + l.rank[3];
    }

    if (parts > 1) {
        // This part's record to memory, past the XCD's own L2; the last workgroup of the row to arrive joins them, in the parts' order.
        int *counter = static_cast<int *>(a.workspace) + row;
        char *records = static_cast<char *>(a.workspace) + kCounterSlots * 4 + (int64_t)row * parts * kRecordBytes;
        {
            int *w = reinterpret_cast<int *>(records + part * kRecordBytes);
            auto put = [&](int i, int value) { __hip_atomic_store(w + i, value, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
            if (t == 0) {
                put(0, __builtin_bit_cast(int, all.m));
                put(1, __builtin_bit_cast(int, all.s));
                put(2, __builtin_bit_cast(int, all.t));
                put(3, before);
            }
            for (int i = t; i < k; i += THREADS) {
                const uint64_t key = i < have ? l.list[i] : 0;
                put(4 + 2 * i, (int)(unsigned)key);
                put(5 + 2 * i, (int)(unsigned)(key >> 32));
            }
        }
        // The stores and the loads behind them go past the L2s one by one: a release and an acquire of the counter would write back and drop all of an
        // XCD's L2 for each workgroup (64 x 50001, 448 workgroups, no top classes: 11.7 us for 7.9).  C++ promises no order of relaxed accesses to different words; it comes
        // from the hardware, as the memory model of gfx942 in LLVM's guide to the AMDGPU backend has it: an agent's store (sc1) counts as outstanding (vmcnt) until
        // it is where the other XCDs' loads of that scope look.  What a release would add, writing back the L2's other lines, is about none of these words.
        __builtin_amdgcn_s_waitcnt(0);   // this thread's stores have been made
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __syncthreads();                 // ... and so have the workgroup's
        if (t == 0) l.last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
        __syncthreads();
        if (!l.last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        if (t == 0) {
            __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            l.n = 0;
        }
        auto get = [&](int p, int i) { return __hip_atomic_load(reinterpret_cast<int *>(records + p * kRecordBytes) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        // A lane a part (kParts <= 64), joined as the threads were.
        const int p = lane < parts ? lane : 0;
        Soft one{lane < parts ? __builtin_bit_cast(float, get(p, 0)) : -INFINITY, lane < parts ? __builtin_bit_cast(float, get(p, 1)) : 0.f,
                 lane < parts ? __builtin_bit_cast(float, get(p, 2)) : 0.f};
        before = wave_all(lane < parts ? get(p, 3) : 0, plus);
        all = meet(one, c2);
        __syncthreads();
        if (k > 0) {
            constexpr int EACH = kParts * kAnswerMostTop / THREADS;
            uint64_t key[EACH], most = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                key[i] = 0;
                const int at = i * THREADS + t;
                if (at < parts * k) {
                    const int p = at / k, j = at - p * k;
                    key[i] = (uint64_t)(unsigned)get(p, 5 + 2 * j) << 32 | (unsigned)get(p, 4 + 2 * j);
                    most = most > key[i] ? most : key[i];
                }
            }
            l.order[0][t] = (unsigned)(most >> 32);
            __syncthreads();
            int many;
            const unsigned tau = kth_of<THREADS>(l.order[0], k, lane, 0, many);
            if (most)
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (key[i] && (unsigned)(key[i] >> 32) >= tau) l.list[atomicAdd(&l.n, 1)] = key[i];
            __syncthreads();
            have = first_of(l, l.n, k);
            __syncthreads();
        }
    }

    const bool bad = !(all.s < INFINITY) || all.m == INFINITY, empty = all.m == -INFINITY;
    const float ls = logf(all.s);
    if (t == 0) {
        float lp = bad || !inside ? NAN : empty ? -INFINITY : (xg - all.m) * a.scale - ls;
        if (g < 0) lp = 0.f;
        if (a.logp) a.logp[row] = lp;
        if (a.rank) a.rank[row] = bad || !inside ? -1 : before;
        if (a.entropy) a.entropy[row] = bad ? NAN : empty ? 0.f : ls - all.t * 0.693147181f / all.s;
    }
    if (t < k) {
        const bool some = t < have && !bad;
        const uint64_t key = some ? l.list[t] : 0;
        a.top_id[(int64_t)row * k + t] = some ? (int)~(unsigned)key : -1;
        a.top_logp[(int64_t)row * k + t] = bad ? NAN : some ? (of_order((unsigned)(key >> 32)) - all.m) * a.scale - ls : -INFINITY;
    }
}

template <int THREADS>
static void launch_answer_threads(const AnswerArgs &a, dim3 grid, int parts, hipStream_t s) {
    if (a.dtype == DT_F32) answer_kernel<float, THREADS><<<grid, THREADS, 0, s>>>(a, parts);
    else if (a.dtype == DT_F16) answer_kernel<f16, THREADS><<<grid, THREADS, 0, s>>>(a, parts);
    else answer_kernel<bf16, THREADS><<<grid, THREADS, 0, s>>>(a, parts);
}

size_t answer_workspace_bytes() { return kCounterSlots * 4 + (size_t)kRecords * kRecordBytes; }

hipError_t launch_answer(const AnswerArgs &a, hipStream_t s) {
    if (a.rows < 1 || a.rows > kAnswerMostRows || a.classes < 1 || a.classes > kAnswerMostClasses || a.top < 0 || a.top > kAnswerMostTop || (a.top > 0 && (!a.top_id || !a.top_logp))) return hipErrorInvalidValue;
    // Shared are as many rows as there are counters, each by as many workgroups as records and segments allow: 256 x 64741 bf16 21.8 us in four parts a row, 257 rows in
    // one 34.1; 64 x 50001 11.9 in seven.
    const int segments = (a.classes + kSegment - 1) / kSegment;
    int parts = 1;
    if (a.workspace && a.rows <= kCounterSlots) {
        parts = kRecords / a.rows;
        parts = parts < kParts ? parts : kParts;
        parts = parts < segments ? parts : segments;
    }
    const dim3 grid((unsigned)a.rows * parts);
    // Short rows, more than two a CU, have a wave to themselves, and no barrier: 1802 x 37 14.3 -> 7.0 us, 1962 x 1741 16.4 -> 9.6; but one row of 1000 5.2 -> 5.5.
    if (a.rows > kRowsOfAWave && a.classes <= kFewest * kEach) launch_answer_threads<kFewest>(a, grid, 1, s);
    else launch_answer_threads<kThreads>(a, grid, parts, s);
    return hipGetLastError();
}

}  // namespace cw
