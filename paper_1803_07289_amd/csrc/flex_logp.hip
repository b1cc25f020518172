// Log probabilities of given classes, entropy, log-sum-exp and the best alternatives of every position's C scores, and the
// gradient of the scores.
//   m = max x, s = sum exp(x - m), u = sum exp(x - m) (x - m):  lse = m + ln s,  logp = x_t - m - ln s,  H = ln s - u / s
//   p = exp(x - lse):  grad_x = grad_logp ([c = t] - p) - grad_H p (x - lse + H)
// A score of -inf has p = 0 and no share of anything; positions whose target is no class are ignored (outputs zero, no
// alternatives, gradient zero, scores not looked at); one without any score above -inf has logp = lse = -inf, H = 0.
//
// A score is read once and kept in a register until its position is done: the maximum, the two sums and the alternatives all come from
// there.  Of positions too long for that, a part's running sums are kept, and what may be among the best is read again.
#include "flex_elem.hpp"
#include <algorithm>

namespace flex {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float MASKED = -1e5f;       // stands for x - m = -inf where it is multiplied by exp(x - m) = 0
constexpr int NO_CLASS = 0x7FFFFFFF;
// Up to this maximum exp(x - m) is 2^(x log2(e) - shift), one fused operation, with shift = m log2(e) rounded: the sums are then about the
// shift, and delta = m log2(e) - shift, up to 2^-8 here, is taken out of them once they are finished.  Above it, the difference first.
constexpr float SHIFT_MAX = 65536.f;

struct LogpArgs {
    const int32_t *target;
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_class;
    int64_t rows, stride;             // positions; elements from row to row: of a position's scores, or of a class's (channel-major)
    int N, C, top;
};

// A maximum of a number and a NaN is the number, also if the NaN signals: the mode register's bit 9 off, for the wave.
__device__ __forceinline__ void maxima_of_numbers() { __builtin_amdgcn_s_setreg(1 | 9 << 6, 0); }

struct Sums {
    float m, s, u;
};
// m as the sums are taken about it: an empty position's is no number to subtract
__device__ __forceinline__ float centre(float m) { return m == -INFINITY ? 0.f : m; }

// The sums of n, each about its own m, as one about the largest.
template <int n>
__device__ __forceinline__ Sums joined(const Sums (&k)[n])
{
    Sums all{k[0].m, 0.f, 0.f};
#pragma unroll
    for (int i = 1; i < n; ++i) all.m = fmaxf(all.m, k[i].m);
    const float m = centre(all.m);
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float d = fmaxf(k[i].m - m, MASKED), e = __builtin_amdgcn_exp2f(d * LOG2E);
        all.s += k[i].s * e;
        all.u += (k[i].u + k[i].s * d) * e;
    }
    return all;
}
__device__ __forceinline__ void add_score(Sums &a, float x, float m)
{
    const float z = x - m, e = __builtin_amdgcn_exp2f(z * LOG2E);
    a.s += e;
    a.u += e * fmaxf(z, MASKED);
}
// m log2(e), rounded: nothing that is subtracted from it is fused with the product
__device__ __forceinline__ float rounded_shift(float m)
{
#pragma clang fp contract(off)
    return m * LOG2E;
}
// what m log2(e) is more than its rounded value
__device__ __forceinline__ float shift_error(float m, float shift) { return __builtin_fmaf(m, LOG2E, -shift); }
// ln of the sum about its largest score, whose own term is 1: never below 0, where rounding alone would take it (no score: -inf)
__device__ __forceinline__ float log_sum(float s, float away = 0.f)
{
    const float l = logf(s) - away;
    return l < 0.f && s > 0.f ? 0.f : l;
}
__device__ __forceinline__ void store_sums(const LogpArgs &a, int64_t row, float target_score, const Sums &k, float log_s)
{
    if (a.target) a.logp[row] = k.s == 0.f ? -INFINITY : target_score - k.m - log_s;
    const float h = log_s - k.u / k.s;
    a.entropy[row] = k.s == 0.f || h < 0.f ? 0.f : h;
    a.lse[row] = k.m + log_s;
}
struct Alternative {
    float logp;
    int c;
    __device__ __forceinline__ Alternative() {}
    __device__ __forceinline__ Alternative(float v, int c, const Sums &k, float log_s)
        : logp(v == -INFINITY ? -INFINITY : v - k.m - log_s), c(v == -INFINITY ? -1 : c) {}
};
__device__ __forceinline__ void store_top(const LogpArgs &a, int64_t at, float v, int c, const Sums &k, float log_s)
{
    const Alternative t(v, c, k, log_s);
    a.top_logp[at] = t.logp;
    a.top_class[at] = t.c;
}
// n of them behind one another
template <int n>
__device__ __forceinline__ void store_tops(const LogpArgs &a, int64_t at, const Alternative (&t)[4])
{
#pragma unroll
    for (int q = 0; q < n; ++q) a.top_logp[at + q] = t[q].logp;
#pragma unroll
    for (int q = 0; q < n; ++q) a.top_class[at + q] = t[q].c;
}
__device__ __forceinline__ bool ignored(const LogpArgs &a, int t) { return a.target && (t < 0 || t >= a.C); }

// ---- the best of many ------------------------------------------------------------------------------------------------------

// the bits of a float, ordered like the floats (of the two zeros the positive one: they are equal)
__device__ __forceinline__ uint32_t order_key(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order_key(uint32_t k)
{
    return __builtin_bit_cast(float, k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
// a 16-bit score in the upper half of a word, zeros of one sign, and back
template <class T>
__device__ __forceinline__ float upper_bits(float v)
{
    if constexpr (std::is_same<T, bf16>::value) return v;
    const uint32_t b = __builtin_bit_cast(uint16_t, (_Float16)(v + 0.f));
    return __builtin_bit_cast(float, b << 16);
}
template <class T>
__device__ __forceinline__ float from_upper_bits(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v);       // (of a negative number's key the lower half is ones)
    if constexpr (std::is_same<T, bf16>::value) return __builtin_bit_cast(float, b & 0xFFFF0000u);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(b >> 16));
}
// A candidate as one number, the better ones the larger: the score, then the class, lower ones first.
typedef unsigned long long Candidate;
__device__ __forceinline__ Candidate candidate(float v, int c) { return (Candidate)order_key(v) << 32 | (uint32_t)~c; }
__device__ __forceinline__ float score_of(Candidate e) { return from_order_key((uint32_t)(e >> 32)); }
__device__ __forceinline__ int class_of(Candidate e) { return (int)~(uint32_t)e; }

// A value that at least n of the wave's 64 lanes reach, the largest such one to within the last 12 bits; -inf if fewer are above
// -inf.  Two bits a step: three counts that do not wait for each other.
__device__ __forceinline__ float reached_by(float v, int n)
{
    const uint32_t key = order_key(v);
    uint32_t found = 0;
#pragma unroll 1
    for (int b = 30; b >= 12; b -= 2) {
        const int one = __popcll(__ballot(key >= (found | 1u << b))), two = __popcll(__ballot(key >= (found | 2u << b))),
                  three = __popcll(__ballot(key >= (found | 3u << b)));
        found |= (three >= n ? 3u : two >= n ? 2u : one >= n ? 1u : 0u) << b;
    }
    return found <= order_key(-INFINITY) ? -INFINITY : from_order_key(found);
}

// f(place, candidate) for each of a list in LDS, its place the number of those before it, by `threads` threads, four to a candidate.
// The list's memory ends on a multiple of eight.
template <class F>
__device__ __forceinline__ void each_ranked(const Candidate *list, int found, int tid, int threads, F f)
{
    for (int i = tid >> 2; i < ((found + 15) & ~15); i += threads >> 2) {      // (whole quads, and all lanes of a wave's quads)
        const Candidate own = list[min(i, found - 1)];
        int rank = 0;
#pragma unroll 4
        for (int o = 2 * (tid & 3); o < found; o += 8) {
            const Candidate x = list[o], y = list[o + 1];
            rank += (int)(x > own) + (int)((y > own) & (o + 1 < found));
        }
        rank += __builtin_amdgcn_update_dpp(0, rank, DPP_XOR1, 0xF, 0xF, true);
        rank += __builtin_amdgcn_update_dpp(0, rank, DPP_XOR2, 0xF, 0xF, true);
        if (i < found && (tid & 3) == 0) f(rank, own);
    }
}

// What a part leaves of itself: its sums and its best scores with their classes.
struct LogpParts {
    Sums *sums;                       // [rows][parts], 16 bytes apart
    Candidate *best;                  // [rows][parts][top], in order; 0: none
    int parts, spans;                 // parts of a row, spans of a part
};
constexpr int SUMS_BYTES = 16, SPAN_LOADS = 4;
template <class T>
constexpr int SPAN = 256 * LANE_ELEMENTS<T> * SPAN_LOADS;     // elements that a workgroup takes at a time: 16 KB

constexpr float LOWEST = -3.4028234663852886e38f;
constexpr int WAVE_LIST = 64 * 4 + FLEX_LOGP_MAX_TOP, LISTS_JOINED = 512;

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ void lds_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---- point-major, rows that a wave holds ----------------------------------------------------------------------------------
// L lanes hold a row, U times 16 bytes each.  A wave's operations decide beside the memory (bf16: 2 bytes in the time of some 10 of
// them), so that lanes hold many elements, and few of them nothing: the steps of a reduction are shared by more.
// The best score is the maximum over the lanes, its class the smallest among those that hold it; it is then taken out of its 16 bytes,
// the only ones that are looked at where a row has 32 lanes or more, and so on for each alternative.  Where a row has the wave to itself and more
// than four are asked for, what reaches the `top`-th largest of the lanes' maxima is listed and ranked, in the time of six.
// Scores of 16 bits go into one number with their classes, for which an element costs two operations instead of five.
// us for 336 MB of scores, 0, 1 and 20 alternatives: bf16, 64 classes 67, 88 and 325, 256 classes 66, 82 and 285, 300 classes 73, 97 and 382,
// 1500 classes 68, 89 and 123 (by the longer rows' workgroups 291, 467 and 550), 4096 classes 77, 98 and 128 (118, 173 and 209);
// fp32, 64 classes 61, 65 and 232, 700 classes 55, 58 and 97 (600 classes 241, 413 and 473), 2048 classes 54, 56 and 82 (79, 131 and 151).
constexpr int ROW_LIST = 96;
template <class T, int L, int U>
__global__ __launch_bounds__(256) void logp_rows_kernel(const T *__restrict__ x, LogpArgs a)
{
    constexpr int N = LANE_ELEMENTS<T>;
    __shared__ Candidate s_list[L == 64 ? 4 : 1][ROW_LIST];
    maxima_of_numbers();
    const int sub = threadIdx.x % L;
    const int64_t row = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const bool mine = row < a.rows;
    const int t = mine && a.target ? a.target[row] : 0;
    const bool skip = !mine || ignored(a, t);
    const T *at = x + row * a.stride;
    float v[U][N], most[U];
    int from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        from[u] = Chunk<T>::from((u * L + sub) * N, a.C);
#pragma unroll
        for (int j = 0; j < N; ++j) v[u][j] = -INFINITY;
        if (!skip) Chunk<T>::load(at + from[u], v[u]);
    }
    const float target_score = !skip && sub == 0 && a.target ? to_f32(at[t]) : 0.f;
    float best = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        Chunk<T>::mask(v[u], (u * L + sub) * N, a.C, -INFINITY);
        most[u] = v[u][0];
#pragma unroll
        for (int j = 1; j < N; ++j) most[u] = fmaxf(most[u], v[u][j]);
        best = fmaxf(best, most[u]);
    }
    const float own_best = best;
    best = lanes_max<L>(best);
    Sums k{centre(best), 0.f, 0.f};
    float away = 0.f;       // what the sums are about is so far below m
    if (!__any(fabsf(k.m) > SHIFT_MAX)) {
        const float shift = rounded_shift(k.m);
        away = shift_error(k.m, shift) * LN2;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float z = __builtin_fmaf(v[u][j], LOG2E, -shift), e = __builtin_amdgcn_exp2f(z);
                k.s += e;
                k.u = __builtin_fmaf(e, fmaxf(z, MASKED), k.u);
            }
        k.u *= LN2;
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) add_score(k, v[u][j], k.m);
    }
    k.s = lanes_sum<L>(k.s);
    k.u = lanes_sum<L>(k.u);
    k.u = __builtin_fmaf(-away, k.s, k.u);      // (of both only the quotient is used, and ln s)
    const float log_s = log_sum(k.s, away);
    if (mine && sub == 0) {
        if (skip) {
            a.logp[row] = a.entropy[row] = a.lse[row] = 0.f;
        } else
            store_sums(a, row, target_score, k, log_s);
    }
    if (a.top == 0) return;
    if (L == 64 && a.top > 4) {
        const float least = reached_by(own_best, a.top);
        int count = least == -INFINITY ? ROW_LIST + 1 : 0;
        Candidate *const list = s_list[threadIdx.x >> 6];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!__any(most[u] >= least)) continue;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const uint64_t takers = __ballot(v[u][j] >= least);
                if (!takers) continue;
                const int place = count + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(takers >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)takers, 0));
                if (v[u][j] >= least && place < ROW_LIST) list[place] = candidate(v[u][j], from[u] + j);
                count += __popcll(takers);
            }
        }
        if (count <= ROW_LIST) {        // (otherwise one after another, as below)
            lds_in_order();
            each_ranked(list, count, sub, 64, [&](int rank, Candidate e) {
                if (rank < a.top) store_top(a, row * a.top + rank, score_of(e), class_of(e), k, log_s);
            });
            return;
        }
    }
    // L alternatives, one to a lane, then L stores in one
    float held = -INFINITY;
    int held_class = -1;
    const auto hold = [&](int i, float score, int c) {
        const int place = i % L;
        if (sub == place) {
            held = score;
            held_class = c;
        }
        if (mine && (place == L - 1 || i + 1 == a.top) && sub <= place) store_top(a, row * a.top + i - place + sub, held, held_class, k, log_s);
    };
    if constexpr (sizeof(T) == 2) {
        // a score of 16 bits and its class in one number, the better ones the larger, no two alike; 0: none
        uint32_t key[U][N], most_key[U], best_key = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            most_key[u] = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                key[u][j] = v[u][j] > -INFINITY ? (order_key(upper_bits<T>(v[u][j])) & 0xFFFF0000u) | (uint32_t)(0xFFFF - from[u] - j) : 0u;
                most_key[u] = max(most_key[u], key[u][j]);
            }
            best_key = max(best_key, most_key[u]);
        }
        for (int i = 0; i < a.top; ++i) {
            best_key = lanes_reduce<L>(best_key, [](uint32_t a, uint32_t b) { return max(a, b); });
            hold(i, best_key ? from_upper_bits<T>(from_order_key(best_key & 0xFFFF0000u)) : -INFINITY, 0xFFFF - (int)(best_key & 0xFFFFu));
            if (i + 1 == a.top) break;
            uint32_t next = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (L < 32 || most_key[u] == best_key) {        // (of few lanes some row's best is nearly always here)
                    most_key[u] = 0;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        key[u][j] = key[u][j] == best_key ? 0u : key[u][j];
                        most_key[u] = max(most_key[u], key[u][j]);
                    }
                }
                next = max(next, most_key[u]);
            }
            best_key = next;
        }
        return;
    }
    for (int i = 0; i < a.top; ++i) {
        int c = NO_CLASS;
#pragma unroll
        for (int u = U - 1; u >= 0; --u)
            if (L < 32 || most[u] == best)
#pragma unroll
                for (int j = N - 1; j >= 0; --j)
                    if (v[u][j] == best) c = from[u] + j;
        c = lanes_min<L>(c);
        hold(i, best, c);
        if (i + 1 == a.top) break;
        float next = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (L < 32 || most[u] == best) {
                most[u] = -INFINITY;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (from[u] + j == c) v[u][j] = -INFINITY;
                    most[u] = fmaxf(most[u], v[u][j]);
                }
            }
            next = fmaxf(next, most[u]);
        }
        best = lanes_max<L>(next);
    }
}

// ---- point-major, longer rows ---------------------------------------------------------------------------------------------
// A workgroup runs along a part of a row, 16 KB at a time, the next 16 KB on their way meanwhile.  A lane's sums are about its own
// maximum so far and meet at the end.  What an element costs decides beside the memory (bf16: 2 bytes in the time of some 11 vector
// operations): exp counts four, the product and difference in front of it are one fused operation, the maximum takes two elements a
// step.  A lane's sums are about its maximum's rounded shift while the wave has met none above SHIFT_MAX, then about the maximum itself, as
// all are when they meet.
// Alternatives: the `top`-th largest of the 64 maxima that four lanes each have met so far is reached by `top` scores of the part, so
// only what reaches it can be among the best; that goes to the wave's list in LDS.  The bound is found after the first span and
// renewed when as many again have passed, from whatever maxima the other waves have left by then: each is a score of the part,
// and an older one is a lower bound too.  A list that fills up (rows of equal scores, ascending rows) is cut to the best `top`;
// scores of later spans then have to exceed the last of them.  The lists meet in one, cut by the largest bound of the four waves,
// and are ranked there.  Parts of one row meet in logp_join_kernel.
// 2046 x 129280 bf16, a tenth ignored, 8 alternatives: 91 us (476 MB, 5.2 TB/s).  One row of 131072 bf16, 20 alternatives: 6 us in 16 parts
// and 4.5 to join them.  336 MB of scores, 0, 1 and 20 alternatives: bf16, 5000 classes 93, 143 and 174 us (a span is 8192), 131072 classes
// 55, 58 and 73; fp32, 4096 classes 49, 66 and 83, 131072 classes 53, 59 and 67.
template <class T>
__global__ __launch_bounds__(256) void logp_part_kernel(const T *__restrict__ x, LogpArgs a, LogpParts p)
{
    constexpr int N = LANE_ELEMENTS<T>, U = SPAN_LOADS, GROUPS = U * N / 4;
    typedef typename Chunk<T>::V V;
    maxima_of_numbers();
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned part = blockIdx.x % p.parts;
    const int64_t row = blockIdx.x / p.parts;
    const int t = a.target ? a.target[row] : 0;
    if (ignored(a, t)) {
        if (part == 0) {
            if (tid == 0) a.logp[row] = a.entropy[row] = a.lse[row] = 0.f;
            if (tid < a.top) {
                a.top_logp[row * a.top + tid] = -INFINITY;
                a.top_class[row * a.top + tid] = -1;
            }
        }
        return;
    }
    __shared__ Sums s_sums[4];
    __shared__ float s_bound[4];
    __shared__ volatile float s_most[64];
    __shared__ int s_count;
    __shared__ Candidate s_list[4][WAVE_LIST], s_cut[4][FLEX_LOGP_MAX_TOP], s_joined[LISTS_JOINED];
    Candidate *const list = s_list[wave];
    const T *at = x + row * a.stride;
    const int begin = (int)part * p.spans * SPAN<T>, end = min(a.C, begin + p.spans * SPAN<T>);
    V next[U];
    auto request = [&](int c) {
#pragma unroll
        for (int u = 0; u < U; ++u) next[u] = __builtin_nontemporal_load((const V *)(at + Chunk<T>::from(c + (u * 256 + tid) * N, a.C)));
    };
    request(begin);
    const float target_score = tid == 0 && a.target && p.parts == 1 ? to_f32(at[t]) : 0.f;
    Sums k{-INFINITY, 0.f, 0.f};       // of the lane; u in units of ln 2
    float about = -INFINITY;           // the shift that they are about, unless the wave is far
    bool far = false;
    const auto about_maximum = [&]() {
        const float m = centre(k.m), d = shift_error(m, rounded_shift(m)), e = __builtin_amdgcn_exp2f(-d);
        k.u = __builtin_fmaf(-d, k.s, k.u) * e;
        k.s *= e;
    };
    float least = LOWEST, bound = LOWEST;       // what a candidate reaches; what `top` scores of the part are known to reach
    float last = -INFINITY;            // the least of the list when it was last cut
    int count = 0, renew = begin;      // the wave's list; where its bound is due

    // the list's best `top`, in order
    auto cut = [&]() {
        lds_in_order();
        each_ranked(list, count, lane, 64, [&](int rank, Candidate e) {
            if (rank < a.top) s_cut[wave][rank] = e;
        });
        lds_in_order();
        if (count <= a.top) return;
        if (lane < a.top) list[lane] = s_cut[wave][lane];
        count = a.top;
        last = score_of(s_cut[wave][a.top - 1]);
        bound = fmaxf(bound, last);
        least = fmaxf(least, last);
        lds_in_order();
    };

    for (int c = begin; c < end; c += SPAN<T>) {
        float v[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) v[u][j] = to_f32(next[u][j]);
        if (c + SPAN<T> < end) request(c + SPAN<T>);
        if (c + SPAN<T> > a.C)
#pragma unroll
            for (int u = 0; u < U; ++u) Chunk<T>::mask(v[u], c + (u * 256 + tid) * N, a.C, -INFINITY);
        float most[GROUPS], span_most = -INFINITY;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const float *w = &v[g / (N / 4)][g % (N / 4) * 4];
            most[g] = max3(max3(w[0], w[1], w[2]), w[3], -INFINITY);
            span_most = fmaxf(span_most, most[g]);
        }
        const float was = k.m, now = fmaxf(was, span_most), m = centre(now), was_about = about;
        if (!far && __any(fabsf(m) > SHIFT_MAX)) {
            about_maximum();
            far = true;
        }
        k.m = now;
        about = rounded_shift(now);
        const float shift = centre(about);
        {
            const float d = fmaxf(far ? (was - m) * LOG2E : was_about - shift, MASKED), e = __builtin_amdgcn_exp2f(d);
            k.u = (k.u + k.s * d) * e;
            k.s *= e;
        }
        float s[2] = {0.f, 0.f}, q[2] = {0.f, 0.f};
        if (!far) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float z = __builtin_fmaf(v[u][j], LOG2E, -shift), e = __builtin_amdgcn_exp2f(z);
                    s[j & 1] += e;
                    q[j & 1] = __builtin_fmaf(e, fmaxf(z, MASKED), q[j & 1]);
                }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float z = (v[u][j] - m) * LOG2E, e = __builtin_amdgcn_exp2f(z);
                    s[j & 1] += e;
                    q[j & 1] = __builtin_fmaf(e, fmaxf(z, MASKED), q[j & 1]);
                }
        }
        k.s += s[0] + s[1];
        k.u += q[0] + q[1];
        if (a.top == 0 || !(c == begin || __any(span_most >= least))) continue;
        if (c >= renew) {
            const float four = lanes_max<4>(k.m);
            if ((lane & 3) == 0) s_most[tid >> 2] = four;
            if (c == begin) __syncthreads();
            bound = fmaxf(bound, reached_by(s_most[lane], a.top));
            least = fmaxf(least, bound);
            renew = c + (c - begin) + SPAN<T>;
        }
        unsigned groups = 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) groups |= most[g] >= least ? 1u << g : 0u;
        while (const uint64_t lanes = __ballot(groups != 0)) {
            if (count + 4 * __popcll(lanes) > WAVE_LIST) cut();
            const int g = groups ? __builtin_ctz(groups) : 0, own = c + (g / (N / 4) * 256 + tid) * N;
            const int from = Chunk<T>::from(own, a.C) + g % (N / 4) * 4;
            float w[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (groups) Chunk<T, 4>::load(at + from, w);
            groups &= groups - 1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool take = w[j] >= least && from + j >= own;
                const uint64_t mask = __ballot(take);
                const int place = count + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
                if (take) list[place] = candidate(w[j], from + j);
                count += __popcll(mask);
            }
        }
        // equal scores of later spans come after the list's (not after those of a wave that may be ahead, from which a larger bound is)
        if (least == last) least = from_order_key(order_key(last) + 1);
    }
    if (count > LISTS_JOINED / 4) cut();
    if (!far) about_maximum();
    Sums all{lanes_max<64>(k.m), 0.f, 0.f};
    {
        const float d = fmaxf((k.m - centre(all.m)) * LOG2E, MASKED), e = __builtin_amdgcn_exp2f(d);
        all.s = lanes_sum<64>(k.s * e);
        all.u = lanes_sum<64>((k.u + k.s * d) * e) * LN2;
    }
    if (tid == 0) s_count = 0;
    if (lane == 0) {
        s_sums[wave] = all;
        s_bound[wave] = bound;
    }
    __syncthreads();
    k = joined(s_sums);
    k.m = p.parts == 1 ? centre(k.m) : k.m;
    const float log_s = log_sum(k.s);
    if (tid == 0) {
        if (p.parts == 1) store_sums(a, row, target_score, k, log_s);
        else *(Sums *)((char *)p.sums + (row * p.parts + part) * SUMS_BYTES) = k;
    }
    if (a.top == 0) return;
    bound = fmaxf(fmaxf(s_bound[0], s_bound[1]), fmaxf(s_bound[2], s_bound[3]));
    for (int i = lane; i < count; i += 64) {
        const Candidate e = list[i];
        if (score_of(e) >= bound) s_joined[atomicAdd(&s_count, 1)] = e;
    }
    __syncthreads();
    const int found = s_count;
    auto put = [&](int i, Candidate e) {
        if (p.parts == 1) store_top(a, row * a.top + i, e ? score_of(e) : -INFINITY, class_of(e), k, log_s);
        else p.best[(row * p.parts + part) * a.top + i] = e;
    };
    each_ranked(s_joined, found, tid, 256, [&](int rank, Candidate e) {
        if (rank < a.top) put(rank, e);
    });
    for (int i = found + tid; i < a.top; i += 256) put(i, 0);
}

// The parts of a row, one to a lane of the row's wave: sums joined, and the alternatives as in a part: the lanes look at the first 64 of
// the parts' best, second best and so on, the `top`-th largest of those is reached by at least as many, and what reaches it
// goes to a list.
constexpr int PARTS_MAX = 64;
template <class T>
__global__ __launch_bounds__(64) void logp_join_kernel(const T *__restrict__ x, LogpArgs a, LogpParts p)
{
    __shared__ Candidate s_list[PARTS_MAX * FLEX_LOGP_MAX_TOP];
    __shared__ int s_count;
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    // all that there is to load is asked for at once (an ignored row's parts have left nothing, and nothing comes of it)
    const int t = a.target ? a.target[row] : 0;
    Sums k{-INFINITY, 0.f, 0.f};
    if (lane < p.parts) k = *(const Sums *)((const char *)p.sums + (row * p.parts + lane) * SUMS_BYTES);
    const Candidate *lists = p.best + row * p.parts * a.top;
    const int entries = p.parts * a.top, depth = 64 / p.parts;
    Candidate looked_at = 0, first = 0;
    if (lane < depth * p.parts && lane / p.parts < a.top) looked_at = lists[lane % p.parts * a.top + lane / p.parts];
    if (lane < entries) first = lists[lane];
    if (ignored(a, t)) return;
    const float target_score = lane == 0 && a.target ? to_f32(x[row * a.stride + t]) : 0.f;
    if (lane == 0) s_count = 0;
    const float m = centre(lanes_max<64>(k.m));
    const float d = fmaxf(k.m - m, MASKED), e = __builtin_amdgcn_exp2f(d * LOG2E);
    k = Sums{m, lanes_sum<64>(k.s * e), lanes_sum<64>((k.u + k.s * d) * e)};
    const float log_s = log_sum(k.s);
    if (lane == 0) store_sums(a, row, target_score, k, log_s);
    if (a.top == 0) return;
    const float least = reached_by(looked_at ? score_of(looked_at) : -INFINITY, a.top);
    __syncthreads();
    for (int i = lane; i < entries; i += 64) {
        const Candidate e = i < 64 ? first : lists[i];
        if (e && score_of(e) >= least) s_list[atomicAdd(&s_count, 1)] = e;
    }
    __syncthreads();
    const int found = s_count;
    each_ranked(s_list, found, lane, 64, [&](int rank, Candidate e) {
        if (rank < a.top) store_top(a, row * a.top + rank, score_of(e), class_of(e), k, log_s);
    });
    for (int i = found + lane; i < a.top; i += 64) store_top(a, row * a.top + i, -INFINITY, NO_CLASS, k, log_s);
}

// ---- channel-major, and point-major rows of few classes ----------------------------------------------------------------------
// A row of C <= R elements to a lane; what lies behind it is left as it is.
template <class T, int R>
__device__ __forceinline__ void load_few(const T *row, int C, float (&v)[R])
{
    constexpr int N = LANE_ELEMENTS<T>;
#pragma unroll
    for (int q = 0; q < R; q += N) {
        if (q + N <= C) {
            float piece[N];
            Chunk<T>::load(row + q, piece);
#pragma unroll
            for (int j = 0; j < N; ++j) v[q + j] = piece[j];
        } else
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (q + j < C) v[q + j] = to_f32(row[q + j]);
    }
}

// A lane to a position, W waves of a workgroup share the classes: R of them a wave in registers, or (R = 0) any number, read again
// for each alternative.  What the waves find meets in LDS.
// ROWS: point-major; the lanes of a wave read their rows 16 bytes at a time, which fills whole lines over a few loads.
// 1M x 13 fp32 with 3 alternatives, point-major: 18.9 us, 92 MB (without alternatives 13.6, 68 MB); channel-major 20 (13.9).  A wave's
// stores decide beside the memory: those of a row's alternatives, 4 bytes at a time, made it 21.6.  Channel-major, 168 MB of scores, 0, 3 and
// 20 alternatives: fp32, 16 classes 31 us, 43 and -, 64 36, 43 and 136, 256 54, 111 and 429, 400 60, 244 and 1316; bf16, 16 classes 37, 73 and - (113
// when each load was converted in a branch of its own), 64 48, 78 and 259, 256 94, 203 and 814, 400 93, 382 and 2098.  (R = 0 reads all scores
// twice and once more for each alternative.)
template <class T, int W, int R, bool ROWS>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void logp_lanes_kernel(const T *__restrict__ x, LogpArgs a)
{
    __shared__ Sums s_sums[W][64];
    __shared__ float s_best[W][64];
    __shared__ int s_class[W][64];
    maxima_of_numbers();
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
    const unsigned tile = W == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x, tiles = ROWS ? 1u : (unsigned)(a.N + 63) / 64;
    const int64_t b = ROWS ? 0 : tile / tiles;
    const int64_t n = (int64_t)(ROWS ? tile : tile % tiles) * 64 + lane;
    const bool mine = ROWS ? n < a.rows : n < a.N && b * a.N < a.rows;
    const int64_t row = b * a.N + n;
    const int t = mine && a.target ? a.target[row] : 0;
    const bool skip = !mine || ignored(a, t);
    const T *at = ROWS ? x + row * a.stride : x + b * a.C * a.stride + n;
    const int64_t step = ROWS ? 1 : a.stride;
    const int per = R ? R : (a.C + W - 1) / W, first = wave * per, last = min(first + per, a.C);
    float v[R ? R : 1];
    Sums k{-INFINITY, 0.f, 0.f};
    float best = -INFINITY;
    if (R) {
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = -INFINITY;
        if constexpr (ROWS) {
            // (an ignored row's scores lie in lines that its neighbours need: they are loaded beside the target, and not used)
            if (mine) load_few<T, R>(at, a.C, v);
        } else {
            // (all loads before the first is converted, in no branch)
            T raw[R ? R : 1];
            const T *from = mine ? at : x;
#pragma unroll
            for (int i = 0; i < R; ++i) raw[i] = from[min(first + i, a.C - 1) * step];
#pragma unroll
            for (int i = 0; i < R; ++i) v[i] = first + i < last ? to_f32(raw[i]) : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) best = fmaxf(best, v[i]);
        k.m = best;
        const float m = centre(best);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (first + i / 4 * 4 < last) add_score(k, v[i], m);
    } else if (!skip) {
#pragma unroll 8
        for (int c = first; c < last; ++c) best = fmaxf(best, to_f32(at[c * step]));
        k.m = best;
        const float m = centre(best);
#pragma unroll 8
        for (int c = first; c < last; ++c) add_score(k, to_f32(at[c * step]), m);
    }
    if (W > 1) {
        s_sums[wave][lane] = k;
        __syncthreads();
        Sums all[W];
#pragma unroll
        for (int w = 0; w < W; ++w) all[w] = s_sums[w][lane];
        k = joined(all);
    }
    k.m = centre(k.m);
    const float log_s = logf(k.s);
    if (wave == 0 && mine) {
        if (skip) a.logp[row] = a.entropy[row] = a.lse[row] = 0.f;
        else store_sums(a, row, a.target ? to_f32(at[t * step]) : 0.f, k, log_s);
    }
    if (W == 1) {
        // the first of those that are the maximum goes at once: three vector operations an element
        const auto next = [&]() {
            best = -INFINITY;
#pragma unroll
            for (int r = 0; r < R; ++r) best = fmaxf(best, v[r]);
            bool found = false;
            int c = NO_CLASS;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool hit = v[r] == best && !found;
                found |= hit;
                c = hit ? r : c;
                v[r] = hit ? -INFINITY : v[r];
            }
            return Alternative(skip ? -INFINITY : best, c, k, log_s);
        };
        if (!ROWS) {
            for (int i = 0; i < a.top; ++i) {
                const Alternative t = next();
                const int64_t to = (b * a.top + i) * a.N + n;
                if (mine) a.top_logp[to] = t.logp;
                if (mine) a.top_class[to] = t.c;
            }
            return;
        }
        // (four at a time: a row's lie behind one another)
        for (int i = 0; i < a.top; i += 4) {
            Alternative t[4];
            const int many = min(4, a.top - i);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (q < many) t[q] = next();
            if (!mine) continue;
            const int64_t to = row * a.top + i;
            if (many == 4) store_tops<4>(a, to, t);
            else if (many == 3) store_tops<3>(a, to, t);
            else if (many == 2) store_tops<2>(a, to, t);
            else store_tops<1>(a, to, t);
        }
        return;
    }
    float last_best = INFINITY;
    int last_class = -1;
    for (int i = 0; i < a.top; ++i) {
        best = -INFINITY;
        int c = NO_CLASS;
        if (R) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (v[r] > best) { best = v[r]; c = first + r; }
        } else if (!skip) {
#pragma unroll 8
            for (int r = first; r < last; ++r) {
                const float y = to_f32(at[r * step]);
                const bool better = y > best && (y < last_best || (y == last_best && r > last_class));
                best = better ? y : best;
                c = better ? r : c;
            }
        }
        s_best[wave][lane] = best;
        s_class[wave][lane] = c;
        __syncthreads();
        best = s_best[0][lane];
        c = s_class[0][lane];
#pragma unroll
        for (int w = 1; w < W; ++w)
            if (s_best[w][lane] > best) { best = s_best[w][lane]; c = s_class[w][lane]; }
        __syncthreads();
        if (wave == 0 && mine) store_top(a, (b * a.top + i) * a.N + n, skip ? -INFINITY : best, c, k, log_s);
        last_best = best;
        last_class = c;
        if (R)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (first + r == c) v[r] = -INFINITY;
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------------------
// An lse is one fp32 number, and its last bit a factor of every p: up to 2^-24 |lse| of it.  Above LSE_EXACT (2^-17) a row's p are therefore
// divided by their sum, which costs such a row another pass: by the threads that have it or, where several workgroups do, by one of them
// alone, so that in place nothing is read that another one has written.  (A forward pass's lse is no less than the largest score: no power
// overflows.)
constexpr float LSE_EXACT = 128.f;

struct LogpBwdArgs {
    const int32_t *target;
    const float *lse, *entropy, *grad_logp, *grad_entropy;
    int64_t rows, stride, grad_stride;           // positions; elements from row to row of the scores and of their gradient
    int N, C;
};
struct LogpBwdRow {
    int t;
    bool zero;
    float lse, gl, gh, h, log2_share = 0.f;      // the last: minus log2 of the sum of the p, where they are divided by it
    __device__ __forceinline__ LogpBwdRow(const LogpBwdArgs &a, int64_t row)
    {
        t = a.target ? a.target[row] : -1;
        lse = a.lse[row];
        zero = (a.target && (t < 0 || t >= a.C)) || lse == -INFINITY;
        gl = a.grad_logp ? a.grad_logp[row] : 0.f;
        gh = a.grad_entropy ? a.grad_entropy[row] : 0.f;
        h = a.grad_entropy ? a.entropy[row] : 0.f;
    }
    __device__ __forceinline__ bool far() const { return !zero && fabsf(lse) > LSE_EXACT && fabsf(lse) < INFINITY; }
    __device__ __forceinline__ float term(float x) const { return __builtin_amdgcn_exp2f((x - lse) * LOG2E); }
    // terms: the sum over all of the row's scores (of an lse that is not the row's own it may be no number to divide by)
    __device__ __forceinline__ void divide_by(float terms)
    {
        if (!(terms > 0.f && terms < INFINITY)) return;
        log2_share = -log2f(terms);
        h = __builtin_fmaf(log2_share, LN2, h);
    }
    __device__ __forceinline__ float operator()(float x, int c) const
    {
        const float lp = x - lse, p = __builtin_amdgcn_exp2f(__builtin_fmaf(lp, LOG2E, log2_share));
        const float v = -p * (gl + gh * (fmaxf(lp, MASKED) + h));
        return c == t ? v + gl : v;
    }
};

// A row by L neighbouring threads, whose elements are a thread's own in both passes.
template <class T, int L>
__device__ __forceinline__ void logp_bwd_far_row(const T *at, T *to, int C, LogpBwdRow f)
{
    constexpr int N = LANE_ELEMENTS<T>, AHEAD = L == 256 ? 4 : 1;        // (registers of the others are few)
    const int sub = threadIdx.x % L, pieces = C / N;
    float terms = 0.f;
#pragma unroll AHEAD
    for (int i = sub; i < pieces; i += L) {
        float v[N];
        Chunk<T>::load(at + i * N, v);
#pragma unroll
        for (int j = 0; j < N; ++j) terms += f.term(v[j]);
    }
    for (int c = pieces * N + sub; c < C; c += L) terms += f.term(to_f32(at[c]));
    terms = lanes_sum<L < 64 ? L : 64>(terms);
    if (L > 64) {
        __shared__ float s_terms[L / 64 + 1];
        if ((threadIdx.x & 63) == 0) s_terms[threadIdx.x >> 6] = terms;
        __syncthreads();
        terms = 0.f;
#pragma unroll
        for (int i = 0; i < L / 64; ++i) terms += s_terms[i];
    }
    f.divide_by(terms);
#pragma unroll AHEAD
    for (int i = sub; i < pieces; i += L) {
        float v[N];
        Chunk<T>::load(at + i * N, v);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = f(v[j], i * N + j);
        Chunk<T>::store(to + i * N, v);
    }
    for (int c = pieces * N + sub; c < C; c += L) to[c] = (T)f(to_f32(at[c]), c);
}

// Point-major: L lanes to a row, U times 16 bytes each, `chunks` workgroups behind one another along long rows (L = 256).  Bound by memory
// where rows fill their lanes: 336 MB of scores and as much of gradients, bf16, 64 classes 125 us (5.3 TB/s), 100 classes 218, 600 115, 131072
// 112 (6.0 TB/s); fp32, 40 classes 145, 600 115, 131072 112; with scores about 200: bf16 199, 293, 166 and 234, fp32 242, 148 and 263.
template <class T, int L, int U>
__global__ __launch_bounds__(256) void logp_bwd_rows_kernel(const T *x, T *gx, LogpBwdArgs a, int chunks)
{
    constexpr int N = LANE_ELEMENTS<T>;
    const int64_t row = L == 256 ? blockIdx.x / chunks : (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    if (row >= a.rows) return;
    const T *at = x + row * a.stride;
    T *to = gx + row * a.grad_stride;
    const int c0 = ((L == 256 ? (int)(blockIdx.x % chunks) * U * L : 0) + (int)(threadIdx.x % L)) * N;
    const LogpBwdRow f(a, row);
    // (in place no lane may read what another one writes: the elements of the row's end, fewer than a piece, are their lane's own; of
    // several pieces they have registers and operations of their own, so that no other piece waits for them: bf16, 1500 classes 134 and 128 us; of
    // one piece they share its operations: bf16, 100 classes 218 and, apart, 243)
    constexpr bool APART = U > 1;
    typename Chunk<T>::V raw[U];
    T last[N - 1];
    const int end = a.C / N * N;
    const bool has_end = end < a.C && end >= c0 && end < c0 + U * L * N && (end - c0) % (L * N) == 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (!f.zero && c0 + u * L * N + N <= a.C) raw[u] = *(const typename Chunk<T>::V *)(at + c0 + u * L * N);
    if (!f.zero && has_end)
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (end + j < a.C) {
                if (APART) last[j] = at[end + j];
                else raw[0][j] = at[end + j];
            }
    if (__builtin_expect(f.far(), 0)) {
        if (L < 256 || blockIdx.x % chunks == row % chunks) logp_bwd_far_row<T, L>(at, to, a.C, f);        // (all the XCDs have some)
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + u * L * N;
        if (APART && c + N > a.C) break;
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = f.zero ? 0.f : f(to_f32(raw[u][j]), c + j);
        if (APART) Chunk<T>::store(to + c, v);
        else Chunk<T>::store_row(to, c, a.C, v);
    }
    if (APART && has_end)
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (end + j < a.C) to[end + j] = (T)(f.zero ? 0.f : f(to_f32(last[j]), end + j));
}

// Point-major rows of up to R classes, one to a lane.
template <class T, int R>
__global__ __launch_bounds__(256) void logp_bwd_few_kernel(const T *x, T *gx, LogpBwdArgs a)
{
    constexpr int N = LANE_ELEMENTS<T>;
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    T *to = gx + row * a.grad_stride;
    float v[R];
    load_few<T, R>(x + row * a.stride, a.C, v);
    LogpBwdRow f(a, row);
    if (f.far()) {
        float terms = 0.f;
#pragma unroll
        for (int c = 0; c < R; ++c)
            if (c < a.C) terms += f.term(v[c]);
        f.divide_by(terms);
    }
#pragma unroll
    for (int q = 0; q < R; q += N) {
        float piece[N];
#pragma unroll
        for (int j = 0; j < N; ++j) piece[j] = f.zero ? 0.f : f(v[q + j], q + j);
        if (q < a.C) Chunk<T>::store_row(to, q, a.C, piece);
    }
}

// Channel-major: a lane to a position, a workgroup to 256 of them and 16 classes.  168 MB of scores and as much of gradients: fp32,
// 16 classes 81 us, 64 76, 256 74; bf16, which a wave loads in half lines, 16 classes 110, 64 108, 256 95; with scores about 200, fp32 102, 214 and
// 181, bf16 142, 351 and 260.
constexpr int BWD_CLASSES = 16;
template <class T>
__global__ __launch_bounds__(256) void logp_bwd_cols_kernel(const T *x, T *gx, LogpBwdArgs a, unsigned tiles, unsigned parts)
{
    const unsigned part = blockIdx.x % parts, tile = blockIdx.x / parts % tiles;
    const int64_t b = blockIdx.x / parts / tiles;
    const int n = tile * 256 + threadIdx.x;
    if (n >= a.N) return;
    const int first = part * BWD_CLASSES, many = min(BWD_CLASSES, a.C - first);
    const T *at = x + (b * a.C + first) * a.stride + n;
    T *to = gx + (b * a.C + first) * a.grad_stride + n;
    // (an ignored position's scores share their lines with its neighbours': nothing is saved by not reading them)
    T v[BWD_CLASSES];
#pragma unroll
    for (int i = 0; i < BWD_CLASSES; ++i) v[i] = at[min(i, many - 1) * a.stride];        // (in no branch: all before the first is converted)
    LogpBwdRow f(a, b * a.N + n);
    if (f.far()) {        // one part's lane takes all of the position's classes
        if (part != tile % parts) return;
        at -= first * a.stride;
        to -= first * a.grad_stride;
        float terms = 0.f;
        for (int c = 0; c < a.C; c += BWD_CLASSES) {
            float some = 0.f;
#pragma unroll 4
            for (int i = c; i < min(c + BWD_CLASSES, a.C); ++i) some += f.term(to_f32(at[i * a.stride]));
            terms += some;
        }
        f.divide_by(terms);
#pragma unroll 4
        for (int c = 0; c < a.C; ++c) to[c * a.grad_stride] = (T)f(to_f32(at[c * a.stride]), c);
        return;
    }
#pragma unroll
    for (int i = 0; i < BWD_CLASSES; ++i)
        if (i < many) to[i * a.grad_stride] = (T)(f.zero ? 0.f : f(to_f32(v[i]), first + i));
}

// ---- launches -------------------------------------------------------------------------------------------------------------

// f(L, U) with the first of these lanes and 16-byte pieces that hold C.
#define FLEX_ROW_LANES(L, U) \
    if (C <= L * U * LANE_ELEMENTS<T>) return f(std::integral_constant<int, L>{}, std::integral_constant<int, U>{});
template <class T, class F>
static hipError_t with_row_lanes(int C, F f)
{
    FLEX_ROW_LANES(4, 2)
    FLEX_ROW_LANES(4, 3)
    FLEX_ROW_LANES(4, 4)
    FLEX_ROW_LANES(8, 3)
    FLEX_ROW_LANES(8, 4)
    FLEX_ROW_LANES(16, 3)
    FLEX_ROW_LANES(16, 4)
    FLEX_ROW_LANES(32, 3)
    FLEX_ROW_LANES(32, 4)
    FLEX_ROW_LANES(64, 3)
    FLEX_ROW_LANES(64, 4)
    FLEX_ROW_LANES(64, 6)
    FLEX_ROW_LANES(64, 8)
    return hipErrorInvalidValue;
}
// whole waves, for rows of more than 64 lanes' elements
template <class T, class F>
static hipError_t with_row_wave(int C, F f)
{
    FLEX_ROW_LANES(64, 2)
    return with_row_lanes<T>(C, f);
}
// the gradient: many lanes rather than many elements, whole lines at a time, but not half of them idle
template <class T, class F>
static hipError_t with_row_lanes_bwd(int C, F f)
{
    FLEX_ROW_LANES(4, 1)
    FLEX_ROW_LANES(4, 2)
    FLEX_ROW_LANES(4, 3)
    FLEX_ROW_LANES(16, 1)
    FLEX_ROW_LANES(8, 3)
    FLEX_ROW_LANES(32, 1)
    FLEX_ROW_LANES(16, 3)
    FLEX_ROW_LANES(64, 1)
    FLEX_ROW_LANES(32, 3)
    FLEX_ROW_LANES(64, 2)
    FLEX_ROW_LANES(64, 3)
    FLEX_ROW_LANES(64, 4)
    return hipErrorInvalidValue;
}
#undef FLEX_ROW_LANES
// the most that a row kernel takes: 64 lanes x 8 x 16 bytes, the gradient's 64 x 4 x 16
static int row_columns_max(int dtype) { return 8192 / (int)dtype_bytes(dtype); }
static int row_columns_bwd_max(int dtype) { return 4096 / (int)dtype_bytes(dtype); }

// How a long row is cut: into parts of whole spans, so many that there are eight workgroups to a compute unit, or that a part is one
// span, at most PARTS_MAX.
struct PartPlan {
    int parts, spans;
};
static PartPlan plan_parts(int64_t rows, int C, int dtype)
{
    const int span = 256 * SPAN_LOADS * (16 / (int)dtype_bytes(dtype)), all = (int)cdiv64(C, span);
    const int wanted = (int)std::min<int64_t>(std::min(all, PARTS_MAX), std::max<int64_t>(1, 8 * device_cu_count() / rows));
    const int spans = (int)cdiv64(all, wanted);
    return PartPlan{(int)cdiv64(all, spans), spans};
}
static size_t parts_sums_bytes(int64_t rows, int parts) { return align256((size_t)rows * parts * SUMS_BYTES); }

template <class T>
static hipError_t launch_logp_rows(const T *x, const LogpArgs &a, int dtype, void *ws, hipStream_t s)
{
    // A lane to a row up to 32 classes: us, four or eight lanes to a row and one, 2M rows, top 3: fp32, 13 classes 59 and 40, 17 classes
    // 96 and 49, 24 classes 95 and 64, 32 classes 94 and 90; bf16, 13 classes 67 and 38, 24 classes 61 and 43, 32 classes 58 and 53.
    if (a.C <= 32) {
        const dim3 grid((unsigned)cdiv64(a.rows, 256));
        if (a.C <= 16) hipLaunchKernelGGL((logp_lanes_kernel<T, 1, 16, true>), grid, dim3(256), 0, s, x, a);
        else if (a.C <= 24) hipLaunchKernelGGL((logp_lanes_kernel<T, 1, 24, true>), grid, dim3(256), 0, s, x, a);
        else hipLaunchKernelGGL((logp_lanes_kernel<T, 1, 32, true>), grid, dim3(256), 0, s, x, a);
        return hipGetLastError();
    }
    if (a.C <= row_columns_max(dtype)) {
        const auto launch = [&](auto l, auto u) {
            constexpr int L = decltype(l)::value, U = decltype(u)::value;
            hipLaunchKernelGGL((logp_rows_kernel<T, L, U>), dim3((unsigned)cdiv64(a.rows, 256 / L)), dim3(256), 0, s, x, a);
            return hipGetLastError();
        };
        // a wave to a row against fewer lanes, us, 336 MB, 8 and 20 alternatives: bf16, 512 classes 196 and 239, 149 and 288, 1000 classes
        // 126 and 155, 127 and 215; fp32, 256 classes 185 and 211, 120 and 243, 512 classes 105 and 126, 106 and 217
        return a.top > 4 && a.C > 64 * LANE_ELEMENTS<T> ? with_row_wave<T>(a.C, launch) : with_row_lanes<T>(a.C, launch);
    }
    const PartPlan q = plan_parts(a.rows, a.C, dtype);
    const LogpParts p{(Sums *)ws, (Candidate *)((char *)ws + parts_sums_bytes(a.rows, q.parts)), q.parts, q.spans};
    hipLaunchKernelGGL(logp_part_kernel<T>, dim3((unsigned)(a.rows * q.parts)), dim3(256), 0, s, x, a, p);
    if (q.parts > 1)
        hipLaunchKernelGGL(logp_join_kernel<T>, dim3((unsigned)a.rows), dim3(64), 0, s, x, a, p);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_logp_cols(const T *x, const LogpArgs &a, int B, hipStream_t s)
{
    const int64_t tiles = B * cdiv64(a.N, 64);
    const dim3 grid((unsigned)tiles), four((unsigned)cdiv64(tiles, 4));
    if (a.C <= 8) hipLaunchKernelGGL((logp_lanes_kernel<T, 1, 8, false>), four, dim3(256), 0, s, x, a);
    else if (a.C <= 16) hipLaunchKernelGGL((logp_lanes_kernel<T, 1, 16, false>), four, dim3(256), 0, s, x, a);
    else if (a.C <= 32) hipLaunchKernelGGL((logp_lanes_kernel<T, 2, 16, false>), grid, dim3(128), 0, s, x, a);
    else if (a.C <= 64) hipLaunchKernelGGL((logp_lanes_kernel<T, 4, 16, false>), grid, dim3(256), 0, s, x, a);
    else if (a.C <= 128) hipLaunchKernelGGL((logp_lanes_kernel<T, 8, 16, false>), grid, dim3(512), 0, s, x, a);
    else if (a.C <= 256) hipLaunchKernelGGL((logp_lanes_kernel<T, 16, 16, false>), grid, dim3(1024), 0, s, x, a);
    else hipLaunchKernelGGL((logp_lanes_kernel<T, 16, 0, false>), grid, dim3(1024), 0, s, x, a);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_logp_bwd(const T *x, T *gx, const LogpBwdArgs &a, int B, bool bcn, int dtype, hipStream_t s)
{
    if (bcn) {
        const unsigned tiles = (unsigned)(a.N + 255) / 256, parts = (unsigned)(a.C + BWD_CLASSES - 1) / BWD_CLASSES;
        const int64_t grid = (int64_t)B * tiles * parts;
        hipLaunchKernelGGL(logp_bwd_cols_kernel<T>, dim3((unsigned)grid), dim3(256), 0, s, x, gx, a, tiles, parts);
        return hipGetLastError();
    }
    // A lane to a row of at most 32 bytes: us, four lanes to a row and one, 2M rows: fp32, 2 classes 28 and 14, 8 classes 35 and 30,
    // 13 classes 44 and 73; bf16, 5 classes 45 and 20, 13 classes 52 and 40, 24 classes 44 and 56.
    constexpr int FEW = 32 / (int)sizeof(T);
    if (a.C <= FEW) {
        hipLaunchKernelGGL((logp_bwd_few_kernel<T, FEW>), dim3((unsigned)cdiv64(a.rows, 256)), dim3(256), 0, s, x, gx, a);
        return hipGetLastError();
    }
    if (a.C <= row_columns_bwd_max(dtype))
        return with_row_lanes_bwd<T>(a.C, [&](auto l, auto u) {
            constexpr int L = decltype(l)::value, U = decltype(u)::value;
            hipLaunchKernelGGL((logp_bwd_rows_kernel<T, L, U>), dim3((unsigned)cdiv64(a.rows, 256 / L)), dim3(256), 0, s, x, gx, a, 1);
            return hipGetLastError();
        });
    constexpr int U = 2;
    const int chunks = (int)cdiv64(a.C, 256 * LANE_ELEMENTS<T> * U);
    hipLaunchKernelGGL((logp_bwd_rows_kernel<T, 256, U>), dim3((unsigned)(a.rows * chunks)), dim3(256), 0, s, x, gx, a, chunks);
    return hipGetLastError();
}

}  // namespace flex

using namespace flex;

// Threads of a launch, at most: channel-major to 16 classes of a position, the waves of a workgroup being a power of two up to 16;
// point-major to 16 bytes of a row, to 32 of one longer than 64 lanes hold.
static int64_t logp_threads(int B, int N, int C, int dtype, int layout)
{
    if (layout == FLEX_LAYOUT_BCN) {
        int64_t waves = 1;
        while (waves < 16 && waves * 16 < C) waves *= 2;
        return B * cdiv64(N, 256) * 256 * std::max(waves, cdiv64(C, BWD_CLASSES));
    }
    const int lane = 16 / (int)dtype_bytes(dtype);
    int64_t threads = C <= row_columns_bwd_max(dtype) ? 4 : 256 * cdiv64(C, 256 * lane * 2);
    while (threads < 64 && threads * lane < C) threads *= 2;
    return (int64_t)B * N * threads;
}

static bool logp_sizes_ok(int B, int N, int C, int64_t row_stride, int dtype, int layout)
{
    return positions_ok(B, N) && C > 0 && C <= FLEX_LOGP_MAX_CLASSES && (layout == FLEX_LAYOUT_BCN || layout == FLEX_LAYOUT_BNC) &&
           dtype_ok(dtype) && row_stride >= (layout == FLEX_LAYOUT_BCN ? N : C) && row_stride < ((int64_t)1 << 31) &&
           one_launch(logp_threads(B, N, C, dtype, layout));
}

extern "C" {

size_t flexlogp_fwd_workspace_bytes(int B, int N, int C, int top, int dtype, int layout)
{
    if (!logp_sizes_ok(B, N, C, layout == FLEX_LAYOUT_BCN ? N : C, dtype, layout) || top < 0 || top > FLEX_LOGP_MAX_TOP || top > C) return 0;
    if (layout == FLEX_LAYOUT_BCN || C <= row_columns_max(dtype)) return FLEX_LOGP_NO_WORKSPACE;
    const int64_t rows = (int64_t)B * N;
    const int parts = plan_parts(rows, C, dtype).parts;
    return parts == 1 ? FLEX_LOGP_NO_WORKSPACE : parts_sums_bytes(rows, parts) + align256((size_t)rows * parts * top * sizeof(Candidate));
}

int flexlogp_fwd(const void *logits, const int32_t *target, float *logp, float *entropy, float *lse, float *top_logp,
                 int32_t *top_class, int B, int N, int C, int top, int64_t row_stride, int dtype, int layout,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    if (!logits || !entropy || !lse || (target == nullptr) != (logp == nullptr)) return FLEX_ERR_NULL;
    if (top > 0 && (!top_logp || !top_class)) return FLEX_ERR_NULL;
    if (!logp_sizes_ok(B, N, C, row_stride, dtype, layout) || top < 0 || top > FLEX_LOGP_MAX_TOP || top > C) return FLEX_ERR_SHAPE;
    const size_t need = flexlogp_fwd_workspace_bytes(B, N, C, top, dtype, layout);
    if (need > FLEX_LOGP_NO_WORKSPACE && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return FLEX_ERR_WORKSPACE;
    const bool bcn = layout == FLEX_LAYOUT_BCN;
    const LogpArgs a{target, logp, entropy, lse, top_logp, top_class, (int64_t)B * N, row_stride, N, C, top};
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        return bcn ? launch_logp_cols<T>((const T *)logits, a, B, (hipStream_t)stream)
                   : launch_logp_rows<T>((const T *)logits, a, dtype, workspace, (hipStream_t)stream);
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

int flexlogp_bwd(const void *logits, const int32_t *target, const float *lse, const float *entropy, const float *grad_logp,
                 const float *grad_entropy, void *grad_logits, int B, int N, int C, int64_t row_stride, int64_t grad_row_stride,
                 int dtype, int layout, void *stream)
{
    if (!logits || !lse || !grad_logits || (!grad_logp && !grad_entropy) || (grad_logp && !target) || (grad_entropy && !entropy))
        return FLEX_ERR_NULL;
    if (!logp_sizes_ok(B, N, C, row_stride, dtype, layout) || !logp_sizes_ok(B, N, C, grad_row_stride, dtype, layout)) return FLEX_ERR_SHAPE;
    const bool bcn = layout == FLEX_LAYOUT_BCN;
    const int64_t e_bytes = (int64_t)dtype_bytes(dtype);
    if (!(logits == grad_logits && row_stride == grad_row_stride) &&
        rows_share(logits, row_stride * e_bytes, grad_logits, grad_row_stride * e_bytes, (int64_t)B * (bcn ? C : N), (bcn ? N : C) * e_bytes))
        return FLEX_ERR_SHAPE;
    const LogpBwdArgs a{target, lse, entropy, grad_logp, grad_entropy, (int64_t)B * N, row_stride, grad_row_stride, N, C};
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        return launch_logp_bwd<T>((const T *)logits, (T *)grad_logits, a, B, bcn, dtype, (hipStream_t)stream);
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

}  // extern "C"
