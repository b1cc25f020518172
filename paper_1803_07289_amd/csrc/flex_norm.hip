// Layer norm over the channels of every position, forward and backward.
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   with xh = (x - mean) rstd and h = g w:  grad_x = rstd (h - mean(h) - xh mean(h xh)),
//   grad_w = sum over positions of g xh, grad_b = sum of g.
// Sums and statistics are fp32; the mean square is taken about the mean, which loses nothing to cancellation.  Memory bounds all of it:
// a row is read once and stays in registers (fp32) until it is done; only rows too long for that are read again, from L2.
#include "flex_elem.hpp"
#include <algorithm>

namespace flex {

// A vector over the channels, in the tensor's type or in fp32: columns c .. c + N.
template <class T>
struct Param {
    const void *p;
    int f32;
    __device__ __forceinline__ void load(int c, float (&x)[LANE_ELEMENTS<T>]) const
    {
        constexpr int N = LANE_ELEMENTS<T>;
        if (sizeof(T) == 4 || f32) Chunk<float, N>::load((const float *)p + c, x);
        else Chunk<T>::load((const T *)p + c, x);
    }
    __device__ __forceinline__ float operator[](int c) const { return sizeof(T) == 4 || f32 ? ((const float *)p)[c] : to_f32(((const T *)p)[c]); }
};

// Sum over the L threads that share a row: lanes of a wave, or waves through LDS (`place`: slots of its own for each sum between two
// barriers of the caller, one for each wave of the workgroup).
template <int L>
__device__ __forceinline__ float row_sum(float v, float *place)
{
    if (L <= 64) return lanes_sum<L <= 64 ? L : 64>(v);
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = v;
    __syncthreads();
    place += (threadIdx.x >> 6) / (L / 64) * (L / 64);
    v = place[0];
#pragma unroll
    for (int i = 1; i < L / 64; ++i) v += place[i];
    return v;
}

// what lane i has, on all of them
__device__ __forceinline__ float lane_value(float v, int i)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), i));
}

// Sums of columns c0 .. of C: x holds the columns from Chunk::from(c0, C) on, those before c0 another lane's.
template <int N>
__device__ __forceinline__ void store_columns(float *to, int c0, int C, const float (&x)[N])
{
    if (c0 + N <= C) Chunk<float, N>::store(to + c0, x);
    else
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (C - N + j >= c0) to[C - N + j] = x[j];
}

// ---- point-major ------------------------------------------------------------------------------------------------------------
// L threads hold a row, U times 16 bytes each; a group of them takes R rows, which it asks for together.  NARROW: rows of fewer
// channels than 16 bytes hold.
// Memory bounds it where enough of it is asked for at once: the registers of R U = 3 to 4 pieces a thread, and few idle lanes.
// 1M x 128 fp32: 176 us (1.03 GB, 5.9 TB/s).  x and y of 336 MB: bf16, 64 channels 66 us, 264 69 (by 64 lanes 86), 1100 67 (by 256 lanes
// 123), 2100 68 (by 256 lanes 82), 4096 63; fp32, 64 channels 61, 2048 59, 4096 63.
template <class T, int L, int U, int R, bool NARROW>
__global__ __launch_bounds__(L > 256 ? L : 256) void norm_rows_kernel(const T *__restrict__ x, Param<T> w, Param<T> b, T *__restrict__ y,
                                                                      float *mean_out, float *rstd_out, int64_t rows, int C, float eps)
{
    constexpr int N = LANE_ELEMENTS<T>, WG = L > 256 ? L : 256, G = WG / L;
    __shared__ float s_place[2 * R][WG / 64];
    const int sub = threadIdx.x % L;
    const int64_t row0 = (int64_t)blockIdx.x * (G * R) + threadIdx.x / L;
    float v[R][U][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t row = min(row0 + r * G, rows - 1);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c0 = (u * L + sub) * N;
            if (NARROW) {
#pragma unroll
                for (int j = 0; j < N; ++j) v[r][u][j] = c0 + j < C ? to_f32(x[row * C + c0 + j]) : 0.f;
            } else
                Chunk<T>::load(x + row * C + Chunk<T>::from(c0, C), v[r][u]);
        }
    }
    const float count = (float)C;
    float mean[R], rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float own[N];
#pragma unroll
            for (int j = 0; j < N; ++j) own[j] = v[r][u][j];
            if (!NARROW) Chunk<T>::mask(own, (u * L + sub) * N, C, 0.f);
#pragma unroll
            for (int j = 0; j < N; ++j) sum += own[j];
        }
        mean[r] = row_sum<L>(sum, s_place[2 * r]) / count;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float sq = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c0 = (u * L + sub) * N;
            float d[N];
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = v[r][u][j] - mean[r];
            if (NARROW) {
#pragma unroll
                for (int j = 0; j < N; ++j) d[j] = c0 + j < C ? d[j] : 0.f;
            } else
                Chunk<T>::mask(d, c0, C, 0.f);
#pragma unroll
            for (int j = 0; j < N; ++j) sq += d[j] * d[j];
        }
        rstd[r] = 1.f / sqrtf(row_sum<L>(sq, s_place[2 * r + 1]) / count + eps);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c0 = (u * L + sub) * N;
        if (c0 >= C) break;
        const int from = NARROW ? c0 : Chunk<T>::from(c0, C);
        float ww[N], bb[N];
        if (w.p) {
            if (NARROW) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    ww[j] = c0 + j < C ? w[c0 + j] : 0.f;
                    bb[j] = c0 + j < C ? b[c0 + j] : 0.f;
                }
            } else {
                w.load(from, ww);
                b.load(from, bb);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r * G;
            if (row >= rows) break;
            float out[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                out[j] = (v[r][u][j] - mean[r]) * rstd[r];
                if (w.p) out[j] = out[j] * ww[j] + bb[j];
            }
            T *to = y + row * C;
            if (NARROW) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (c0 + j < C) to[c0 + j] = (T)out[j];
            } else
                Chunk<T>::store(to + from, out);        // (columns of another lane's too: the same values)
        }
    }
    if (sub == 0)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r * G;
            if (row >= rows) break;
            if (mean_out) mean_out[row] = mean[r];
            if (rstd_out) rstd_out[row] = rstd[r];
        }
}

// Rows of any length, a workgroup to each, read three times, an element to a lane.  x of 168 MB, forward and backward: 20000 channels fp32 137
// and 226 us, bf16 233 and 419; 2^20 channels, which leave most compute units without a row, fp32 1212 and 1268, bf16 1510 and 2012.
template <class T>
__global__ __launch_bounds__(1024) void norm_long_rows_kernel(const T *__restrict__ x, Param<T> w, Param<T> b, T *__restrict__ y,
                                                              float *mean_out, float *rstd_out, int C, float eps)
{
    __shared__ float s_place[2][16];
    const int64_t row = blockIdx.x;
    const T *at = x + row * C;
    const float count = (float)C;
    float sum = 0.f, sq = 0.f;
    for (int c = threadIdx.x; c < C; c += 1024) sum += to_f32(at[c]);
    const float mean = row_sum<1024>(sum, s_place[0]) / count;
    for (int c = threadIdx.x; c < C; c += 1024) {
        const float d = to_f32(at[c]) - mean;
        sq += d * d;
    }
    const float rstd = 1.f / sqrtf(row_sum<1024>(sq, s_place[1]) / count + eps);
    for (int c = threadIdx.x; c < C; c += 1024) {
        const float d = (to_f32(at[c]) - mean) * rstd;
        y[row * C + c] = (T)(w.p ? d * w[c] + b[c] : d);
    }
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
}

// Two sums at once, over the L threads of each row of a workgroup.
template <int L, int WAVES>
__device__ __forceinline__ void row_sums(float &a, float &b, float (*place)[WAVES])
{
    if (L <= 64) {
        a = lanes_sum<L <= 64 ? L : 64>(a);
        b = lanes_sum<L <= 64 ? L : 64>(b);
        return;
    }
    a = lanes_sum<64>(a);
    b = lanes_sum<64>(b);
    const int wave = threadIdx.x >> 6, first = wave / (L / 64) * (L / 64);
    if ((threadIdx.x & 63) == 0) {
        place[0][wave] = a;
        place[1][wave] = b;
    }
    __syncthreads();
    a = place[0][first];
    b = place[1][first];
#pragma unroll
    for (int i = 1; i < L / 64; ++i) {
        a += place[0][first + i];
        b += place[1][first + i];
    }
}

// Backward: groups of L threads (up to 32, or 1024) walk over rows, the next row of each on its way, their columns' shares of
// grad_w and grad_b in registers; those of a workgroup's groups are added up at the end: one partial sum of 2 C a workgroup.
// A row stays as it was read and is converted twice, for its two sums and for its results: half the registers.  The weights are in
// LDS where rows are long: read from memory they would queue behind the next row.  No store is in a branch: a wait for the next
// row could not be told from one for the store then.  Lanes past a row's end and groups past the last row store what another one
// stores too, the same values.
// PARAMS: with grad_w and grad_b (gx may be null then); otherwise only gx.
// Measured with x, grad_out and grad_x of 504 MB: bf16, 64 channels 105 us (4.8 TB/s), 128 104, 16384 110; fp32, 64 channels 100.
constexpr int rows_bwd_threads(int L) { return L > 256 ? L : 256; }
template <class T, int L, int U, bool PARAMS, bool NARROW>
__global__ __launch_bounds__(rows_bwd_threads(L)) void norm_rows_bwd_kernel(const T *__restrict__ x, Param<T> w, const T *__restrict__ g,
                                                                            const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                            T *__restrict__ gx, float *__restrict__ partials,
                                                                            int64_t rows, int C)
{
    constexpr int N = LANE_ELEMENTS<T>, WG = rows_bwd_threads(L), G = WG / L;
    constexpr bool SHARED = L > 64;
    typedef typename Chunk<T>::V V;
    __shared__ float s_place[2][2][WG / 64];
    __shared__ __attribute__((aligned(16))) float s_weight[SHARED ? L * U * N : 1];
    const int sub = threadIdx.x % L, group = threadIdx.x / L;
    const float count = (float)C;
    const int64_t step = (int64_t)gridDim.x * G;
    struct Row {
        Words x[U], g[U];
        float mean, rstd;
    } one, two;
    // (one row to a wave: its address in scalar registers)
    auto row_of = [&](int64_t first) {
        const int64_t row = min(first + group, rows - 1);
        return L < 64 ? row : (int64_t)__builtin_amdgcn_readfirstlane((int)row);
    };
    auto request = [&](Row &to, int64_t first) {
        const int64_t row = row_of(first);
        const T *const xrow = x + row * C, *const grow = g + row * C;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c0 = (u * L + sub) * N;
            if (NARROW) {
                V a, b;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    a[j] = c0 + j < C ? xrow[c0 + j] : (T)0.f;
                    b[j] = c0 + j < C ? grow[c0 + j] : (T)0.f;
                }
                to.x[u] = __builtin_bit_cast(Words, a);
                to.g[u] = __builtin_bit_cast(Words, b);
            } else {
                to.x[u] = __builtin_bit_cast(Words, *(const V *)(xrow + (unsigned)Chunk<T>::from(c0, C)));
                to.g[u] = __builtin_bit_cast(Words, *(const V *)(grow + (unsigned)Chunk<T>::from(c0, C)));
            }
        }
        to.mean = mean[row];
        to.rstd = rstd[row];
    };
    int64_t first = (int64_t)blockIdx.x * G;
    request(one, first);
    float own_w[SHARED ? 1 : U][N], gw[U][N], gb[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c0 = (u * L + sub) * N;
        float ww[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            ww[j] = 1.f;
            gw[u][j] = gb[u][j] = 0.f;
        }
        if (w.p && (!SHARED || group == 0)) {
            if (NARROW) {
#pragma unroll
                for (int j = 0; j < N; ++j) ww[j] = c0 + j < C ? w[c0 + j] : 0.f;
            } else
                w.load(Chunk<T>::from(c0, C), ww);
        }
        if (SHARED && group == 0) Chunk<float, N>::store(s_weight + c0, ww);
        if (!SHARED)
#pragma unroll
            for (int j = 0; j < N; ++j) own_w[SHARED ? 0 : u][j] = ww[j];
    }
    if (SHARED) __syncthreads();
    auto weights = [&](int u, float (&ww)[N]) {
        if (SHARED) {
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                const v4f four = *(const v4f *)(s_weight + (u * L + sub) * N + j);
#pragma unroll
                for (int k = 0; k < 4; ++k) ww[j + k] = four[k];
            }
        } else
#pragma unroll
            for (int j = 0; j < N; ++j) ww[j] = own_w[SHARED ? 0 : u][j];
    };
    int turn = 0;
    auto take = [&](Row &now, Row &then, int64_t first) {
        const bool mine = first + group < rows;
        T *const to = gx + row_of(first) * C;
        request(then, first + step);        // (behind the last row: the last one again)
        Words (&xr)[U] = now.x, (&gr)[U] = now.g;
        const float m = now.mean, r = now.rstd;
        float s1 = 0.f, s2 = 0.f;
        if (!PARAMS || gx) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int skip = NARROW ? 0 : (u * L + sub) * N + N - C;       // columns that are another lane's
                float xx[N], gg[N], ww[N];
                unpack<T>(xr[u], xx);
                unpack<T>(gr[u], gg);
                weights(u, ww);
                if (skip > 0)
#pragma unroll
                    for (int j = 0; j < N; ++j) gg[j] = j < skip ? 0.f : gg[j];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float xh = (xx[j] - m) * r, h = gg[j] * ww[j];
                    s1 += h;
                    s2 += h * xh;
                }
                if (U > 1) __builtin_amdgcn_sched_barrier(0);       // (the pieces one after the other, in the same registers)
            }
            row_sums<L>(s1, s2, s_place[turn]);
            s1 /= count;
            s2 /= count;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c0 = (u * L + sub) * N, skip = !mine ? N : NARROW ? 0 : c0 + N - C;
            if (sizeof(T) == 2) asm("" : "+v"(xr[u]), "+v"(gr[u]));       // converted again here, and not kept from above
            float xx[N], gg[N];
            unpack<T>(xr[u], xx);
            unpack<T>(gr[u], gg);
#pragma unroll
            for (int j = 0; j < N; ++j) xx[j] = (xx[j] - m) * r;
            if (!PARAMS || gx) {
                float ww[N], out[N];
                weights(u, ww);
#pragma unroll
                for (int j = 0; j < N; ++j) out[j] = (gg[j] * ww[j] - s1 - xx[j] * s2) * r;
                if (NARROW) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (c0 + j < C) to[c0 + j] = (T)out[j];
                } else
                    Chunk<T>::store(to + (unsigned)Chunk<T>::from(c0, C), out);
            }
            if (!PARAMS) continue;
            if (skip > 0)
#pragma unroll
                for (int j = 0; j < N; ++j) gg[j] = j < skip ? 0.f : gg[j];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                gw[u][j] += gg[j] * xx[j];
                gb[u][j] += gg[j];
            }
            if (U > 1) __builtin_amdgcn_sched_barrier(0);
        }
        turn ^= 1;
    };
    // (a workgroup's groups take as many turns as each other: lanes and barriers stay together)
    while (true) {
        take(one, two, first);
        if ((first += step) >= rows) break;
        take(two, one, first);
        if ((first += step) >= rows) break;
    }
    if (!PARAMS) return;
    // groups of one wave by lane, then those of the workgroup (waves, or groups of several) through LDS
    constexpr int LL = L < 64 ? 64 : L, GG = WG / LL;
    __shared__ float s_sum[GG > 1 ? (GG - 1) * L * U * N : 1];
    const int other = threadIdx.x / LL;
    float *const to = partials + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float (&acc)[U][N] = which ? gb : gw;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                for (int o = L; o < 64; o <<= 1) acc[u][j] += __shfl_xor(acc[u][j], o);
                if (other > 0 && threadIdx.x % LL < L) s_sum[((other - 1) * U * N + u * N + j) * L + sub] = acc[u][j];
            }
        if (GG > 1) __syncthreads();
        if (threadIdx.x < L) {
#pragma unroll 1
            for (int k = 0; k < GG - 1; ++k)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[u][j] += s_sum[(k * U * N + u * N + j) * L + sub];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c0 = (u * L + sub) * N;
                if (NARROW) Chunk<float, N>::store_row(to + which * C, c0, C, acc[u]);
                else if (c0 < C) store_columns(to + which * C, c0, C, acc[u]);
            }
        }
        if (GG > 1) __syncthreads();
    }
}

// Backward of rows that take W waves of 16 bytes a lane (1 to 16): as many groups of W waves in a workgroup as 16 waves make, D rows
// of each group in registers, all but one of them on their way.  With grad_w and grad_b one workgroup to a compute unit, since each
// leaves a partial sum (8188 x 5120 bf16: 10 MB of them beside the 252 MB that have to move; two workgroups 7 us more), without
// at least two.  A wave's vector operations decide beside the memory, 14 an element: nothing in a turn is chosen by a lane's place, what
// is another lane's has weight 0 in the row's sums and is left out when the parameters' are stored.
// 8188 x 5120 bf16: 46 us with the 4 us of the partial sums' sum (5.5 TB/s; adding x and grad_out 44), without the parameters' 42.
// x, grad_out and grad_x of 504 MB: bf16, 264 channels 101 us (33 of 64 lanes), 512 98, 1000 100, 2048
// 97, 8192 101; fp32, 132 channels 96, 1024 95, 4096 97.
template <class T, bool PARAMS, bool GRAD_X, int D>
__global__ __launch_bounds__(1024) void norm_wide_rows_bwd_kernel(const T *__restrict__ x, Param<T> w, const T *__restrict__ g,
                                                                  const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                  T *__restrict__ gx, float *__restrict__ partials, int64_t rows, int C,
                                                                  int W)
{
    constexpr int N = LANE_ELEMENTS<T>;
    typedef typename Chunk<T>::V V;
    __shared__ float s_place[2][2][16], s_sum[PARAMS ? 1024 * N : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = (int)(blockDim.x >> 6) / W;
    const int group = wave / W, sub = (int)threadIdx.x - group * W * 64, c0 = sub * N;
    const unsigned from = (unsigned)Chunk<T>::from(c0, C);
    const float part = 1.f / (float)C;
    const int64_t step = (int64_t)gridDim.x * G;
    int zero;       // (in a vector register: a row's statistics come behind its elements, not through the scalar cache, which LDS waits for)
    asm("v_mov_b32 %0, 0" : "=v"(zero));
    struct Row {
        Words x, g;
        float mean, rstd;
    } ring[D];
    auto request = [&](Row &to, int64_t first) {
        const int64_t row = min(first + group, rows - 1);
        to.x = __builtin_bit_cast(Words, *(const V *)(x + row * C + from));
        to.g = __builtin_bit_cast(Words, *(const V *)(g + row * C + from));
        to.mean = (mean + row)[zero];
        to.rstd = (rstd + row)[zero];
    };
    // weights, and those in the row's sums: a lane that reads at the row's end has another lane's columns too, whose sums are that one's
    float ww[N], own[N], gw[N], gb[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        ww[j] = 1.f;
        gw[j] = gb[j] = 0.f;
    }
    if (w.p) w.load(from, ww);
#pragma unroll
    for (int j = 0; j < N; ++j) own[j] = (int)from + j < c0 ? 0.f : ww[j];
    int64_t first = (int64_t)blockIdx.x * G;
#pragma unroll
    for (int d = 0; d < D - 1; ++d) request(ring[d], first + d * step);
    int turn = 0;
    auto take = [&](const Row &now, int64_t first) {
        float xx[N], gg[N];
        unpack<T>(now.x, xx);
        unpack<T>(now.g, gg);
#pragma unroll
        for (int j = 0; j < N; ++j) xx[j] = (xx[j] - now.mean) * now.rstd;
        if (GRAD_X) {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = gg[j] * own[j];
                s1 += h;
                s2 = __builtin_fmaf(h, xx[j], s2);
            }
            s1 = lanes_sum<64>(s1);
            s2 = lanes_sum<64>(s2);
            if (lane == 0) {
                s_place[turn][0][wave] = s1;
                s_place[turn][1][wave] = s2;
            }
            __syncthreads();
            const int from_wave = group * W + min(lane, W - 1);
            s1 = s_place[turn][0][from_wave];
            s2 = s_place[turn][1][from_wave];
            turn ^= 1;
            s1 = lane_value(lanes_sum<16>(lane < W ? s1 : 0.f), 0) * part;
            s2 = lane_value(lanes_sum<16>(lane < W ? s2 : 0.f), 0) * part;
            // (a group past the last row stores what another one stores too, the same values: no store in a branch)
            T *const to = gx + min(first + group, rows - 1) * C;
            float out[N];
#pragma unroll
            for (int j = 0; j < N; ++j) out[j] = __builtin_fmaf(-xx[j], s2, __builtin_fmaf(gg[j], ww[j], -s1)) * now.rstd;
            Chunk<T>::store(to + from, out);
        }
        if (PARAMS && first + group < rows)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                gw[j] = __builtin_fmaf(gg[j], xx[j], gw[j]);
                gb[j] += gg[j];
            }
    };
    for (bool more = true; more;)
#pragma unroll
        for (int d = 0; d < D; ++d) {
            request(ring[(d + D - 1) % D], first + (D - 1) * step);        // (behind the last row: the last one again)
            take(ring[d], first);
            if ((first += step) >= rows) {
                more = false;
                break;
            }
        }
    if (!PARAMS) return;
    float *const to = partials + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float (&acc)[N] = which ? gb : gw;
        if (G > 1) {
            __syncthreads();
            if (group > 0)
#pragma unroll
                for (int j = 0; j < N; ++j) s_sum[((group - 1) * N + j) * W * 64 + sub] = acc[j];
            __syncthreads();
        }
        if (group == 0) {
            for (int k = 0; k < G - 1; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += s_sum[(k * N + j) * W * 64 + sub];
            if (c0 < C) store_columns(to + which * C, c0, C, acc);
        }
    }
}

template <class T>
__global__ __launch_bounds__(1024) void norm_long_rows_bwd_kernel(const T *__restrict__ x, Param<T> w, const T *__restrict__ g,
                                                                  const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                  T *__restrict__ gx, int C)
{
    __shared__ float s_place[2][16];
    const int64_t row = blockIdx.x;
    const float count = (float)C, m = mean[row], r = rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < C; c += 1024) {
        const float h = to_f32(g[row * C + c]) * (w.p ? w[c] : 1.f);
        s1 += h;
        s2 += h * ((to_f32(x[row * C + c]) - m) * r);
    }
    s1 = row_sum<1024>(s1, s_place[0]) / count;
    s2 = row_sum<1024>(s2, s_place[1]) / count;
    for (int c = threadIdx.x; c < C; c += 1024) {
        const float h = to_f32(g[row * C + c]) * (w.p ? w[c] : 1.f);
        gx[row * C + c] = (T)((h - s1 - (to_f32(x[row * C + c]) - m) * r * s2) * r);
    }
}

// Parameters' partial sums of long rows: a thread to a channel, a slice of the positions to a row of workgroups.
template <class T>
__global__ __launch_bounds__(256) void norm_long_rows_params_kernel(const T *__restrict__ x, const T *__restrict__ g,
                                                                    const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                    float *__restrict__ partials, int64_t rows, int64_t per, int C)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    float gw = 0.f, gb = 0.f;
    const int64_t end = min(rows, (int64_t)(blockIdx.y + 1) * per);
    for (int64_t row = (int64_t)blockIdx.y * per; row < end; ++row) {
        const float v = to_f32(g[row * C + c]);
        gw += v * ((to_f32(x[row * C + c]) - mean[row]) * rstd[row]);
        gb += v;
    }
    partials[((int64_t)blockIdx.y * 2 + 0) * C + c] = gw;
    partials[((int64_t)blockIdx.y * 2 + 1) * C + c] = gb;
}

// ---- channel-major ----------------------------------------------------------------------------------------------------------
// A lane to P positions, W waves of a workgroup share the channels: R of them a wave in registers, or (R = 0) any number, read again.
// P = 2 of 16 bits, so that a wave's loads are whole lines.
// Bound by memory.  us, x of 168 MB, forward and backward: fp32, 16 channels 81 and 133, 64 83 and 140, 200 81 and 116, 400 124 and 243; bf16,
// 16 channels 88 and 137 (a position to a lane 105 and 158), 64 87 and 143 (113 and 171), 200 91 and 149 (115 and 149), 400 222 and 414.
constexpr int COL_CHANNELS = 16;

// sums over the waves of a workgroup, by position
template <int W, int P>
__device__ __forceinline__ void waves_sum(float (&v)[P], float (*place)[P][64])
{
    if (W == 1) return;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < P; ++q) place[threadIdx.x >> 6][q][lane] = v[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < P; ++q) {
        v[q] = place[0][q][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) v[q] += place[i][q][lane];
    }
}

template <class T, int W, int R, int P>
__global__ __launch_bounds__(64 * W) void norm_cols_kernel(const T *__restrict__ x, Param<T> w, Param<T> b, T *__restrict__ y,
                                                           float *mean_out, float *rstd_out, int N, int C, float eps)
{
    typedef typename Chunk<T, P>::V V;
    __shared__ float s_place[2][W][P][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned tiles = (unsigned)(N + 64 * P - 1) / (64 * P);
    const int64_t cloud = blockIdx.x / tiles;
    const int n = (int)(blockIdx.x % tiles) * 64 * P + lane * P, n0 = min(n, N - P);
    const bool mine = n < N;        // (the last of an odd number of positions: with the one before it, which another lane writes too, the same)
    const int per = R ? R : (C + W - 1) / W, first = wave * per, last = min(first + per, C);
    const int64_t base = cloud * C * (int64_t)N + n0;
    const float count = (float)C;
    float v[R ? R : 1][P], mean[P], rstd[P];
    V raw[R ? R : 1];        // (all loads before the first is converted, in no branch)
#pragma unroll
    for (int q = 0; q < P; ++q) mean[q] = rstd[q] = 0.f;
    if (R) {
#pragma unroll
        for (int i = 0; i < R; ++i) raw[i] = *(const V *)(x + base + (int64_t)min(first + i, C - 1) * N);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                v[i][q] = first + i < last ? to_f32(raw[i][q]) : 0.f;
                mean[q] += v[i][q];
            }
    } else
#pragma unroll 8
        for (int c = first; c < last; ++c) mean[0] += to_f32(x[base + (int64_t)c * N]);
    const float ww = R && w.p && lane < last - first ? w[first + lane] : 1.f, bb = R && w.p && lane < last - first ? b[first + lane] : 0.f;
    waves_sum<W, P>(mean, s_place[0]);
#pragma unroll
    for (int q = 0; q < P; ++q) mean[q] /= count;
    if (R) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const float d = v[i][q] - mean[q];
                if (first + i < last) rstd[q] += d * d;
            }
    } else
#pragma unroll 8
        for (int c = first; c < last; ++c) {
            const float d = to_f32(x[base + (int64_t)c * N]) - mean[0];
            rstd[0] += d * d;
        }
    waves_sum<W, P>(rstd, s_place[1]);
#pragma unroll
    for (int q = 0; q < P; ++q) rstd[q] = 1.f / sqrtf(rstd[q] / count + eps);
    if (R) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int q = 0; q < P; ++q) v[i][q] = (v[i][q] - mean[q]) * rstd[q] * lane_value(ww, i) + lane_value(bb, i);
        if (!mine) return;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (first + i < last) Chunk<T, P>::store(y + base + (int64_t)(first + i) * N, v[i]);
    } else {
        if (!mine) return;
#pragma unroll 8
        for (int c = first; c < last; ++c) {
            const float d = (to_f32(x[base + (int64_t)c * N]) - mean[0]) * rstd[0];
            y[base + (int64_t)c * N] = (T)(w.p ? d * w[c] + b[c] : d);
        }
    }
    if (wave == 0) {
        if (mean_out) Chunk<float, P>::store(mean_out + cloud * N + n0, mean);
        if (rstd_out) Chunk<float, P>::store(rstd_out + cloud * N + n0, rstd);
    }
}

// Backward: a workgroup walks over tiles of 64 P positions; a lane adds its positions' shares of grad_w and grad_b up for each of its
// channels, the lanes of a wave meet at the end.
template <class T, int W, bool PARAMS, int P>
__global__ __launch_bounds__(64 * W) void norm_cols_bwd_kernel(const T *__restrict__ x, Param<T> w, const T *__restrict__ g,
                                                               const float *__restrict__ mean, const float *__restrict__ rstd,
                                                               T *__restrict__ gx, float *__restrict__ partials, int N, int C,
                                                               unsigned tiles, unsigned total)
{
    constexpr int R = COL_CHANNELS;
    typedef typename Chunk<T, P>::V V;
    __shared__ float s_place[2][W][2 * P][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = wave * R, many = min(R, C - first);
    const float count = (float)C;
    const float ww = w.p && lane < many ? w[first + lane] : 1.f;
    float gw[R], gb[R];
#pragma unroll
    for (int i = 0; i < R; ++i) gw[i] = gb[i] = 0.f;
    int turn = 0;
    for (unsigned tile = blockIdx.x; tile < total; tile += gridDim.x, turn ^= 1) {
        const int64_t cloud = tile / tiles;
        const int n = (int)(tile % tiles) * 64 * P + lane * P, n0 = min(n, N - P);
        const int64_t base = (cloud * C + first) * (int64_t)N + n0, at = cloud * N + n0;
        V xr[R], gr[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            xr[i] = *(const V *)(x + base + (int64_t)min(i, many - 1) * N);
            gr[i] = *(const V *)(g + base + (int64_t)min(i, many - 1) * N);
        }
        float m[P], r[P], s[2 * P];
        Chunk<float, P>::load(mean + at, m);
        Chunk<float, P>::load(rstd + at, r);
#pragma unroll
        for (int q = 0; q < 2 * P; ++q) s[q] = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const float xh = (to_f32(xr[i][q]) - m[q]) * r[q], gg = i < many ? to_f32(gr[i][q]) : 0.f, h = gg * lane_value(ww, i);
                s[q] += h;
                s[P + q] += h * xh;
                if (PARAMS) {
                    const float own = n0 + q >= n ? gg : 0.f;        // (another lane counts a position before n; behind the last there is none)
                    gw[i] += own * xh;
                    gb[i] += own;
                }
            }
        if (PARAMS && !gx) continue;
        waves_sum<W, 2 * P>(s, s_place[turn]);
#pragma unroll
        for (int q = 0; q < 2 * P; ++q) s[q] /= count;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (P > 1) asm("" : "+v"(xr[i]), "+v"(gr[i]));       // converted again here, and not kept from above
            float out[P];
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const float xh = (to_f32(xr[i][q]) - m[q]) * r[q];
                out[q] = (to_f32(gr[i][q]) * lane_value(ww, i) - s[q] - xh * s[P + q]) * r[q];
            }
            if (i < many && n < N) Chunk<T, P>::store(gx + base + (int64_t)i * N, out);
        }
    }
    if (!PARAMS) return;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float a = lanes_sum<64>(gw[i]), b = lanes_sum<64>(gb[i]);
        if (i < many && lane == i) {
            partials[(int64_t)blockIdx.x * 2 * C + first + i] = a;
            partials[(int64_t)blockIdx.x * 2 * C + C + first + i] = b;
        }
    }
}

// more channels than the waves hold: read twice
template <class T>
__global__ __launch_bounds__(1024) void norm_many_cols_bwd_kernel(const T *__restrict__ x, Param<T> w, const T *__restrict__ g,
                                                                  const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                  T *__restrict__ gx, int N, int C)
{
    constexpr int W = 16;
    __shared__ float s_place[W][2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned tiles = (unsigned)(N + 63) / 64;
    const int64_t cloud = blockIdx.x / tiles;
    const int n = (int)(blockIdx.x % tiles) * 64 + lane;
    const int per = (C + W - 1) / W, first = wave * per, last = min(first + per, C);
    const int64_t base = cloud * C * (int64_t)N + min(n, N - 1), at = cloud * N + min(n, N - 1);
    const float m = mean[at], r = rstd[at], count = (float)C;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll 8
    for (int c = first; c < last; ++c) {
        const float h = to_f32(g[base + (int64_t)c * N]) * (w.p ? w[c] : 1.f);
        s1 += h;
        s2 += h * ((to_f32(x[base + (int64_t)c * N]) - m) * r);
    }
    float s[2] = {s1, s2};
    waves_sum<W, 2>(s, s_place);
    s1 = s[0] / count;
    s2 = s[1] / count;
    if (n >= N) return;
#pragma unroll 8
    for (int c = first; c < last; ++c) {
        const float h = to_f32(g[base + (int64_t)c * N]) * (w.p ? w[c] : 1.f);
        gx[base + (int64_t)c * N] = (T)((h - s1 - (to_f32(x[base + (int64_t)c * N]) - m) * r * s2) * r);
    }
}

// their parameters' partial sums: a workgroup to a channel and a slice of the positions
template <class T>
__global__ __launch_bounds__(256) void norm_many_cols_params_kernel(const T *__restrict__ x, const T *__restrict__ g,
                                                                    const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                    float *__restrict__ partials, int64_t rows, int64_t per, int N, int C)
{
    __shared__ float s_place[2][4];
    const int c = blockIdx.x;
    const int64_t end = min(rows, (int64_t)(blockIdx.y + 1) * per);
    float gw = 0.f, gb = 0.f;
    for (int64_t row = (int64_t)blockIdx.y * per + threadIdx.x; row < end; row += 256) {
        const int64_t at = (row / N * C + c) * N + row % N;
        const float v = to_f32(g[at]);
        gw += v * ((to_f32(x[at]) - mean[row]) * rstd[row]);
        gb += v;
    }
    gw = row_sum<256>(gw, s_place[0]);
    gb = row_sum<256>(gb, s_place[1]);
    if (threadIdx.x == 0) {
        partials[((int64_t)blockIdx.y * 2 + 0) * C + c] = gw;
        partials[((int64_t)blockIdx.y * 2 + 1) * C + c] = gb;
    }
}

// ---- partial sums to gradients ------------------------------------------------------------------------------------------------
// COLUMNS to a workgroup, 1024 / COLUMNS threads to each, in the same order at every call: 64, which lines are read whole for, where
// that makes 64 workgroups, otherwise 16.
template <int COLUMNS>
__global__ __launch_bounds__(1024) void norm_params_sum_kernel(const float *__restrict__ partials, int slices, void *gw, void *gb, int C,
                                                               int pdtype)
{
    __shared__ float s_sum[16][COLUMNS];
    const int own = threadIdx.x % COLUMNS, column = blockIdx.x * COLUMNS + own;
    float sum = 0.f;
    if (column < 2 * C)
#pragma unroll 16
        for (int i = threadIdx.x / COLUMNS; i < slices; i += 1024 / COLUMNS) sum += partials[(int64_t)i * 2 * C + column];
    for (int o = COLUMNS; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    s_sum[threadIdx.x >> 6][own] = sum;
    __syncthreads();
    if (threadIdx.x >= COLUMNS || column >= 2 * C) return;
    sum = s_sum[0][own];
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += s_sum[i][own];
    if (column < C) store_param(gw, pdtype, column, sum);
    else store_param(gb, pdtype, column - C, sum);
}

// ---- launches -----------------------------------------------------------------------------------------------------------------

// The row kernels' threads and 16-byte pieces: the smallest that hold C, in steps of at most a half, up to what one wave holds.  f(L, U);
// false: none.
template <class T, class F>
static bool with_row_threads(int C, F f)
{
    constexpr int N = LANE_ELEMENTS<T>;
#define FLEX_ROW_THREADS(L, U) \
    if (C <= L * U * N) return f(std::integral_constant<int, L>{}, std::integral_constant<int, U>{}), true;
    FLEX_ROW_THREADS(4, 1)
    FLEX_ROW_THREADS(8, 1)
    FLEX_ROW_THREADS(16, 1)
    FLEX_ROW_THREADS(32, 1)
    FLEX_ROW_THREADS(16, 3)
    FLEX_ROW_THREADS(64, 1)
    FLEX_ROW_THREADS(32, 3)
    FLEX_ROW_THREADS(64, 2)
    FLEX_ROW_THREADS(64, 3)
    FLEX_ROW_THREADS(64, 4)
    FLEX_ROW_THREADS(128, 3)
    FLEX_ROW_THREADS(256, 2)
    FLEX_ROW_THREADS(256, 3)
    FLEX_ROW_THREADS(256, 4)
    FLEX_ROW_THREADS(1024, 2)
    if constexpr (N == 4) FLEX_ROW_THREADS(1024, 4)
#undef FLEX_ROW_THREADS
    return false;
}
// The longest rows that those hold: 1024 threads, 16 elements each.
constexpr int ROW_CHANNELS_MAX = 16384, COL_CHANNELS_MAX = 16 * COL_CHANNELS;

// f(W): the waves that hold C channels, channel-major
template <class F>
static void with_col_waves(int C, F f)
{
    if (C <= COL_CHANNELS) f(std::integral_constant<int, 1>{});
    else if (C <= 2 * COL_CHANNELS) f(std::integral_constant<int, 2>{});
    else if (C <= 4 * COL_CHANNELS) f(std::integral_constant<int, 4>{});
    else if (C <= 8 * COL_CHANNELS) f(std::integral_constant<int, 8>{});
    else f(std::integral_constant<int, 16>{});
}

// f(P): positions to a lane, channel-major: two of 16 bits, so that a wave's loads are whole lines
template <class T, class F>
static void with_positions(int N, F f)
{
    if constexpr (sizeof(T) == 2)
        if (N >= 2) return f(std::integral_constant<int, 2>{});
    f(std::integral_constant<int, 1>{});
}

// Rows of more than 32 lanes of 16 bytes, up to 16 waves: the backward pass has a kernel for them.
static bool wide_rows(int C, int lane) { return C > 32 * lane && C <= 1024 * lane; }
static int wide_waves(int C, int lane) { return (C + 64 * lane - 1) / (64 * lane); }

// Rows that a group of the forward pass takes together
constexpr int rows_together(int L, int U) { return L > 64 || U == 4 ? 1 : U == 1 ? 4 : 2; }

// Threads of a launch that has some for every position, at most
static int64_t norm_threads(int B, int N, int C, int dtype, bool bcn)
{
    if (bcn) {
        int64_t waves = 16;
        if (C <= COL_CHANNELS_MAX) with_col_waves(C, [&](auto w) { waves = decltype(w)::value; });
        return B * cdiv64(N, 64) * 64 * waves;
    }
    int64_t threads = 1024;
    const auto of_row = [&](auto l, auto u) { threads = decltype(l)::value / rows_together(decltype(l)::value, decltype(u)::value); };
    if (dtype == FLEX_F32) with_row_threads<float>(C, of_row);
    else with_row_threads<bf16>(C, of_row);
    return (int64_t)B * N * threads;
}
constexpr int64_t WALKERS = 1 << 20;        // workgroups, at most, of those backward kernels that walk over the positions

// Partial sums of grad_w and grad_b: the workgroups that walk over the positions, four turns at least to each where there are more than 64
// (us, four turns always and this: fp32, 9 x 11650 28.7 and 17.4; bf16, 40 x 1000 9.4 and 7.4, 1000 x 768 10.9 and 8.9).
static int norm_slices(int B, int N, int C, int dtype, bool bcn)
{
    const int64_t rows = (int64_t)B * N, cus = device_cu_count();
    if (bcn) {
        if (C > COL_CHANNELS_MAX) return (int)std::min<int64_t>(64, cdiv64(rows, 4096));
        const int64_t waves = cdiv64(C, COL_CHANNELS);
        return (int)std::min<int64_t>(B * cdiv64(N, dtype == FLEX_F32 || C > 8 * COL_CHANNELS ? 64 : 128), std::max<int64_t>(cus, 8 * cus / waves));
    }
    if (C > ROW_CHANNELS_MAX) return (int)std::min<int64_t>(64, cdiv64(rows, 16));
    const int lane = 16 / (int)dtype_bytes(dtype);
    int groups = wide_rows(C, lane) ? 16 / wide_waves(C, lane) : 1;
    for (const int L : {32, 16, 8, 4})
        if (C <= L * lane) groups = 256 / L;
    return (int)std::min({cdiv64(rows, groups), std::max<int64_t>(64, cdiv64(rows, 4 * groups)), C <= 32 * lane ? 4 * cus : cus});
}

template <class T>
static hipError_t launch_norm_fwd(const T *x, const void *weight, const void *bias, T *y, float *mean, float *rstd, int B, int N,
                                  int C, float eps, int pdtype, bool bcn, hipStream_t s)
{
    const int64_t rows = (int64_t)B * N;
    const Param<T> w{weight, pdtype == FLEX_F32}, b{bias, pdtype == FLEX_F32};
    if (bcn) {
        if (C > COL_CHANNELS_MAX) {
            hipLaunchKernelGGL((norm_cols_kernel<T, 16, 0, 1>), dim3((unsigned)(B * cdiv64(N, 64))), dim3(1024), 0, s, x, w, b, y, mean, rstd, N, C,
                               eps);
            return hipGetLastError();
        }
        with_col_waves(C, [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            with_positions<T>(N, [&](auto positions) {
                constexpr int P = decltype(positions)::value;
                hipLaunchKernelGGL((norm_cols_kernel<T, W, COL_CHANNELS, P>), dim3((unsigned)(B * cdiv64(N, 64 * P))), dim3(64 * W), 0, s, x, w, b,
                                   y, mean, rstd, N, C, eps);
            });
        });
        return hipGetLastError();
    }
    if (!with_row_threads<T>(C, [&](auto l, auto u) {
            constexpr int L = decltype(l)::value, U = decltype(u)::value, R = rows_together(L, U);
            const dim3 grid((unsigned)cdiv64(rows, (int64_t)std::max(256 / L, 1) * R)), wg(std::max(L, 256));
            if constexpr (L == 4)
                if (C < LANE_ELEMENTS<T>) {
                    hipLaunchKernelGGL((norm_rows_kernel<T, L, U, R, true>), grid, wg, 0, s, x, w, b, y, mean, rstd, rows, C, eps);
                    return;
                }
            hipLaunchKernelGGL((norm_rows_kernel<T, L, U, R, false>), grid, wg, 0, s, x, w, b, y, mean, rstd, rows, C, eps);
        }))
        hipLaunchKernelGGL(norm_long_rows_kernel<T>, dim3((unsigned)rows), dim3(1024), 0, s, x, w, b, y, mean, rstd, C, eps);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_norm_bwd(const T *x, const void *weight, const T *g, const float *mean, const float *rstd, T *gx, void *gw,
                                  void *gb, int B, int N, int C, int dtype, int pdtype, bool bcn, float *partials, hipStream_t s)
{
    const int64_t rows = (int64_t)B * N;
    const Param<T> w{weight, pdtype == FLEX_F32};
    const int slices = norm_slices(B, N, C, dtype, bcn);
    if (bcn && C <= COL_CHANNELS_MAX) {
        with_col_waves(C, [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            auto launch = [&](auto params, auto positions) {
                constexpr int P = decltype(positions)::value;
                const unsigned tiles = (unsigned)(N + 64 * P - 1) / (64 * P), total = (unsigned)B * tiles;
                const int64_t workgroups = gw ? slices : std::min<int64_t>(total, WALKERS);
                hipLaunchKernelGGL((norm_cols_bwd_kernel<T, W, decltype(params)::value, P>), dim3((unsigned)workgroups), dim3(64 * W), 0, s, x, w,
                                   g, mean, rstd, gx, partials, N, C, tiles, total);
            };
            if (!gw) with_positions<T>(N, [&](auto positions) { launch(std::false_type{}, positions); });
            else if constexpr (W == 16) launch(std::true_type{}, std::integral_constant<int, 1>{});       // (two, and the sums do not fit the registers)
            else with_positions<T>(N, [&](auto positions) { launch(std::true_type{}, positions); });
        });
    } else if (bcn) {
        if (gx)
            hipLaunchKernelGGL(norm_many_cols_bwd_kernel<T>, dim3((unsigned)(B * cdiv64(N, 64))), dim3(1024), 0, s, x, w, g, mean, rstd, gx,
                               N, C);
        if (gw)
            hipLaunchKernelGGL(norm_many_cols_params_kernel<T>, dim3((unsigned)C, (unsigned)slices), dim3(256), 0, s, x, g, mean, rstd,
                               partials, rows, cdiv64(rows, slices), N, C);
    } else if (wide_rows(C, LANE_ELEMENTS<T>)) {
        const int W = wide_waves(C, LANE_ELEMENTS<T>), groups = 16 / W;
        auto launch = [&](auto params, auto grad_x, auto deep, int64_t workgroups) {
            hipLaunchKernelGGL((norm_wide_rows_bwd_kernel<T, decltype(params)::value, decltype(grad_x)::value, decltype(deep)::value>),
                               dim3((unsigned)workgroups), dim3(64 * W * groups), 0, s, x, w, g, mean, rstd, gx, partials, rows, C, W);
        };
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 3> three;
        if (gw && gx) launch(std::true_type{}, std::true_type{}, three, slices);
        else if (gw) launch(std::true_type{}, std::false_type{}, three, slices);
        else
            launch(std::false_type{}, std::true_type{}, two,
                   std::min({cdiv64(rows, groups), std::max<int64_t>(2 * device_cu_count(), cdiv64(rows, 16 * groups)), WALKERS}));
    } else if (!with_row_threads<T>(C, [&](auto l, auto u) {
                   constexpr int L = decltype(l)::value, U = decltype(u)::value;
                   if constexpr ((L <= 32 && U == 1) || L == 1024) {       // (the others are wide rows)
                       constexpr int WG = rows_bwd_threads(L);
                       const dim3 wg(WG), grid((unsigned)(gw ? slices : std::min(cdiv64(rows, WG / L), WALKERS)));
                       auto launch = [&](auto params, auto narrow) {
                           hipLaunchKernelGGL((norm_rows_bwd_kernel<T, L, U, decltype(params)::value, decltype(narrow)::value>), grid, wg, 0,
                                              s, x, w, g, mean, rstd, gx, partials, rows, C);
                       };
                       if constexpr (L == 4)
                           if (C < LANE_ELEMENTS<T>) {
                               if (gw) launch(std::true_type{}, std::true_type{});
                               else launch(std::false_type{}, std::true_type{});
                               return;
                           }
                       if (gw) launch(std::true_type{}, std::false_type{});
                       else launch(std::false_type{}, std::false_type{});
                   }
               })) {
        if (gx) hipLaunchKernelGGL(norm_long_rows_bwd_kernel<T>, dim3((unsigned)rows), dim3(1024), 0, s, x, w, g, mean, rstd, gx, C);
        if (gw)
            hipLaunchKernelGGL(norm_long_rows_params_kernel<T>, dim3((unsigned)((C + 255) / 256), (unsigned)slices), dim3(256), 0, s, x, g,
                               mean, rstd, partials, rows, cdiv64(rows, slices), C);
    }
    if (gw) {
        auto launch = [&](auto columns) {
            constexpr int COLUMNS = decltype(columns)::value;
            hipLaunchKernelGGL(norm_params_sum_kernel<COLUMNS>, dim3((unsigned)(2 * C + COLUMNS - 1) / COLUMNS), dim3(1024), 0, s, partials,
                               slices, gw, gb, C, pdtype);
        };
        if (2 * C >= 64 * 64) launch(std::integral_constant<int, 64>{});
        else launch(std::integral_constant<int, 16>{});
    }
    return hipGetLastError();
}

}  // namespace flex

using namespace flex;

static bool norm_sizes_ok(int B, int N, int C, int layout, int dtype, int param_dtype)
{
    return positions_ok(B, N) && C > 0 && C <= FLEX_NORM_MAX_CHANNELS && (layout == FLEX_LAYOUT_BCN || layout == FLEX_LAYOUT_BNC) &&
           dtype_ok(dtype) && (param_dtype == FLEX_F32 || param_dtype == dtype) &&
           one_launch(norm_threads(B, N, C, dtype, layout == FLEX_LAYOUT_BCN));
}
static bool norm_tensors_share(const void *a, const void *b, int B, int N, int C, int dtype)
{
    const int64_t bytes = (int64_t)B * N * C * (int64_t)dtype_bytes(dtype);
    return rows_share(a, bytes, b, bytes, 1, bytes);
}

extern "C" {

int flexnorm_fwd(const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd, int B, int N, int C,
                 float eps, int dtype, int param_dtype, int layout, void *stream)
{
    if (!x || !y || (weight == nullptr) != (bias == nullptr)) return FLEX_ERR_NULL;
    if (!norm_sizes_ok(B, N, C, layout, dtype, param_dtype) || !(eps >= 0.f) || norm_tensors_share(x, y, B, N, C, dtype)) return FLEX_ERR_SHAPE;
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        return launch_norm_fwd<T>((const T *)x, weight, bias, (T *)y, mean, rstd, B, N, C, eps, param_dtype, layout == FLEX_LAYOUT_BCN,
                                  (hipStream_t)stream);
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

size_t flexnorm_bwd_workspace_bytes(int B, int N, int C, int dtype, int layout)
{
    if (!norm_sizes_ok(B, N, C, layout, dtype, dtype)) return 0;
    return align256((size_t)norm_slices(B, N, C, dtype, layout == FLEX_LAYOUT_BCN) * 2 * C * sizeof(float));
}

int flexnorm_bwd(const void *x, const void *weight, const void *grad_out, const float *mean, const float *rstd, void *grad_x,
                 void *grad_weight, void *grad_bias, int B, int N, int C, int dtype, int param_dtype, int layout,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !grad_out || !mean || !rstd || (grad_weight == nullptr) != (grad_bias == nullptr) || (!grad_x && !grad_weight))
        return FLEX_ERR_NULL;
    if (!norm_sizes_ok(B, N, C, layout, dtype, param_dtype) ||
        (grad_x && (norm_tensors_share(x, grad_x, B, N, C, dtype) || norm_tensors_share(grad_out, grad_x, B, N, C, dtype)))) return FLEX_ERR_SHAPE;
    if (grad_weight && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < flexnorm_bwd_workspace_bytes(B, N, C, dtype, layout)))
        return FLEX_ERR_WORKSPACE;
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        return launch_norm_bwd<T>((const T *)x, weight, (const T *)grad_out, mean, rstd, (T *)grad_x, grad_weight, grad_bias, B, N, C, dtype,
                                  param_dtype, layout == FLEX_LAYOUT_BCN, (float *)workspace, (hipStream_t)stream);
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

}  // extern "C"
