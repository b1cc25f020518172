// Element types of the operators around the layers (layer norm, log probabilities, optimizer step): fp32, bf16 and fp16
// tensors, computed on in fp32; rows read 16 bytes a lane; reductions over the lanes that share a row.
#pragma once
#include "flex_common.hpp"
#include "../../include/flexconv.h"
#include <algorithm>
#include <type_traits>

namespace flex {

typedef __bf16 bf16;

template <class T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

static inline bool dtype_ok(int d) { return d == FLEX_F32 || d == FLEX_BF16 || d == FLEX_F16; }
static inline size_t dtype_bytes(int d) { return d == FLEX_F32 ? 4 : 2; }
// Positions of a call: those of a last workgroup that lies past the end are numbered in an int too.
static inline bool positions_ok(int B, int N) { return B > 0 && N > 0 && (int64_t)B * N <= INT32_MAX - 1023; }
// Whether two sets of `rows` rows of `width` bytes, which lie sa and sb bytes apart, share memory.
static inline bool rows_share(const void *a, int64_t sa, const void *b, int64_t sb, int64_t rows, int64_t width)
{
    const int64_t d = (int64_t)((uintptr_t)b - (uintptr_t)a);
    if (d >= (rows - 1) * sa + width || -d >= (rows - 1) * sb + width) return false;
    if (sa == sb) {        // halves of wider rows, say: their places within a row decide
        const int64_t place = ((d % sa) + sa) % sa;
        return place < width || place > sa - width;
    }
    for (int64_t i = 0; i < rows; ++i) {        // the rows of b around the place of a's row i: the first that ends behind its begin
        const int64_t j = std::max<int64_t>(0, (i * sa - d - width) / sb);
        for (int64_t k = j; k < std::min(rows, j + 3); ++k)
            if (d + k * sb < i * sa + width && i * sa < d + k * sb + width) return true;
    }
    return false;
}
// A launch counts its threads in 32 bits.
static inline bool one_launch(int64_t threads) { return threads < (int64_t)1 << 32; }

// f(T{}) with the element type that a flex_dtype names
template <class F>
static inline hipError_t with_dtype(int d, F f)
{
    if (d == FLEX_F32) return f(float{});
    if (d == FLEX_BF16) return f(bf16{});
    return f(_Float16{});
}

// Elements a lane takes at once; rows may begin at any element (the hardware takes any alignment, and a row's lines are the same).
template <class T>
constexpr int LANE_ELEMENTS = 16 / (int)sizeof(T);
template <class T, int N = LANE_ELEMENTS<T>>
struct Chunk {
    typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    static __device__ __forceinline__ void load(const T *p, float (&x)[N])
    {
        const V v = *(const V *)p;
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = to_f32(v[j]);
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[N])
    {
        V v;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (T)x[j];
        *(V *)p = v;
    }
    // Where a lane that is to take columns c0 .. of a row of C >= N reads: at the row's last N columns rather than past its end, so
    // that no load waits in a branch.  What is not its own then (before c0) is for mask() to overwrite.
    static __device__ __forceinline__ int from(int c0, int C) { return min(c0, C - N); }
    static __device__ __forceinline__ void mask(float (&x)[N], int c0, int C, float fill)
    {
        if (c0 + N > C)
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (C - N + j < c0) x[j] = fill;
    }
    static __device__ __forceinline__ void store_row(T *row, int c0, int C, const float (&x)[N])
    {
        if (c0 + N <= C) store(row + c0, x);
        else
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (c0 + j < C) row[c0 + j] = (T)x[j];
    }
};

// 16 bytes of elements as four words, for what is kept in registers and looked at more than once
typedef uint32_t Words __attribute__((ext_vector_type(4)));
template <class T>
__device__ __forceinline__ void unpack(const Words &w, float (&x)[LANE_ELEMENTS<T>])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = w[i];
        if constexpr (sizeof(T) == 4) x[i] = __builtin_bit_cast(float, b);
        else if constexpr (std::is_same<T, bf16>::value) {
            x[2 * i] = __builtin_bit_cast(float, b << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, b & 0xFFFF0000u);
        } else {
            x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)b);
            x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(b >> 16));
        }
    }
}

// ---- reductions over groups of L neighbouring lanes, the result on every one of them -----------------------------------------
// Up to 16 lanes by DPP (quad permutes, then the mirrored half row and row, whose halves hold one value each by then), then by
// swapping rows of 16 and halves of 32 lanes between a value and its copy; all lanes of a group have to be active.

constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// op of the two values that swap(v, v) leaves.  (They are taken out of their vector first: a bit cast of a vector's element casts the
// first one, whichever it is given.)
template <class V, class Swap, class Op>
__device__ __forceinline__ V swap_reduce(V v, Swap swap, Op op)
{
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto r = swap(b, b);
    const unsigned one = r[0], two = r[1];
    return op(__builtin_bit_cast(V, one), __builtin_bit_cast(V, two));
}
template <int L, class V, class Op>
__device__ __forceinline__ V lanes_reduce(V v, Op op)
{
    const auto moved = [](V v, auto ctrl) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    if (L >= 2) v = op(v, moved(v, std::integral_constant<int, DPP_XOR1>{}));
    if (L >= 4) v = op(v, moved(v, std::integral_constant<int, DPP_XOR2>{}));
    if (L >= 8) v = op(v, moved(v, std::integral_constant<int, DPP_HALF_MIRROR>{}));
    if (L >= 16) v = op(v, moved(v, std::integral_constant<int, DPP_MIRROR>{}));
    if (L >= 32) v = swap_reduce(v, [](unsigned a, unsigned b) { return __builtin_amdgcn_permlane16_swap(a, b, false, false); }, op);
    if (L >= 64) v = swap_reduce(v, [](unsigned a, unsigned b) { return __builtin_amdgcn_permlane32_swap(a, b, false, false); }, op);
    return v;
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v)
{
    return lanes_reduce<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float lanes_max(float v)
{
    return lanes_reduce<L>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ __forceinline__ int lanes_min(int v)
{
    return lanes_reduce<L>(v, [](int a, int b) { return min(a, b); });
}

// an element of a vector over the channels in a parameter type that is known at run time
__device__ __forceinline__ void store_param(void *p, int dtype, int64_t i, float v)
{
    if (dtype == FLEX_F32) ((float *)p)[i] = v;
    else if (dtype == FLEX_BF16) ((bf16 *)p)[i] = (bf16)v;
    else ((_Float16 *)p)[i] = (_Float16)v;
}

}  // namespace flex
