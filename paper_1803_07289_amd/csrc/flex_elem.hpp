// Element types of the operators around the layers (layer norm, log probabilities, optimizer step): fp32, bf16 and fp16
// tensors, computed on in fp32.
#pragma once
#include "flex_common.hpp"
#include "../../include/flexconv.h"

namespace flex {

typedef __bf16 bf16;

template <class T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

static inline bool dtype_ok(int d) { return d == FLEX_F32 || d == FLEX_BF16 || d == FLEX_F16; }
static inline size_t dtype_bytes(int d) { return d == FLEX_F32 ? 4 : 2; }

// f(T{}) with the element type that a flex_dtype names
template <class F>
static inline hipError_t with_dtype(int d, F f)
{
    if (d == FLEX_F32) return f(float{});
    if (d == FLEX_BF16) return f(bf16{});
    return f(_Float16{});
}

// a vector over the channels in a parameter type that is known at run time (read rarely: once a workgroup, or from a cache)
__device__ __forceinline__ float load_param(const void *p, int dtype, int64_t i)
{
    if (dtype == FLEX_F32) return ((const float *)p)[i];
    if (dtype == FLEX_BF16) return to_f32(((const bf16 *)p)[i]);
    return to_f32(((const _Float16 *)p)[i]);
}
__device__ __forceinline__ void store_param(void *p, int dtype, int64_t i, float v)
{
    if (dtype == FLEX_F32) ((float *)p)[i] = v;
    else if (dtype == FLEX_BF16) ((bf16 *)p)[i] = (bf16)v;
    else ((_Float16 *)p)[i] = (_Float16)v;
}

// sums over the wave, the same on every lane
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

}  // namespace flex
