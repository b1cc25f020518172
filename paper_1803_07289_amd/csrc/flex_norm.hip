// Layer norm over the channels of every position, forward and backward.
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   with xh = (x - mean) rstd and h = g w:  grad_x = rstd (h - mean(h) - xh mean(h xh)),
//   grad_w = sum over positions of g xh, grad_b = sum of g.
// Sums and statistics are fp32; the mean square is taken about the mean (two passes), which loses nothing to cancellation.
#include "flex_elem.hpp"
#include <algorithm>

namespace flex {

// A wave for each position; channel c of position p of cloud b is x[b * C * N + p * ps + c * cs].
template <class T>
__global__ __launch_bounds__(256) void norm_fwd_kernel(const T *__restrict__ x, const void *w, const void *b, T *__restrict__ y,
                                                       float *mean_out, float *rstd_out, int64_t rows, int N, int C, int64_t ps,
                                                       int64_t cs, float eps, int pdtype)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int64_t base = row / N * ((int64_t)N * C) + row % N * ps;
    float sum = 0.f;
    for (int c = lane; c < C; c += 64) sum += to_f32(x[base + c * cs]);
    const float mean = wave_sum(sum) / (float)C;
    float sq = 0.f;
    for (int c = lane; c < C; c += 64) {
        const float d = to_f32(x[base + c * cs]) - mean;
        sq += d * d;
    }
    const float rstd = 1.f / sqrtf(wave_sum(sq) / (float)C + eps);
    for (int c = lane; c < C; c += 64) {
        const float v = (to_f32(x[base + c * cs]) - mean) * rstd;
        y[base + c * cs] = (T)(w ? v * load_param(w, pdtype, c) + load_param(b, pdtype, c) : v);
    }
    if (lane == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
}

template <class T>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const T *__restrict__ x, const void *w, const T *__restrict__ g,
                                                       const float *mean, const float *rstd, T *__restrict__ gx, int64_t rows,
                                                       int N, int C, int64_t ps, int64_t cs, int pdtype)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int64_t base = row / N * ((int64_t)N * C) + row % N * ps;
    const float m = mean[row], r = rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int c = lane; c < C; c += 64) {
        const float h = to_f32(g[base + c * cs]) * (w ? load_param(w, pdtype, c) : 1.f);
        s1 += h;
        s2 += h * ((to_f32(x[base + c * cs]) - m) * r);
    }
    s1 = wave_sum(s1) / (float)C;
    s2 = wave_sum(s2) / (float)C;
    for (int c = lane; c < C; c += 64) {
        const float h = to_f32(g[base + c * cs]) * (w ? load_param(w, pdtype, c) : 1.f);
        gx[base + c * cs] = (T)((h - s1 - (to_f32(x[base + c * cs]) - m) * r * s2) * r);
    }
}

// partials[slice][0 | 1][C]: a thread sums one channel over its slice of positions
template <class T>
__global__ __launch_bounds__(256) void norm_params_kernel(const T *__restrict__ x, const T *__restrict__ g, const float *mean,
                                                          const float *rstd, float *partials, int64_t rows, int64_t per, int N,
                                                          int C, int64_t ps, int64_t cs)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    float gw = 0.f, gb = 0.f;
    const int64_t end = min(rows, (int64_t)(blockIdx.y + 1) * per);
    for (int64_t row = (int64_t)blockIdx.y * per; row < end; ++row) {
        const int64_t at = row / N * ((int64_t)N * C) + row % N * ps + c * cs;
        const float v = to_f32(g[at]);
        gw += v * ((to_f32(x[at]) - mean[row]) * rstd[row]);
        gb += v;
    }
    partials[((int64_t)blockIdx.y * 2 + 0) * C + c] = gw;
    partials[((int64_t)blockIdx.y * 2 + 1) * C + c] = gb;
}

__global__ __launch_bounds__(256) void norm_params_sum_kernel(const float *__restrict__ partials, int slices, void *gw, void *gb,
                                                              int C, int pdtype)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    float a = 0.f, b = 0.f;
    for (int i = 0; i < slices; ++i) {
        a += partials[((int64_t)i * 2 + 0) * C + c];
        b += partials[((int64_t)i * 2 + 1) * C + c];
    }
    store_param(gw, pdtype, c, a);
    store_param(gb, pdtype, c, b);
}

static int norm_slices(int64_t rows) { return (int)std::min<int64_t>(256, cdiv64(rows, 64)); }

}  // namespace flex

using namespace flex;

static bool norm_sizes_ok(int B, int N, int C, int layout, int dtype, int param_dtype)
{
    return B > 0 && N > 0 && C > 0 && (int64_t)B * N < ((int64_t)1 << 31) && (layout == FLEX_LAYOUT_BCN || layout == FLEX_LAYOUT_BNC) &&
           dtype_ok(dtype) && (param_dtype == FLEX_F32 || param_dtype == dtype);
}

extern "C" {

int flexnorm_fwd(const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd, int B, int N, int C,
                 float eps, int dtype, int param_dtype, int layout, void *stream)
{
    if (!x || !y || (weight == nullptr) != (bias == nullptr)) return FLEX_ERR_NULL;
    if (!norm_sizes_ok(B, N, C, layout, dtype, param_dtype) || !(eps >= 0.f) || x == y) return FLEX_ERR_SHAPE;
    const int64_t rows = (int64_t)B * N, ps = layout == FLEX_LAYOUT_BCN ? 1 : C, cs = layout == FLEX_LAYOUT_BCN ? N : 1;
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        hipLaunchKernelGGL(norm_fwd_kernel<T>, dim3((unsigned)cdiv64(rows, 4)), dim3(256), 0, (hipStream_t)stream, (const T *)x,
                           weight, bias, (T *)y, mean, rstd, rows, N, C, ps, cs, eps, param_dtype);
        return hipGetLastError();
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

size_t flexnorm_bwd_workspace_bytes(int B, int N, int C, int dtype, int layout)
{
    if (!norm_sizes_ok(B, N, C, layout, dtype, dtype)) return 0;
    return align256((size_t)norm_slices((int64_t)B * N) * 2 * C * sizeof(float));
}

int flexnorm_bwd(const void *x, const void *weight, const void *grad_out, const float *mean, const float *rstd, void *grad_x,
                 void *grad_weight, void *grad_bias, int B, int N, int C, int dtype, int param_dtype, int layout,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !grad_out || !mean || !rstd || (grad_weight == nullptr) != (grad_bias == nullptr) || (!grad_x && !grad_weight))
        return FLEX_ERR_NULL;
    if (!norm_sizes_ok(B, N, C, layout, dtype, param_dtype) || grad_x == x || grad_x == grad_out) return FLEX_ERR_SHAPE;
    if (grad_weight && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < flexnorm_bwd_workspace_bytes(B, N, C, dtype, layout)))
        return FLEX_ERR_WORKSPACE;
    const int64_t rows = (int64_t)B * N, ps = layout == FLEX_LAYOUT_BCN ? 1 : C, cs = layout == FLEX_LAYOUT_BCN ? N : 1;
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        if (grad_x)
            hipLaunchKernelGGL(norm_bwd_kernel<T>, dim3((unsigned)cdiv64(rows, 4)), dim3(256), 0, s, (const T *)x, weight,
                               (const T *)grad_out, mean, rstd, (T *)grad_x, rows, N, C, ps, cs, param_dtype);
        if (grad_weight) {
            const int slices = norm_slices(rows);
            hipLaunchKernelGGL(norm_params_kernel<T>, dim3((unsigned)((C + 255) / 256), (unsigned)slices), dim3(256), 0, s,
                               (const T *)x, (const T *)grad_out, mean, rstd, (float *)workspace, rows, cdiv64(rows, slices), N, C, ps, cs);
            hipLaunchKernelGGL(norm_params_sum_kernel, dim3((unsigned)((C + 255) / 256)), dim3(256), 0, s,
                               (const float *)workspace, slices, grad_weight, grad_bias, C, param_dtype);
        }
        return hipGetLastError();
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

}  // extern "C"
