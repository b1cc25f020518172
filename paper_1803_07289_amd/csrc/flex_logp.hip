// Log probabilities of given classes, entropy, log-sum-exp and the best alternatives of every position's C scores, and the
// gradient of the scores.
//   m = max x, s = sum exp(x - m), u = sum exp(x - m) (x - m):  lse = m + ln s,  logp = x_t - m - ln s,  H = ln s - u / s
//   p = exp(x - lse):  grad_x = grad_logp ([c = t] - p) - grad_H p (x - lse + H)
// A score of -inf has p = 0 and no share of anything; positions whose target is no class are ignored (outputs zero, no
// alternatives, gradient zero, scores not looked at); one without any score above -inf has logp = lse = -inf, H = 0.
#include "flex_elem.hpp"

namespace flex {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float MASKED = -1e5f;       // stands for x - m = -inf where it is multiplied by exp(x - m) = 0

struct LogpArgs {
    const int32_t *target;
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_class;
    int64_t rows, bs, ps, cs;         // positions; element strides: cloud, position, class
    int N, C, top, bcn;
};

template <class T>
__global__ __launch_bounds__(256) void logp_fwd_kernel(const T *__restrict__ x, LogpArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.rows) return;
    const int64_t b = row / a.N, n = row % a.N;
    const T *at = x + b * a.bs + n * a.ps;
    const int64_t top_at = a.bcn ? b * a.top * a.N + n : row * a.top, top_step = a.bcn ? a.N : 1;
    const int t = a.target ? a.target[row] : 0;
    if (a.target && (t < 0 || t >= a.C)) {
        if (lane == 0) a.logp[row] = a.entropy[row] = a.lse[row] = 0.f;
        if (lane < a.top) {
            a.top_logp[top_at + lane * top_step] = -INFINITY;
            a.top_class[top_at + lane * top_step] = -1;
        }
        return;
    }
    float m = -INFINITY, s = 0.f, u = 0.f;
    for (int c = lane; c < a.C; c += 64) m = fmaxf(m, to_f32(at[c * a.cs]));
    m = wave_max(m);
    if (m == -INFINITY) m = 0.f;
    for (int c = lane; c < a.C; c += 64) {
        const float z = to_f32(at[c * a.cs]) - m, e = __builtin_amdgcn_exp2f(z * LOG2E);
        s += e;
        u += e * fmaxf(z, MASKED);
    }
    s = wave_sum(s);
    u = wave_sum(u);
    const float log_s = logf(s);
    if (lane == 0) {
        if (a.target) a.logp[row] = s == 0.f ? -INFINITY : to_f32(at[t * a.cs]) - m - log_s;
        a.entropy[row] = s == 0.f ? 0.f : log_s - u / s;
        a.lse[row] = m + log_s;
    }
    float last = INFINITY;
    int last_c = -1;
    for (int k = 0; k < a.top; ++k) {       // the best of those behind the last one found
        float best = -INFINITY;
        int best_c = INT_MAX;
        for (int c = lane; c < a.C; c += 64) {
            const float v = to_f32(at[c * a.cs]);
            if (v > best && (v < last || (v == last && c > last_c))) { best = v; best_c = c; }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float v = __shfl_xor(best, o);
            const int c = __shfl_xor(best_c, o);
            if (v > best || (v == best && c < best_c)) { best = v; best_c = c; }
        }
        last = best;
        last_c = best_c;
        if (lane == 0) {
            a.top_logp[top_at + k * top_step] = best == -INFINITY ? -INFINITY : best - m - log_s;
            a.top_class[top_at + k * top_step] = best == -INFINITY ? -1 : best_c;
        }
    }
}

struct LogpBwdArgs {
    const int32_t *target;
    const float *lse, *entropy, *grad_logp, *grad_entropy;
    int64_t rows, bs, ps, cs, gbs, gps, gcs;     // strides of the scores and of their gradient
    int N, C;
};

template <class T>
__global__ __launch_bounds__(256) void logp_bwd_kernel(const T *x, T *gx, LogpBwdArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.rows) return;
    const int64_t b = row / a.N, n = row % a.N;
    const T *at = x + b * a.bs + n * a.ps;
    T *to = gx + b * a.gbs + n * a.gps;
    const int t = a.target ? a.target[row] : -1;
    const float lse = a.lse[row];
    if ((a.target && (t < 0 || t >= a.C)) || lse == -INFINITY) {
        for (int c = lane; c < a.C; c += 64) to[c * a.gcs] = (T)0.f;
        return;
    }
    const float gl = a.target && a.grad_logp ? a.grad_logp[row] : 0.f, gh = a.grad_entropy ? a.grad_entropy[row] : 0.f;
    const float h = a.grad_entropy ? a.entropy[row] : 0.f;
    for (int c = lane; c < a.C; c += 64) {
        const float lp = to_f32(at[c * a.cs]) - lse, p = __builtin_amdgcn_exp2f(lp * LOG2E);
        const float v = -p * (gl + gh * (fmaxf(lp, MASKED) + h));
        to[c * a.gcs] = (T)(c == t ? v + gl : v);
    }
}

}  // namespace flex

using namespace flex;

static bool logp_sizes_ok(int B, int N, int C, int64_t row_stride, int dtype, int layout)
{
    return B > 0 && N > 0 && C > 0 && C <= FLEX_LOGP_MAX_CLASSES && (int64_t)B * N < ((int64_t)1 << 31) &&
           (layout == FLEX_LAYOUT_BCN || layout == FLEX_LAYOUT_BNC) && dtype_ok(dtype) &&
           row_stride >= (layout == FLEX_LAYOUT_BCN ? N : C) && row_stride < ((int64_t)1 << 31);
}

extern "C" {

size_t flexlogp_fwd_workspace_bytes(int B, int N, int C, int top, int dtype, int layout)
{
    if (!logp_sizes_ok(B, N, C, layout == FLEX_LAYOUT_BCN ? N : C, dtype, layout) || top < 0 || top > FLEX_LOGP_MAX_TOP || top > C) return 0;
    return 256;
}

int flexlogp_fwd(const void *logits, const int32_t *target, float *logp, float *entropy, float *lse, float *top_logp,
                 int32_t *top_class, int B, int N, int C, int top, int64_t row_stride, int dtype, int layout,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    if (!logits || !entropy || !lse || (target == nullptr) != (logp == nullptr)) return FLEX_ERR_NULL;
    if (top > 0 && (!top_logp || !top_class)) return FLEX_ERR_NULL;
    if (!logp_sizes_ok(B, N, C, row_stride, dtype, layout) || top < 0 || top > FLEX_LOGP_MAX_TOP || top > C) return FLEX_ERR_SHAPE;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < flexlogp_fwd_workspace_bytes(B, N, C, top, dtype, layout))
        return FLEX_ERR_WORKSPACE;
    const bool bcn = layout == FLEX_LAYOUT_BCN;
    LogpArgs a{target, logp, entropy, lse, top_logp, top_class, (int64_t)B * N, (bcn ? C : N) * row_stride,
               bcn ? 1 : row_stride, bcn ? row_stride : 1, N, C, top, bcn};
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        hipLaunchKernelGGL(logp_fwd_kernel<T>, dim3((unsigned)cdiv64(a.rows, 4)), dim3(256), 0, (hipStream_t)stream, (const T *)logits, a);
        return hipGetLastError();
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
    if (logits == grad_logits && row_stride != grad_row_stride) return FLEX_ERR_SHAPE;
    const bool bcn = layout == FLEX_LAYOUT_BCN;
    LogpBwdArgs a{target, lse, entropy, grad_logp, grad_entropy, (int64_t)B * N,
                  (bcn ? C : N) * row_stride, bcn ? 1 : row_stride, bcn ? row_stride : 1,
                  (bcn ? C : N) * grad_row_stride, bcn ? 1 : grad_row_stride, bcn ? grad_row_stride : 1, N, C};
    const hipError_t e = with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        hipLaunchKernelGGL(logp_bwd_kernel<T>, dim3((unsigned)cdiv64(a.rows, 4)), dim3(256), 0, (hipStream_t)stream, (const T *)logits,
                           (T *)grad_logits, a);
        return hipGetLastError();
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

}  // extern "C"
