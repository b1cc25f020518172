// One AdamW step over a list of parameter tensors, with states in fp32 or in 8 bits.
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  g the gradient times grad_scale
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
// States in 8 bits: e4m3 values, and an e8m0 byte (a power of two) for every 32 of them that brings the largest to (224, 448].
// What a step changes in a state, a thousandth of it for v, is far below the spacing of e4m3, so that rounding to nearest would
// never move it: states are rounded at random, with probabilities that make the mean exact.  v is kept by its root, which spreads
// its range over twice the exponents; the choice between two roots is made so that the square has the right mean, and a v
// above zero is never stored as zero, which would leave eps alone under m.  The random bits are a hash of (seed, step,
// tensor, element).  What leads to a state is rounded operation by operation (no fused multiply-adds but where they are exact), a block's
// exponent is that of a correctly rounded root, and a code hardly depends on its root's last bit (see second_code): states are the same
// bits wherever the formulas are evaluated in fp32, but for a random number of 0 within an ulp of a code's border.
#include "flex_elem.hpp"
#include <algorithm>
#include <math.h>
#include <string.h>

#pragma clang fp contract(off)

namespace flex {

constexpr int ADAMW_CHUNK = 2048;           // elements that a workgroup takes: 256 threads x 8
constexpr int ADAMW_BATCH = 32;             // tensors that one launch enters in the plan
constexpr int ADAMW_GRADS = 448;            // gradient pointers that one launch takes

struct AdamwHeader {
    double beta1, beta2, beta1_t, beta2_t;  // the powers: of the steps done
    int64_t steps;
    float b1, b2, a1, a2, eps;              // a1 = 1 - b1, a2 = 1 - b2
    uint32_t seed;
    // what adamw_begin_kernel leaves for the step
    float step_size, rsqrt_c2, grad_scale;
    int32_t active;
    double lr;
    uint32_t key;
    uint32_t pad[3];
};
struct AdamwTensor {
    void *p, *m, *v;
    uint8_t *m_scale, *v_scale;
    void *copy;
    uint32_t count, first;                  // elements, its first chunk
    double decay;
};
static_assert(sizeof(AdamwHeader) <= 256 && sizeof(AdamwTensor) == 64, "");

// The plan in device memory: header, tensors, their gradients, the tensor of every chunk.
struct AdamwPlan {
    AdamwHeader *header;
    AdamwTensor *tensors;
    const void **grads;
    uint32_t *owner;
};
static size_t adamw_owner_at(int n) { return 256 + align256(sizeof(AdamwTensor) * (size_t)n) + align256(sizeof(void *) * (size_t)n); }
static AdamwPlan adamw_plan(void *plan, int n)
{
    char *at = (char *)plan;
    return AdamwPlan{(AdamwHeader *)at, (AdamwTensor *)(at + 256), (const void **)(at + 256 + align256(sizeof(AdamwTensor) * (size_t)n)),
                     (uint32_t *)(at + adamw_owner_at(n))};
}

struct AdamwEntries {
    AdamwTensor t[ADAMW_BATCH];
};

__global__ __launch_bounds__(256) void adamw_plan_kernel(AdamwPlan plan, AdamwHeader header, AdamwEntries e, int at)
{
    const AdamwTensor t = e.t[blockIdx.x];
    if (threadIdx.x == 0) {
        plan.tensors[at + blockIdx.x] = t;
        if (at == 0 && blockIdx.x == 0) *plan.header = header;
    }
    const uint32_t chunks = (t.count + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
    for (uint32_t i = threadIdx.x; i < chunks; i += 256) plan.owner[t.first + i] = (uint32_t)(at + blockIdx.x);
}

__device__ __forceinline__ uint32_t adamw_mix(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;      // the fractions of sqrt(2) and sqrt(3)
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

struct AdamwGrads {
    const void *g[ADAMW_GRADS];
};

// Enters the gradients' addresses and, in its first launch, begins the step: its number, its powers, what they make of lr.
// A grad_scale that is not finite: no step.
__global__ __launch_bounds__(ADAMW_GRADS) void adamw_begin_kernel(AdamwPlan plan, AdamwGrads g, int at, int n, double lr,
                                                                   const float *lr_dev, const float *grad_scale)
{
    if ((int)threadIdx.x < n) plan.grads[at + threadIdx.x] = g.g[threadIdx.x];
    if (at != 0 || threadIdx.x != 0) return;
    AdamwHeader &h = *plan.header;
    const float scale = grad_scale ? *grad_scale : 1.f;
    h.active = isfinite(scale);
    if (!h.active) return;
    if (lr_dev) lr = (double)*lr_dev;
    h.grad_scale = scale;
    h.steps += 1;
    h.beta1_t *= h.beta1;
    h.beta2_t *= h.beta2;
    h.lr = lr;
    h.step_size = (float)(lr / (1.0 - h.beta1_t));
    h.rsqrt_c2 = (float)(1.0 / sqrt(1.0 - h.beta2_t));
    h.key = adamw_mix(h.seed + (uint32_t)h.steps);
}

// ---- states in 8 bits --------------------------------------------------------------------------------------------------

__device__ __forceinline__ float power2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// The largest of a block's magnitudes: 8 to a lane, four lanes.
__device__ __forceinline__ float block_max(const float (&x)[8])
{
    float m = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
    return lanes_max<4>(m);
}

// The exponent that brings `largest` to (224, 448]; within [-100, 120], so that the powers below stay in fp32.
__device__ __forceinline__ int block_exponent(float largest)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, largest);
    const int e = (int)(bits >> 23) - 135 + ((bits & 0x7FFFFFu) > 0x600000u);
    return min(max(e, -100), 120);
}

// The same of the root of a normal v: half of v's exponent, and one more where the root is above 1.75 times a power of two, that is v above
// 3.0625 times its square (its rounded root is, exactly then).
__device__ __forceinline__ int root_exponent(float v)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    return (int)(((bits >> 23) + 1) >> 1) - 72 + ((bits & 0xFFFFFFu) - 0x440001u < 0x3BFFFFu);
}

// The state that lies up or down from `value` (a first moment times its block's scale) by 16 random bits in the upper half of r: the
// hardware's conversion, which adds them below the last bit kept, subnormals too.  Into byte i of word.
template <int i>
__device__ __forceinline__ uint32_t first_code(float value, uint32_t r, uint32_t word)
{
    return (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(value, (int)r, (int)word, i);
}
// The state of a second moment v, its root and the scale of its block: in steps of e4m3 at the root's exponent, n below it and n + 1 above
// it, their squares n^2 and n^2 + 2 n + 1; up where the random share of the difference lies below v.  (A root that is an ulp too small or
// too large at n's border makes n one less or more, and `up` always or never true: the same code.)
__device__ __forceinline__ uint32_t second_code(float v, float root, float down, uint32_t r16)
{
    const float y = root * down;
    const uint32_t bits = __builtin_bit_cast(uint32_t, y), power = max(bits & 0x7F800000u, 0x3C800000u);      // 2^-6 and up
    const float f = __builtin_bit_cast(float, 0x80800000u - power), f2 = f * down;                              // 8 / power
    const float n = floorf(y * f), w = v * f2 * f2;
    const bool up = (float)r16 * __builtin_fmaf(n, 0x1p-15f, 0x1p-16f) < __builtin_fmaf(-n, n, w);              // (both products exact)
    const int code = (int)((power >> 20) + (uint32_t)n) - 968 + (up ? 1 : 0);
    return (uint32_t)min(max(code, (int)min(__builtin_bit_cast(uint32_t, v), 1u)), 126);       // (the largest finite one; above zero, not zero)
}

__device__ __forceinline__ void store_codes(uint8_t *codes, uint8_t *scale, const uint32_t (&word)[2], int e, int64_t at, int64_t count)
{
    if (at + 8 <= count) {
        typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(1)));
        *(u2 *)(codes + at) = u2{word[0], word[1]};
    } else
        for (int i = 0; i < 8; ++i)
            if (at + i < count) codes[at + i] = (uint8_t)(word[i / 4] >> (8 * (i & 3)));
    if ((threadIdx.x & 3) == 0 && at < count) scale[at / 32] = (uint8_t)(e + 127);
}

__device__ __forceinline__ void load_codes(const uint8_t *codes, const uint8_t *scale, float (&x)[8], int64_t at, int64_t count)
{
    uint32_t v[2] = {0, 0};
    if (at + 8 <= count) {
        typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(1)));
        const u2 w = *(const u2 *)(codes + at);
        v[0] = w[0];
        v[1] = w[1];
    } else
        for (int i = 0; i < 8; ++i)
            if (at + i < count) v[i / 4] |= (uint32_t)codes[at + i] << (8 * (i & 3));
    const float s = at < count ? power2((int)scale[at / 32] - 127) : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], true);
        x[4 * i] = lo[0] * s;
        x[4 * i + 1] = lo[1] * s;
        x[4 * i + 2] = hi[0] * s;
        x[4 * i + 3] = hi[1] * s;
    }
}

// Elements at .. at + 8 of an array of count, zeros behind it.
template <class T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8], int64_t at, int64_t count)
{
    typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    if (at + 8 <= count) {
        const V v = *(const V *)(p + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f32(v[i]);
    } else
        for (int i = 0; i < 8; ++i) x[i] = at + i < count ? to_f32(p[at + i]) : 0.f;
}
template <class T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8], int64_t at, int64_t count)
{
    typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    if (at + 8 <= count) {
        V v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
        *(V *)(p + at) = v;
    } else
        for (int i = 0; i < 8; ++i)
            if (at + i < count) p[at + i] = (T)x[i];
}

// A workgroup to 2048 elements of a tensor, eight to a thread, which makes every access 16 or 8 bytes a lane and a scale's 32 elements
// four lanes.  Memory bounds it: 5.4 TB/s with states in 32 bits and a copy (28 bytes an element, 191M elements: 998 us; at the rate of a copy 869),
// 5.6 with states in 8 (10.1 bytes, 428M elements in bf16: 775 us, 704), where the vector unit has some 60 operations an element to hide.  Larger
// pieces, two pieces a workgroup and accesses past the caches measured the same or worse.
// Roots and quotients are the hardware's approximations, an ulp each: the update is lr times them, an ulp of it no ulp of p.  Of a
// subnormal v the hardware's root is 0; that is told from eps, or in a state of 8 bits from the values beside it, only below the two bounds
// here, and there the root is the full one.
constexpr float ROOT_BESIDE_EPS = 0x1p-38f;         // 2^-63 of a subnormal's root is 2^-25 of it
constexpr float BLOCK_OF_SUBNORMALS = 0x1p-88f;     // the largest v whose block has codes for the root of a subnormal one: 448^2 2^18 2^-126 at most
template <class P, class G, int BITS>
__global__ __launch_bounds__(256) void adamw_step_kernel(AdamwPlan plan, int copy_dtype)
{
    const AdamwHeader &h = *plan.header;
    if (!h.active) return;
    const uint32_t k = plan.owner[blockIdx.x];
    const AdamwTensor t = plan.tensors[k];
    const G *grad = (const G *)plan.grads[k];
    if (!grad) return;                       // a tensor without a gradient keeps its values and states
    const int64_t at = (int64_t)(blockIdx.x - t.first) * ADAMW_CHUNK + threadIdx.x * 8;
    float p[8], g[8], m[8], v[8], root[8];
    load8((const P *)t.p, p, at, t.count);
    load8(grad, g, at, t.count);
    if (BITS == 32) {
        load8((const float *)t.m, m, at, t.count);
        load8((const float *)t.v, v, at, t.count);
    } else {
        load_codes((const uint8_t *)t.m, t.m_scale, m, at, t.count);
        load_codes((const uint8_t *)t.v, t.v_scale, v, at, t.count);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= v[i];
    }
    const float keep = (float)(1.0 - h.lr * t.decay);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        g[i] *= h.grad_scale;
        m[i] = m[i] * h.b1 + g[i] * h.a1;
        v[i] = v[i] * h.b2 + g[i] * g[i] * h.a2;
    }
    bool full_roots = h.eps < h.rsqrt_c2 * ROOT_BESIDE_EPS;
    int ev = 0;
    if (BITS == 8) {
        const float largest = block_max(v);
        full_roots |= __any(largest > 0.f && largest < BLOCK_OF_SUBNORMALS);
        ev = full_roots ? block_exponent(sqrtf(largest)) : largest > 0.f ? root_exponent(largest) : block_exponent(0.f);
    }
    if (__builtin_expect(full_roots, 0))
#pragma unroll
        for (int i = 0; i < 8; ++i) root[i] = sqrtf(v[i]);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) root[i] = __builtin_amdgcn_sqrtf(v[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float by = m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(root[i], h.rsqrt_c2, h.eps));
        p[i] = __builtin_fmaf(-by, h.step_size, p[i] * keep);
    }
    store8((P *)t.p, p, at, t.count);
    if (t.copy) {
        if (copy_dtype == FLEX_BF16) store8((bf16 *)t.copy, p, at, t.count);
        else store8((_Float16 *)t.copy, p, at, t.count);
    }
    if (BITS == 32) {
        store8((float *)t.m, m, at, t.count);
        store8((float *)t.v, v, at, t.count);
        return;
    }
    const uint32_t key = adamw_mix(h.key + k);
    const int em = block_exponent(block_max(m));
    const float down_m = power2(-em), down_v = power2(-ev);
    uint32_t cm[2] = {0, 0}, cv[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = adamw_mix((uint32_t)at + i + key);
        uint32_t &word = cm[i / 4];
        const float y = m[i] * down_m;
        word = (i & 3) == 0 ? first_code<0>(y, r << 16, word) : (i & 3) == 1 ? first_code<1>(y, r << 16, word)
             : (i & 3) == 2 ? first_code<2>(y, r << 16, word) : first_code<3>(y, r << 16, word);
        cv[i / 4] |= second_code(v[i], root[i], down_v, r >> 16) << (8 * (i & 3));
    }
    store_codes((uint8_t *)t.m, t.m_scale, cm, em, at, t.count);
    store_codes((uint8_t *)t.v, t.v_scale, cv, ev, at, t.count);
}

}  // namespace flex

using namespace flex;

static bool adamw_list_ok(const flex_adamw_tensor *t, int n, int64_t *chunks)
{
    int64_t c = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].count < 0 || t[i].count >= ((int64_t)1 << 31)) return false;
        c += cdiv64(t[i].count, ADAMW_CHUNK);
    }
    *chunks = c;
    return one_launch(c * 256);
}

extern "C" {

size_t flexadamw_plan_bytes(const flex_adamw_tensor *tensors, int n)
{
    int64_t chunks;
    if (!tensors || n <= 0 || n > (1 << 20) || !adamw_list_ok(tensors, n, &chunks)) return 0;
    return adamw_owner_at(n) + align256(sizeof(uint32_t) * (size_t)chunks);
}

int flexadamw_plan_build(const flex_adamw_tensor *tensors, int n, int param_dtype, int state_bits, int copy_dtype, double beta1,
                         double beta2, double eps, int64_t steps, uint32_t seed, void *plan, size_t plan_bytes, flex_adamw *out,
                         void *stream)
{
    if (!tensors || !plan || !out) return FLEX_ERR_NULL;
    const size_t need = flexadamw_plan_bytes(tensors, n);
    if (need == 0 || !dtype_ok(param_dtype) || (state_bits != 8 && state_bits != 32) || (copy_dtype != FLEX_BF16 && copy_dtype != FLEX_F16) ||
        !(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.) || !((float)eps >= 1.17549435e-38f) || steps < 0) return FLEX_ERR_SHAPE;
    for (int i = 0; i < n; ++i)
        if (tensors[i].count > 0 && (!tensors[i].param || !tensors[i].exp_avg || !tensors[i].exp_avg_sq ||
                                     (state_bits == 8 && (!tensors[i].avg_scale || !tensors[i].avg_sq_scale)))) return FLEX_ERR_NULL;
    if (((uintptr_t)plan & 255) || plan_bytes < need) return FLEX_ERR_WORKSPACE;
    AdamwHeader h{};
    h.beta1 = beta1;
    h.beta2 = beta2;
    h.beta1_t = pow(beta1, (double)steps);
    h.beta2_t = pow(beta2, (double)steps);
    h.steps = steps;
    h.b1 = (float)beta1;
    h.b2 = (float)beta2;
    h.a1 = (float)(1. - beta1);
    h.a2 = (float)(1. - beta2);
    h.eps = (float)eps;
    h.seed = seed;
    const AdamwPlan p = adamw_plan(plan, n);
    uint32_t chunk = 0;
    for (int at = 0; at < n; at += ADAMW_BATCH) {
        AdamwEntries e{};
        const int many = std::min(ADAMW_BATCH, n - at);
        for (int i = 0; i < many; ++i) {
            const flex_adamw_tensor &t = tensors[at + i];
            e.t[i] = AdamwTensor{t.param, t.exp_avg, t.exp_avg_sq, t.avg_scale, t.avg_sq_scale, t.copy, (uint32_t)t.count, chunk, t.weight_decay};
            chunk += (uint32_t)cdiv64(t.count, ADAMW_CHUNK);
        }
        hipLaunchKernelGGL(adamw_plan_kernel, dim3((unsigned)many), dim3(256), 0, (hipStream_t)stream, p, h, e, at);
    }
    if (hipGetLastError() != hipSuccess) return FLEX_ERR_HIP;
    *out = flex_adamw{plan, (int64_t)chunk, n, param_dtype, state_bits, copy_dtype};
    return FLEX_OK;
}

int flexadamw_step(const flex_adamw *adamw, const void *const *grads, int n, int grad_dtype, double lr, const float *lr_dev,
                   const float *grad_scale, void *stream)
{
    if (!adamw || !adamw->plan || !grads) return FLEX_ERR_NULL;
    if (n != adamw->tensors || n <= 0 || !dtype_ok(grad_dtype) || !dtype_ok(adamw->param_dtype) ||
        (adamw->state_bits != 8 && adamw->state_bits != 32) || adamw->chunks < 0 || !one_launch(adamw->chunks * 256) || !isfinite(lr))
        return FLEX_ERR_SHAPE;
    const AdamwPlan p = adamw_plan(adamw->plan, n);
    const hipStream_t s = (hipStream_t)stream;
    for (int at = 0; at < n; at += ADAMW_GRADS) {
        AdamwGrads g;
        const int many = std::min(ADAMW_GRADS, n - at);
        memcpy(g.g, grads + at, sizeof(void *) * (size_t)many);
        memset(g.g + many, 0, sizeof(void *) * (size_t)(ADAMW_GRADS - many));
        hipLaunchKernelGGL(adamw_begin_kernel, dim3(1), dim3(ADAMW_GRADS), 0, s, p, g, at, many, lr, lr_dev, grad_scale);
    }
    if (adamw->chunks == 0) return hipGetLastError() == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
    const dim3 grid((unsigned)adamw->chunks), wg(256);
    const hipError_t e = with_dtype(adamw->param_dtype, [&](auto pt) {
        return with_dtype(grad_dtype, [&](auto gt) {
            typedef decltype(pt) P;
            typedef decltype(gt) G;
            if (adamw->state_bits == 32) hipLaunchKernelGGL((adamw_step_kernel<P, G, 32>), grid, wg, 0, s, p, adamw->copy_dtype);
            else hipLaunchKernelGGL((adamw_step_kernel<P, G, 8>), grid, wg, 0, s, p, adamw->copy_dtype);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? FLEX_OK : FLEX_ERR_HIP;
}

}  // extern "C"
