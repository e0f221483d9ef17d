// Pieces shared by the kernels of the microscaled formats (mx4: 4-bit floating point, ckpt8: 8-bit
// integers, one power of two for every 32 neighbours of a row): loads and stores of eight
// neighbouring floats of any type, the decoders, the activation functions.
#pragma once
#include <type_traits>

#include "lp_device.h"

namespace lp {

constexpr int kMx4Group = 256; // mx4 rows are padded to whole groups of this many elements

static inline size_t mx4_blocks(size_t cols) { return (cols + kMx4Group - 1) / kMx4Group * (kMx4Group / 32); }
static inline size_t ckpt8_blocks(size_t cols) { return (cols + 31) / 32; }

inline size_t dtype_size(lp_dtype t) { return t == LP_F32 ? 4 : 2; }
inline bool dtype_ok(lp_dtype t) { return (int)t >= 0 && (int)t <= 2; }
inline bool actfn_ok(lp_actfn f) { return (int)f >= 0 && (int)f <= 3; }
inline bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// a float tensor of the call: present, aligned to its elements, rows that do not overlap
inline bool floats_ok(const void *p, lp_dtype t, size_t cols, size_t ld) { return p && aligned_to(p, dtype_size(t)) && ld >= cols; }

// f(type tag) for the element type of t
template <typename F>
void with_type(lp_dtype t, F f)
{
    if (t == LP_F32) f((float *)nullptr);
    else if (t == LP_BF16) f((__bf16 *)nullptr);
    else f((_Float16 *)nullptr);
}

// x / d and x % d for 0 <= x < 2^31 with m = floor(2^32 / d) (d = 1: 2^32 - 1) from the host
__device__ __forceinline__ void piece_place(unsigned x, unsigned d, unsigned m, unsigned &q, unsigned &r)
{
    q = __umulhi(x, m);
    r = x - q * d;
    if (r >= d) {
        ++q;
        r -= d;
    }
}
inline unsigned piece_magic(unsigned d) { return d <= 1 ? 0xffffffffu : (unsigned)((1ull << 32) / d); }

// ------------------------------------------------------------------ eight neighbouring floats

typedef float v8f __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));

template <int W>
struct Floats {
    typedef float V __attribute__((ext_vector_type(W)));
};
// One load or store of the whole vector at the element's own alignment (the memory system takes 16 bytes at
// any address), or element by element where fewer than W exist.
template <int W, typename T>
__device__ __forceinline__ typename Floats<W>::V load_floats(const T *p, int n)
{
    typedef T V __attribute__((ext_vector_type(W), aligned(sizeof(T))));
    typename Floats<W>::V v = 0.0f;
    if (n >= W) {
        const V t = *reinterpret_cast<const V *>(p);
        v = __builtin_convertvector(t, typename Floats<W>::V);
    } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            if (j < n) v[j] = (float)p[j];
    }
    return v;
}
template <int W, typename T>
__device__ __forceinline__ void store_floats(T *p, int n, typename Floats<W>::V v)
{
    typedef T V __attribute__((ext_vector_type(W), aligned(sizeof(T))));
    const V t = __builtin_convertvector(v, V);
    if (n >= W) {
        *reinterpret_cast<V *>(p) = t;
    } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            if (j < n) p[j] = t[j];
    }
}
template <typename T>
__device__ __forceinline__ v8f load8(const T *p, int n) { return load_floats<8>(p, n); }
template <typename T>
__device__ __forceinline__ void store8(T *p, int n, v8f v) { store_floats<8>(p, n, v); }

// ------------------------------------------------------------- blocks of 32 in four neighbouring lanes

// largest of the four lanes that hold a block
__device__ __forceinline__ int block_max(int v)
{
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true)); // lanes 1 0 3 2
    return max(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true)); // lanes 2 3 0 1
}

// biased exponent of the block's largest finite magnitude
__device__ __forceinline__ int block_exponent(const v8f &v)
{
    int m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int b = (int)(__float_as_uint(v[j]) & 0x7fffffffu);
        m = max(m, b < 0x7f800000 ? b : 0);
    }
    return block_max(m) >> 23;
}

__device__ __forceinline__ int mx4_scale_byte(int exponent) { return min(max(exponent - 2, 2), 252); }

// ---------------------------------------------------------------------------- codes and values

__device__ __forceinline__ float power_of_byte(int e) { return __uint_as_float((unsigned)e << 23); } // 2^(e - 127), 1 <= e <= 254

// eight mx4 elements (one word of codes) times 2^(e - 127)
__device__ __forceinline__ v8f mx4_values(unsigned w, int e)
{
    const float s = power_of_byte(e);
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    return v8f{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// eight floats to one word of mx4 codes, nearest even, by the hardware's conversion (which divides by 2^(e - 127) and
// saturates); NaN becomes 0
__device__ __forceinline__ unsigned mx4_word(v8f v, int e)
{
    const float s = power_of_byte(e);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] == v[j] ? v[j] : 0.0f;
    unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
}

// eight ckpt8 elements (two words of codes) times 2^(e - 133)
__device__ __forceinline__ v8f ckpt8_values(v2u w, int e)
{
    const float s = power_of_byte(e - 6);
    v8f v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(signed char)(w[j >> 2] >> (8 * (j & 3))) * s;
    return v;
}

// ----------------------------------------------------------------------- activation functions

constexpr double kLog2E = 1.4426950408889634074;      // log2 e
constexpr double kGelu2C = 1.59576912160573071176;    // 2 sqrt(2 / pi)
constexpr double kGeluA = 0.044715;

// SiLU and GELU are h s(z), s the logistic function, z = h or 2 sqrt(2 / pi) (h + A h^3).  Beyond 200 (SiLU) and 20 (GELU) in
// magnitude s is 1 or 0 to all 32 bits, and the powers stay finite.
template <lp_actfn F>
__device__ __forceinline__ float within(float h)
{
    constexpr float far = F == LP_ACT_SILU ? 200.0f : 20.0f;
    return __builtin_amdgcn_fmed3f(h, -far, far);
}

struct Logistic {
    float s, t; // of z and of -z
};
// Both values are quotients of a = exp(-|z|), which cannot overflow: 1 / (1 + a), by the hardware's reciprocal and a Newton step, and a
// times that, so that neither cancels.
// FINE, for results of 32 bits: the argument times log2 e comes in two numbers.  The values are off by 6 half steps, and 3 |z| for the
// rounding of GELU's z.
// Otherwise it comes in one: 2 |z| + 6 half steps, GELU 4 |z| + 6, which is a hundredth of a half step of f16 or bfloat16 where
// these have a result.  8192 x 14336 bfloat16 kept with SiLU in 102 us and its gradient in 100, FINE 107 and 102; a product of
// 8192 x 4096 -> 14336 278, 296.  (In 32 bits there is no difference: memory takes as long.  Without the Newton step 99, 100 and 265, but
// of a tensor of 8192 x 14336 bfloat16 20887 results were rounded to the other side, nearly all of them at one input.)
template <lp_actfn F, bool FINE>
__device__ __forceinline__ Logistic logistic(float h)
{
    float u, low; // z log2 e: FINE, their sum
    if constexpr (FINE) {
        const float g = within<F>(h);
        if (F == LP_ACT_SILU) {
            u = g * (float)kLog2E;
            low = __builtin_fmaf(g, (float)kLog2E, -u);
            low = __builtin_fmaf(g, (float)(kLog2E - (double)(float)kLog2E), low);
        } else {
            const float p = __builtin_fmaf((float)(kGelu2C * kGeluA * kLog2E), g * g, (float)(kGelu2C * kLog2E));
            u = g * p;
            low = __builtin_fmaf(g, p, -u);
        }
    } else if (F == LP_ACT_SILU) {
        u = h * (float)kLog2E;
    } else {
        u = h * __builtin_fmaf((float)(kGelu2C * kGeluA * kLog2E), h * h, (float)(kGelu2C * kLog2E));
    }
    const bool negative = u < 0.0f;
    float a = __builtin_amdgcn_exp2f(-__builtin_fabsf(u)); // (0 below the normal numbers)
    if constexpr (FINE) a = __builtin_fmaf(a * (float)(1.0 / kLog2E), negative ? low : -low, a);
    const float d = 1.0f + a;
    float r = __builtin_amdgcn_rcpf(d);
    r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
    const float ar = a * r;
    return {negative ? ar : r, negative ? r : ar};
}

// The functions; -Inf is taken as a number far out, where the product is a (signed) zero.
template <lp_actfn F, bool FINE>
__device__ __forceinline__ float act_value(float h)
{
    if (F == LP_ACT_RELU) return h < 0.0f ? 0.0f : h;
    const float g = h < -1e30f ? -1e30f : h;
    return g * logistic<F, FINE>(g).s;
}

// d act / dh = s(z) (1 + h s(-z) dz/dh): 0 or 1 to all 32 bits where s is
template <lp_actfn F, bool FINE>
__device__ __forceinline__ float act_slope(float h)
{
    if (F == LP_ACT_RELU) return h > 0.0f ? 1.0f : 0.0f;
    const float g = within<F>(h);
    const Logistic l = logistic<F, FINE>(g);
    const float dz = F == LP_ACT_SILU ? 1.0f : (float)kGelu2C + (float)(3.0 * kGelu2C * kGeluA) * (g * g);
    return l.s * (1.0f + g * l.t * dz);
}

// act(v) on its way to a result of type T
template <typename T, typename V>
__device__ __forceinline__ V act_values(V v, lp_actfn f)
{
    constexpr bool FINE = std::is_same<T, float>::value;
    constexpr int N = sizeof(V) / sizeof(float);
    if (f == LP_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = act_value<LP_ACT_RELU, FINE>(v[j]);
    } else if (f == LP_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = act_value<LP_ACT_SILU, FINE>(v[j]);
    } else if (f == LP_ACT_GELU_TANH) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = act_value<LP_ACT_GELU_TANH, FINE>(v[j]);
    }
    return v;
}

// d times the slopes at h, on its way to a result of type T
template <typename T>
__device__ __forceinline__ v8f act_gradients(v8f d, v8f h, lp_actfn f)
{
    constexpr bool FINE = std::is_same<T, float>::value;
    if (f == LP_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= act_slope<LP_ACT_RELU, FINE>(h[j]);
    } else if (f == LP_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= act_slope<LP_ACT_SILU, FINE>(h[j]);
    } else if (f == LP_ACT_GELU_TANH) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= act_slope<LP_ACT_GELU_TANH, FINE>(h[j]);
    }
    return d;
}

// --------------------------------------------------------------- as called by the products' file

// brings rows x cols floats to mx4, nearest even (no arguments left to check)
void mx4_quantize_launch(const void *x, lp_dtype xt, size_t rows, size_t cols, size_t ldx, void *codes, void *scales, hipStream_t st);

} // namespace lp
