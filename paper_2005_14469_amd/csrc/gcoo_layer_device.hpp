// What the kernels of a sparse layer share: elements of the three types, activations and their slopes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gcoo.h"

namespace gcoo {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <typename T> __device__ __forceinline__ float widen(T x) { return (float)x; }
template <typename T> __device__ __forceinline__ T narrow(float x) { return (T)x; }        // to nearest even

// f(T) for the element type `type`.
template <typename F>
auto with_type(int type, F&& f)
{
    if (type == GCOO_BF16) return f(bf16_t{});
    if (type == GCOO_F16) return f(f16_t{});
    return f(float{});
}

// exp(x + more) for x <= 0, `more` a remainder that x is too coarse to hold: the instruction's power of two, off by a unit in the last place, times what the exponent loses by rounding; 0 below 2^-126, where
// the instruction has no numbers.  (With the library's expf, which has them, and a quotient the product with gelu, 1777 x 2301, 3 %, N = 1117, fp32, took 24.3 us, so 23.9.)
__device__ __forceinline__ float exp_below(float x, float more = 0.0f)
{
    constexpr float hi = 1.44269502f, lo = 1.92596299e-8f, ln2 = 0.693147182f;              // hi + lo = 1 / ln 2
    const float c = fmaxf(x, -200.0f), h = c * hi, e = __builtin_amdgcn_exp2f(h);
    return __builtin_fmaf(e, __builtin_fmaf(ln2, __builtin_fmaf(c, lo, __builtin_fmaf(c, hi, -h)), more), e);
}
// 1 / (x + more) for x >= 1, `more` what x has lost by rounding: the instruction's and one step of Newton's, off by little more than half a unit in the last place.
__device__ __forceinline__ float reciprocal(float x, float more = 0.0f)
{
    const float r = __builtin_amdgcn_rcpf(x);
    return __builtin_fmaf(__builtin_fmaf(-more, r, __builtin_fmaf(-x, r, 1.0f)), r, r);
}
// s(x) = 1 / (1 + exp(-x)) and s(-x) of x >= 0.  In fp32 off by 8 2^-24; for types of 2 bytes by single instructions, (1.5 x + 2) 2^-24.
struct Logistic { float s, tail; };
template <typename T>
__device__ __forceinline__ Logistic logistic(float x)
{
    if constexpr (sizeof(T) == 2) {
        const float e = __expf(-x), s = __builtin_amdgcn_rcpf(1.0f + e);
        return {s, e * s};
    }
    const float e = exp_below(-x), s = reciprocal(1.0f + e);
    return {s, e * s};
}
constexpr float kGeluA = 0.7978845608028654f, kGeluB = 0.044715f, kDensity0 = 0.3989422804014327f;

// silu and gelu_tanh are z s(x), x = q z + r z^3: max(z, 0) - |z| s(-|x|), whose slope is w for negative z and 1 - w else, w = s(-|x|) (1 - |z| s(|x|) (q + 3 r z^2)).  s(-|x|) as a difference would have lost what the factors
// beside it need.
template <bool CUBIC> struct Gate {
    static constexpr float q = CUBIC ? 2.0f * kGeluA : 1.0f, r = CUBIC ? 2.0f * kGeluA * kGeluB : 0.0f;
    static constexpr float most = CUBIC ? 16.0f : 256.0f;             // of |z|: beyond, the exponential is 0
};
template <typename T, bool CUBIC>
__device__ __forceinline__ float gate(float z)
{
    typedef Gate<CUBIC> G;
    if constexpr (sizeof(T) == 2) {
        const float x = CUBIC ? 2.0f * kGeluA * (z + kGeluB * z * z * z) : z;
        return z * __builtin_amdgcn_rcpf(1.0f + __expf(-x));
    }
    const float a = fabsf(fminf(z, G::most));                         // (so it is infinite where z is, and, as z s(x), no number where z is -infinite)
    return __builtin_fmaf(-a, logistic<T>(CUBIC ? a * (G::q + G::r * (a * a)) : a).tail, z <= 0.0f ? 0.0f : z);
}
template <typename T, bool CUBIC>
__device__ __forceinline__ float gate_slope(float z)
{
    typedef Gate<CUBIC> G;
    const float a = fminf(fabsf(z), G::most), a2 = a * a;
    const Logistic l = logistic<T>(CUBIC ? a * (G::q + G::r * a2) : a);
    const float w = l.tail * __builtin_fmaf(-a * l.s, CUBIC ? G::q + 3.0f * G::r * a2 : 1.0f, 1.0f);
    return z != z ? z : (z < 0.0f ? w : 1.0f - w);
}

// Phi(-a) / exp(-a^2 / 2) and exp(-a^2 / 2), a = |z| (where it is more than 16 the exponential is 0, and is so where it is no normal number: what follows would go on with the few bits that are left of it): from these two
// come Phi(z) = 1 - Phi(-z) and the slope of gelu without a difference that would lose what is left of either for negative z.  The quotient falls slowly, like 1 / (a sqrt(2 pi)): t P(t), t = 1 / (1 + p a), P the
// polynomial whose largest relative error over 0 <= a <= 16 is the least that its degree allows (by Remez' exchange, against the function in 64 bits).
//   fp32: of degree 9, 1.6e-8, p = 0.4 and what 1 + p a loses by rounding given to its reciprocal, since the quotient changes by up to twice what t does.  What the square loses by rounding goes into the exponential as a factor: 2^-24 of an exponent of 72 would be 36 units of the result.
//   T of 2 bytes: of degree 7, 1.7e-7, with the exponential and the reciprocal of single instructions: off by (2.5 s + 16) 2^-24 of the value, s the exponent, 2^-16 at z = -14, where half a step of bf16 is between 2^-9 and 2^-8.
struct GaussTail { float q, e; };
template <typename T>
__device__ __forceinline__ GaussTail gauss_tail(float a)
{
    if constexpr (sizeof(T) == 2) {
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.31f, a, 1.0f));
        float p = 0.0359124206f;
        p = __builtin_fmaf(p, t, -0.141914681f); p = __builtin_fmaf(p, t, 0.155632943f); p = __builtin_fmaf(p, t, -0.0154560292f); p = __builtin_fmaf(p, t, 0.110422157f);
        p = __builtin_fmaf(p, t, 0.107669815f); p = __builtin_fmaf(p, t, 0.12407776f); p = __builtin_fmaf(p, t, 0.123655692f);
        return {p * t, __builtin_amdgcn_exp2f(a * a * -0.72134752f)};            // -log2(e) / 2
    }
    a = fminf(a, 16.0f);
    const float s = a * a, lost = __builtin_fmaf(a, a, -s), x = __builtin_fmaf(0.4f, a, 1.0f), t = reciprocal(x, __builtin_fmaf(0.4f, a, 1.0f - x));
    float p = 0.0324279107f;
    p = __builtin_fmaf(p, t, -0.177947655f); p = __builtin_fmaf(p, t, 0.384890705f); p = __builtin_fmaf(p, t, -0.377340198f); p = __builtin_fmaf(p, t, 0.122096606f);
    p = __builtin_fmaf(p, t, -0.0281496216f); p = __builtin_fmaf(p, t, 0.0917519927f); p = __builtin_fmaf(p, t, 0.133058563f); p = __builtin_fmaf(p, t, 0.159636229f);
    p = __builtin_fmaf(p, t, 0.159575492f);
    return {p * t, exp_below(-0.5f * s, -0.5f * lost)};
}

template <typename T>
__device__ __forceinline__ float activate(int act, float z)
{
    switch (act) {
        case GCOO_ACT_RELU: return z <= 0.0f ? 0.0f : z;
        case GCOO_ACT_SILU: return gate<T, false>(z);
        case GCOO_ACT_GELU: {
            // max(z, 0) - |z| Phi(-|z|); as z Phi(z), infinite where z is, and no number where z is -infinite
            const float a = fabsf(fminf(z, 16.0f));
            const GaussTail g = gauss_tail<T>(a);
            return __builtin_fmaf(-a, g.q * g.e, z <= 0.0f ? 0.0f : z);
        }
        case GCOO_ACT_GELU_TANH: return gate<T, true>(z);
        default: return z;
    }
}
// the same for N values: one look at `act` for all of them
template <typename T, int N>
__device__ __forceinline__ void activate_all(int act, float (&z)[N])
{
    if (act == GCOO_ACT_NONE) return;
#define GCOO_EACH(A) _Pragma("unroll") for (int u = 0; u < N; ++u) z[u] = activate<T>(A, z[u]);
    if (act == GCOO_ACT_RELU) { GCOO_EACH(GCOO_ACT_RELU) }
    else if (act == GCOO_ACT_SILU) { GCOO_EACH(GCOO_ACT_SILU) }
    else if (act == GCOO_ACT_GELU) { GCOO_EACH(GCOO_ACT_GELU) }
    else { GCOO_EACH(GCOO_ACT_GELU_TANH) }
#undef GCOO_EACH
}
// dC act'(z)
template <typename T>
__device__ __forceinline__ float slope_times(int act, float z, float d)
{
    switch (act) {
        case GCOO_ACT_RELU: return z <= 0.0f ? 0.0f : d;
        case GCOO_ACT_SILU: return gate_slope<T, false>(z) * d;
        case GCOO_ACT_GELU: {
            // Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi), which for a and -a add up to 1
            const float a = fminf(fabsf(z), 16.0f);
            const GaussTail g = gauss_tail<T>(a);
            const float w = g.e * __builtin_fmaf(-kDensity0, a, g.q);
            return d * (z != z ? z : (z < 0.0f ? w : 1.0f - w));
        }
        case GCOO_ACT_GELU_TANH: return gate_slope<T, true>(z) * d;
        default: return d;
    }
}

// d = d act'(z) for N values
template <typename T, int N>
__device__ __forceinline__ void slope_times_all(int act, const float (&z)[N], float (&d)[N])
{
    if (act == GCOO_ACT_NONE) return;
#define GCOO_EACH(A) _Pragma("unroll") for (int u = 0; u < N; ++u) d[u] = slope_times<T>(A, z[u], d[u]);
    if (act == GCOO_ACT_RELU) { GCOO_EACH(GCOO_ACT_RELU) }
    else if (act == GCOO_ACT_SILU) { GCOO_EACH(GCOO_ACT_SILU) }
    else if (act == GCOO_ACT_GELU) { GCOO_EACH(GCOO_ACT_GELU) }
    else { GCOO_EACH(GCOO_ACT_GELU_TANH) }
#undef GCOO_EACH
}

}  // namespace gcoo
