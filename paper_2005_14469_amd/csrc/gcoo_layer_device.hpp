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

__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
constexpr float kGeluA = 0.7978845608028654f, kGeluB = 0.044715f, kRootHalf = 0.7071067811865476f, kDensity0 = 0.3989422804014327f;

// 1 + erf(z / sqrt(2)) and exp(-z^2 / 2).  T of 2 bytes: by the rational approximation 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions, off by 1.5e-7 at the most, a thousandth of
// what such a T is rounded by, and not by a difference for negative z, with the exponential that the slope needs anyway (14000 x 8000, bf16, the gradient through gelu: 150 us with the library's erf).
template <typename T>
__device__ __forceinline__ float erfc_and_exp(float z, float* e)
{
    *e = __expf(-0.5f * z * z);
    if constexpr (sizeof(T) == 4) return 1.0f + erff(z * kRootHalf);
    const float x = fabsf(z) * kRootHalf, t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    const float p = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    return z < 0.0f ? p * *e : 2.0f - p * *e;
}

template <typename T>
__device__ __forceinline__ float activate(int act, float z)
{
    switch (act) {
        case GCOO_ACT_RELU: return z <= 0.0f ? 0.0f : z;
        case GCOO_ACT_SILU: return z * logistic(z);
        case GCOO_ACT_GELU: {
            float e;
            return 0.5f * z * erfc_and_exp<T>(z, &e);
        }
        case GCOO_ACT_GELU_TANH: return z * logistic(2.0f * kGeluA * (z + kGeluB * z * z * z));
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
// (z s(q z + r z^3))' at z, s the logistic function: s + z s (1 - s) (q + 3 r z^2).  1 - s is E s, E = exp(-(q z + r z^3)): the difference would have lost what the factors behind it
// need.  `c` is z held where E is finite; what is left out there is below 1e-18.
__device__ __forceinline__ float slope_of_gate(float z, float c, float q, float r)
{
    const float c2 = c * c, e = __expf(-c * (q + r * c2)), s = __builtin_amdgcn_rcpf(1.0f + e);
    return z != z ? z : s + c * s * (e * s) * (q + 3.0f * r * c2);
}
// dC act'(z)
template <typename T>
__device__ __forceinline__ float slope_times(int act, float z, float d)
{
    switch (act) {
        case GCOO_ACT_RELU: return z <= 0.0f ? 0.0f : d;
        case GCOO_ACT_SILU: return slope_of_gate(z, fminf(fmaxf(z, -80.0f), 80.0f), 1.0f, 0.0f) * d;
        case GCOO_ACT_GELU: {
            float e;
            const float f = erfc_and_exp<T>(z, &e);
            return d * (0.5f * f + fminf(fmaxf(z, -80.0f), 80.0f) * kDensity0 * e);          // (infinite z, which a sum may be rounded to: 0 or 1)
        }
        case GCOO_ACT_GELU_TANH: return slope_of_gate(z, fminf(fmaxf(z, -8.0f), 8.0f), 2.0f * kGeluA, 2.0f * kGeluA * kGeluB) * d;
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
