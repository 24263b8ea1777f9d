// What the product kernels read and write for a layer with sparse weights: B in fp32 or 16 bits, and in the place of the sums
// C = act(sum + bias) + residual, and Z = sum + bias.
#pragma once
#include "gcoo_layer.hpp"
#include "gcoo_layer_device.hpp"
#include "gcoo_spdm_rows_kernel.hpp"

#include <type_traits>

namespace gcoo {

// COLS adjacent elements at any place.
template <typename T, int COLS> struct Adjacent { typedef T vec __attribute__((ext_vector_type(COLS), aligned(sizeof(T)))); };

template <typename T, int COLS>
__device__ __forceinline__ void layer_load(const void* base, int64_t at, float (&x)[COLS])
{
    const typename Adjacent<T, COLS>::vec v = *reinterpret_cast<const typename Adjacent<T, COLS>::vec*>(static_cast<const T*>(base) + at);
#pragma unroll
    for (int u = 0; u < COLS; ++u) x[u] = widen((T)v[u]);
}
template <typename T, int COLS>
__device__ __forceinline__ void layer_store(void* base, int64_t at, const float (&x)[COLS])
{
    typename Adjacent<T, COLS>::vec v;
#pragma unroll
    for (int u = 0; u < COLS; ++u) v[u] = narrow<T>(x[u]);
    __builtin_nontemporal_store(v, reinterpret_cast<typename Adjacent<T, COLS>::vec*>(static_cast<T*>(base) + at));
}

// Elements [first, last) of COLS, which are columns jc + first .. of row r: first what the residual holds there, then what becomes of the sums x.  A lane stores where it has itself read the
// residual, so that C may be the residual.
template <typename T, int COLS>
__device__ __forceinline__ void layer_residual(const EpilogueArgs& e, int64_t r, int64_t jc, int first, int last, bool there, float (&res)[COLS])
{
#pragma unroll
    for (int u = 0; u < COLS; ++u) res[u] = 0.0f;
    if (!e.residual || !there) return;
    if (first <= 0 && last >= COLS) layer_load<T, COLS>(e.residual, r * e.ldr + jc, res);
    else
#pragma unroll
        for (int u = 0; u < COLS; ++u)
            if (u >= first && u < last) res[u] = widen(static_cast<const T*>(e.residual)[r * e.ldr + jc + u]);
}
template <typename T, int COLS>
__device__ __forceinline__ void layer_put(void* base, int64_t at, int first, int last, const float (&x)[COLS])
{
    if (first <= 0 && last >= COLS) layer_store<T, COLS>(base, at, x);
    else
#pragma unroll
        for (int u = 0; u < COLS; ++u)
            if (u >= first && u < last) static_cast<T*>(base)[at + u] = narrow<T>(x[u]);
}
template <typename T, int COLS>
__device__ __forceinline__ void layer_finish(const EpilogueArgs& e, float bias, int64_t r, int64_t jc, int first, int last, float (&x)[COLS], const float (&res)[COLS])
{
#pragma unroll
    for (int u = 0; u < COLS; ++u) x[u] += bias;
    if (e.Z) layer_put<T, COLS>(e.Z, r * e.ldz + jc, first, last, x);
    activate_all<T, COLS>(e.activation, x);
#pragma unroll
    for (int u = 0; u < COLS; ++u) x[u] += res[u];
    layer_put<T, COLS>(e.C, r * e.ldc + jc, first, last, x);
}

template <typename T, int COLS>
__device__ __forceinline__ void layer_finish(const EpilogueArgs& e, int64_t r, int64_t jc, int first, int last, float (&x)[COLS], const float (&res)[COLS])
{
    layer_finish<T, COLS>(e, e.bias ? e.bias[r] : 0.0f, r, jc, first, last, x, res);
}

// In the place of RowsPlain; TB: the elements of B, T: of all other matrices.
template <typename TB, typename T>
struct LayerIO {
    static constexpr int COLS = 16 / sizeof(TB), BYTES = sizeof(TB);
    EpilogueArgs e;
    static __device__ __forceinline__ float element(const rows_u32x4& b, int u)
    {
        if constexpr (sizeof(TB) == 4) return __uint_as_float(b[u]);
        else if constexpr (__is_same(TB, bf16_t)) return __uint_as_float(u % 2 ? b[u / 2] & 0xffff0000u : b[u / 2] << 16);
        else {
            typedef f16_t pair __attribute__((ext_vector_type(2)));
            const uint32_t word = b[u / 2];                   // (a bit cast of the vector's element itself takes the first one)
            return (float)__builtin_bit_cast(pair, word)[u % 2];
        }
    }
    template <class A>
    __device__ __forceinline__ void store(const RowsArgs&, int32_t r, int32_t jc, int32_t first, int32_t last, const A& acc) const
    {
        float x[COLS];
#pragma unroll
        for (int u = 0; u < COLS; ++u) x[u] = acc.total(u);
        float res[COLS];
        layer_residual<T, COLS>(e, r, jc, first, last, true, res);
        layer_finish<T, COLS>(e, r, jc, first, last, x, res);
    }
};

}  // namespace gcoo
