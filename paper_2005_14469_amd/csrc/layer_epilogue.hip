// Elementwise passes of a sparse layer, and their launchers.
#include "gcoo_layer.hpp"
#include "gcoo_layer_io.hpp"

namespace gcoo {

constexpr int kPassThreads = 256;

// A thread per eight elements, rows by blockIdx.y.
template <typename T>
__global__ __launch_bounds__(kPassThreads) void layer_widen(const T* __restrict__ src, int64_t lds, float* __restrict__ dst, int64_t ldd, int64_t rows, int64_t N)
{
    const int64_t j = ((int64_t)blockIdx.x * kPassThreads + threadIdx.x) * 8;
    if (j >= N) return;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        float x[8];
        if (j + 8 <= N) layer_load<T, 8>(src, r * lds + j, x);
        else
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = j + u < N ? widen(src[r * lds + j + u]) : 0.0f;
        // (what lies behind N in the last piece is part of the padding of a row)
        rows_f32x4* to = reinterpret_cast<rows_f32x4*>(dst + r * ldd + j);
        to[0] = rows_f32x4{x[0], x[1], x[2], x[3]};
        to[1] = rows_f32x4{x[4], x[5], x[6], x[7]};
    }
}

// A matrix without entries.
template <typename T>
__global__ __launch_bounds__(kPassThreads) void layer_no_entries(int64_t m, int64_t N, EpilogueArgs e)
{
    const int64_t j = (int64_t)blockIdx.x * kPassThreads + threadIdx.x;
    if (j >= N) return;
    for (int64_t r = blockIdx.y; r < m; r += gridDim.y) {
        float x[1] = {0.0f}, res[1];
        layer_residual<T, 1>(e, r, j, 0, 1, true, res);
        layer_finish<T, 1>(e, r, j, 0, 1, x, res);
    }
}

static dim3 pass_grid(int64_t rows, int64_t pieces) { return dim3((unsigned)((pieces + kPassThreads - 1) / kPassThreads), (unsigned)(rows < 65535 ? rows : 65535)); }

hipError_t launch_widen(const void* src, int64_t lds, int type, float* dst, int64_t ldd, int64_t rows, int64_t N, hipStream_t s)
{
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        if constexpr (sizeof(T) == 4) return hipErrorInvalidValue;
        else {
            layer_widen<T><<<pass_grid(rows, (N + 7) / 8), dim3(kPassThreads), 0, s>>>(static_cast<const T*>(src), lds, dst, ldd, rows, N);
            return hipGetLastError();
        }
    });
}

hipError_t launch_epilogue(int64_t m, int64_t N, const EpilogueArgs& e, hipStream_t s)
{
    return with_type(e.type, [&](auto t) {
        layer_no_entries<decltype(t)><<<pass_grid(m, N), dim3(kPassThreads), 0, s>>>(m, N, e);
        return hipGetLastError();
    });
}

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(kPassThreads) void layer_epilogue_grad(EpilogueGradArgs a)
{
    __shared__ float part[kPassThreads / 64];
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
        float sum = 0.0f;
        for (int64_t j = threadIdx.x; j < a.N; j += kPassThreads) {
            const float d = widen(static_cast<const T*>(a.dC)[r * a.lddc + j]);
            const float g = a.activation ? slope_times(a.activation, widen(static_cast<const T*>(a.Z)[r * a.ldz + j]), d) : d;
            if (a.dZ) static_cast<T*>(a.dZ)[r * a.lddz + j] = narrow<T>(g);
            sum += g;
        }
        if (!a.dbias) continue;
        sum = wave_sum(sum);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
        __syncthreads();
        if (threadIdx.x == 0) a.dbias[r] = (part[0] + part[1]) + (part[2] + part[3]);
        __syncthreads();
    }
}

hipError_t launch_epilogue_grad(const EpilogueGradArgs& a, hipStream_t s)
{
    return with_type(a.type, [&](auto t) {
        layer_epilogue_grad<decltype(t)><<<dim3((unsigned)(a.m < 0x7fffffff ? a.m : 0x7fffffff)), dim3(kPassThreads), 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace gcoo
