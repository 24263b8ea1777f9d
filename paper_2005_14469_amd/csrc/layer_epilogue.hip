// Elementwise passes of a sparse layer, and their launchers.
#include "gcoo_layer.hpp"
#include "gcoo_layer_device.hpp"

namespace gcoo {

constexpr int kPassThreads = 256;

// A thread per element, rows by blockIdx.y.
template <typename T>
__global__ __launch_bounds__(kPassThreads) void layer_widen(const T* __restrict__ src, int64_t lds, float* __restrict__ dst, int64_t ldd, int64_t rows, int64_t N)
{
    const int64_t j = (int64_t)blockIdx.x * kPassThreads + threadIdx.x;
    if (j >= N) return;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) dst[r * ldd + j] = widen(src[r * lds + j]);
}

template <typename T>
__global__ __launch_bounds__(kPassThreads) void layer_epilogue(const float* P, int64_t ldp, int64_t m, int64_t N, EpilogueArgs e)
{
    const int64_t j = (int64_t)blockIdx.x * kPassThreads + threadIdx.x;
    if (j >= N) return;
    for (int64_t r = blockIdx.y; r < m; r += gridDim.y) {
        const float z = (P ? P[r * ldp + j] : 0.0f) + (e.bias ? e.bias[r] : 0.0f);
        if (e.Z) static_cast<T*>(e.Z)[r * e.ldz + j] = narrow<T>(z);
        float y = activate(e.activation, z);
        if (e.residual) y += widen(static_cast<const T*>(e.residual)[r * e.ldr + j]);
        static_cast<T*>(e.C)[r * e.ldc + j] = narrow<T>(y);
    }
}

static dim3 pass_grid(int64_t rows, int64_t N) { return dim3((unsigned)((N + kPassThreads - 1) / kPassThreads), (unsigned)(rows < 65535 ? rows : 65535)); }

hipError_t launch_widen(const void* src, int64_t lds, int type, float* dst, int64_t ldd, int64_t rows, int64_t N, hipStream_t s)
{
    if (rows < 1 || N < 1) return hipSuccess;
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        layer_widen<T><<<pass_grid(rows, N), dim3(kPassThreads), 0, s>>>(static_cast<const T*>(src), lds, dst, ldd, rows, N);
        return hipGetLastError();
    });
}

hipError_t launch_epilogue(const float* P, int64_t ldp, int64_t m, int64_t N, const EpilogueArgs& e, hipStream_t s)
{
    if (m < 1 || N < 1) return hipSuccess;
    return with_type(e.type, [&](auto t) {
        layer_epilogue<decltype(t)><<<pass_grid(m, N), dim3(kPassThreads), 0, s>>>(P, ldp, m, N, e);
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
