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

__global__ __launch_bounds__(kPassThreads) void layer_realign(const uint16_t* __restrict__ src, int64_t lds, uint16_t* __restrict__ dst, int64_t ldd, int64_t rows, int64_t N)
{
    const int64_t j = ((int64_t)blockIdx.x * kPassThreads + threadIdx.x) * 8;
    if (j >= N) return;
    typedef uint16_t vec __attribute__((ext_vector_type(8)));
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        vec x;
        if (j + 8 <= N) x = *reinterpret_cast<const Adjacent<uint16_t, 8>::vec*>(src + r * lds + j);
        else
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = j + u < N ? src[r * lds + j + u] : (uint16_t)0;
        *reinterpret_cast<vec*>(dst + r * ldd + j) = x;
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

hipError_t launch_realign(const void* src, int64_t lds, void* dst, int64_t ldd, int64_t rows, int64_t N, hipStream_t s)
{
    layer_realign<<<pass_grid(rows, (N + 7) / 8), dim3(kPassThreads), 0, s>>>(static_cast<const uint16_t*>(src), lds, static_cast<uint16_t*>(dst), ldd, rows, N);
    return hipGetLastError();
}

hipError_t launch_epilogue(int64_t m, int64_t N, const EpilogueArgs& e, hipStream_t s)
{
    return with_type(e.type, [&](auto t) {
        layer_no_entries<decltype(t)><<<pass_grid(m, N), dim3(kPassThreads), 0, s>>>(m, N, e);
        return hipGetLastError();
    });
}

// The gradient through the epilogue: LANES lanes on a row (16, 64 or the 256 of a workgroup), each 16 bytes of it at a time, four such pieces of both operands on their way; the row's sum in a fixed tree.
// Rows of a matrix that has few of them are cut into parts, a workgroup each, whose sums epilogue_grad_join adds in their order.
// Bound: memory (14000 x 8000, bf16, silu: 119 us, 672 MB, 5.6 TB/s, where a large copy has 4.9: part of it is still in the memory-side cache); below a megabyte the launch (1000 x 333, fp32, gelu: 4.1 us in the kernel).
template <typename T, int LANES>
__global__ __launch_bounds__(kPassThreads) void layer_epilogue_grad(EpilogueGradArgs a, float* part, int64_t part_cols)
{
    constexpr int V = 16 / sizeof(T), U = 4;
    __shared__ float sums[kPassThreads / 64];
    const int lane = (int)threadIdx.x % LANES;
    const int64_t r = (int64_t)blockIdx.x * (kPassThreads / LANES) + threadIdx.x / LANES;
    if (LANES < kPassThreads && r >= a.m) return;
    const int64_t from = (int64_t)blockIdx.y * part_cols, to = from + part_cols < a.N ? from + part_cols : a.N;
    float sum = 0.0f;
    for (int64_t j0 = from + lane * V; j0 < to; j0 += LANES * V * U) {
        float d[U][V], z[U][V];
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int64_t j = j0 + s * (LANES * V);
            if (j >= to) break;
            if (j + V <= to) {
                layer_load<T, V>(a.dC, r * a.lddc + j, d[s]);
                if (a.activation) layer_load<T, V>(a.Z, r * a.ldz + j, z[s]);
            } else {
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    const bool in = j + u < to;
                    d[s][u] = in ? widen(static_cast<const T*>(a.dC)[r * a.lddc + j + u]) : 0.0f;
                    z[s][u] = in && a.activation ? widen(static_cast<const T*>(a.Z)[r * a.ldz + j + u]) : 0.0f;
                }
            }
        }
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int64_t j = j0 + s * (LANES * V);
            if (j >= to) break;
            slope_times_all<T, V>(a.activation, z[s], d[s]);
            if (a.dZ) {
                if (j + V <= to) layer_store<T, V>(a.dZ, r * a.lddz + j, d[s]);
                else
#pragma unroll
                    for (int u = 0; u < V; ++u)
                        if (j + u < to) static_cast<T*>(a.dZ)[r * a.lddz + j + u] = narrow<T>(d[s][u]);
            }
#pragma unroll
            for (int u = 0; u < V; ++u) sum += j + u < to ? d[s][u] : 0.0f;
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int x = LANES < 64 ? LANES / 2 : 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x, LANES < 64 ? LANES : 64);
    float* out = part ? part + (int64_t)blockIdx.y * a.m : a.dbias;
    if constexpr (LANES <= 64) {
        if (lane == 0) out[r] = sum;
    } else {
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
        __syncthreads();
        if (threadIdx.x == 0) out[r] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    }
}

__global__ __launch_bounds__(kPassThreads) void epilogue_grad_join(const float* part, float* dbias, int64_t m, int32_t parts)
{
    const int64_t r = (int64_t)blockIdx.x * kPassThreads + threadIdx.x;
    if (r >= m) return;
    float sum = part[r];
    for (int32_t p = 1; p < parts; ++p) sum += part[p * m + r];
    dbias[r] = sum;
}

int32_t epilogue_grad_parts(int64_t m, int64_t N)
{
    constexpr int64_t least = 8192;                              // columns of a part
    if (m < 1 || m >= 1024 || N < 2 * least) return 1;
    const int64_t most = N / least, wanted = (2048 + m - 1) / m;
    return (int32_t)(most < wanted ? most : wanted);
}

template <typename T, int LANES>
static hipError_t launch_grad_lanes(const EpilogueGradArgs& a, int32_t parts, float* part, hipStream_t s)
{
    constexpr int64_t rows = kPassThreads / LANES;
    const int64_t grid = (a.m + rows - 1) / rows, cols = ((a.N + parts - 1) / parts + 63) / 64 * 64;
    if (too_wide(grid, kPassThreads)) return hipErrorInvalidConfiguration;
    layer_epilogue_grad<T, LANES><<<dim3((unsigned)grid, (unsigned)parts), dim3(kPassThreads), 0, s>>>(a, parts > 1 ? part : nullptr, cols > 0 ? cols : 64);
    return hipGetLastError();
}

hipError_t launch_epilogue_grad(const EpilogueGradArgs& a, float* part, hipStream_t s)
{
    const int32_t parts = epilogue_grad_parts(a.m, a.N);
    const hipError_t e = with_type(a.type, [&](auto t) {
        typedef decltype(t) T;
        const int64_t pieces = a.N * (int64_t)sizeof(T) / 16;
        if (pieces <= 32) return launch_grad_lanes<T, 16>(a, parts, part, s);
        // (few rows: a workgroup to each; us, 64 lanes and 256: fp32, 1000 x 1000: 10.6 9.1; 4000 x 512: 7.5 9.0; bf16, 4000 x 512: 7.3 12.0; 8000 x 1000: 16.2 23.9; 300 x 8000: 24.5 10.5)
        return pieces <= 256 && (pieces <= 64 || a.m > 2048) ? launch_grad_lanes<T, 64>(a, parts, part, s) : launch_grad_lanes<T, 256>(a, parts, part, s);
    });
    if (e != hipSuccess || parts == 1 || !a.dbias) return e;
    epilogue_grad_join<<<dim3((unsigned)((a.m + kPassThreads - 1) / kPassThreads)), dim3(kPassThreads), 0, s>>>(part, a.dbias, a.m, parts);
    return hipGetLastError();
}

}  // namespace gcoo
