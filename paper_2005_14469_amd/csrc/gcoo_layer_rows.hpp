// The product with its epilogue row by row (gcoo_spdm_rows_kernel.hpp, with B in its own type and the epilogue in the place of the stores), and for few
// columns; instances by type in layer_rows_*.hip.
#pragma once
#include "gcoo_layer_io.hpp"

namespace gcoo {

// (registers for four waves of a SIMD, five with eight rows of B in flight: the epilogue and a lane's eight columns do not leave enough for eight)
template <typename T, int LPR, bool WIDE, int AHEAD, int SUMS, RowsLong LONG>
__global__ __launch_bounds__(kRowsThreads, AHEAD == 16 ? (LPR == 4 || (LPR == 16 && SUMS == 2) ? 3 : 4) : 5) void layer_rows(RowsArgs a, LayerIO<T, T> io, int32_t tiles, int32_t row_wgs, int32_t rpw, int32_t wave_row)
{
    __shared__ __attribute__((aligned(16))) float part[kRowsWaves][LPR * LayerIO<T, T>::COLS];
    rows_item<LPR, WIDE, AHEAD, SUMS, LONG>(a, io, blockIdx.x, tiles, row_wgs, rpw, wave_row, RowsTurns{}, part);
}

// Few columns: LANES lanes share a row, each takes every LANES-th entry, four of them at a time, so that four rows of B are on their way; their sums are added up in a fixed tree.
// A single token reads the entries and hardly anything else.
template <typename T, int LANES, int N>
__global__ __launch_bounds__(kRowsThreads) void layer_few(RowsArgs a, EpilogueArgs e)
{
    const int lane = threadIdx.x % LANES;
    const int64_t r = (int64_t)blockIdx.x * (kRowsThreads / LANES) + threadIdx.x / LANES;
    if (r >= a.m) return;
    const uint32_t kmax = (uint32_t)(a.k - 1);
    const T* B = reinterpret_cast<const T*>(a.B);
    const int n = (int)a.N;
    float sum[N] = {};
    const uint32_t end = (uint32_t)a.row_ptr[r + 1];                     // (unsigned: a step beyond the last of 2^31 entries stays a number)
    for (uint32_t i = (uint32_t)a.row_ptr[r] + (uint32_t)lane; i < end; i += 4 * LANES) {
        uint32_t c[4];
        float v[4], b[4][N];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool in = i + q * LANES < end;
            c[q] = in ? (uint32_t)a.cols[i + q * LANES] : 0xffffffffu;
            v[q] = in ? a.vals[i + q * LANES] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const T* row = B + (int64_t)(c[q] < kmax ? c[q] : kmax) * a.ldb;
#pragma unroll
            for (int j = 0; j < N; ++j) b[q][j] = j < n && i + q * LANES < end ? widen(row[j]) : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] = __builtin_fmaf(v[q], b[q][j], sum[j]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int d = LANES / 2; d >= 1; d >>= 1) sum[j] += __shfl_xor(sum[j], d, LANES);
    if (lane == 0) {
        float res[N];
        layer_residual<T, N>(e, r, 0, 0, n, true, res);
        layer_finish<T, N>(e, r, 0, 0, n, sum, res);
    }
}

template <typename T, int LPR, bool WIDE, int AHEAD, int SUMS>
hipError_t launch_layer_rows_ahead(const RowsArgs& a, const EpilogueArgs& e, int64_t N4, hipStream_t s)
{
    const RowsGrid g = rows_grid(a, LPR, LPR * LayerIO<T, T>::COLS, N4);
    if (g.grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const auto kernel = !a.long_count && a.long_room > 0 ? layer_rows<T, LPR, WIDE, AHEAD, SUMS, kLongPlaces> : layer_rows<T, LPR, WIDE, AHEAD, SUMS, kLongCounted>;
    kernel<<<dim3((unsigned)g.grid), dim3(kRowsThreads), 0, s>>>(a, LayerIO<T, T>{e}, (int32_t)g.tiles, (int32_t)g.row_wgs, (int32_t)g.rpw, g.wave_row);
    return hipGetLastError();
}

template <typename T, int LPR, int SUMS = LPR <= 16 ? 1 : LPR / 16>
hipError_t launch_layer_rows(const RowsArgs& a, const EpilogueArgs& e, int64_t N4, hipStream_t s)
{
    if constexpr (LPR >= 16)
        if (a.nnz <= 16 * a.m) return launch_layer_rows_ahead<T, LPR, false, 8, SUMS>(a, e, N4, s);
    return launch_layer_rows_ahead<T, LPR, false, 16, SUMS>(a, e, N4, s);
}

template <typename T, int LANES>
hipError_t launch_layer_few(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    const dim3 grid((unsigned)((a.m + kRowsThreads / LANES - 1) / (kRowsThreads / LANES))), threads(kRowsThreads);
    if (a.N == 1) layer_few<T, LANES, 1><<<grid, threads, 0, s>>>(a, e);
    else if (a.N <= 4) layer_few<T, LANES, 4><<<grid, threads, 0, s>>>(a, e);
    else layer_few<T, LANES, 8><<<grid, threads, 0, s>>>(a, e);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_layer_rows_of(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    if (a.m < 1 || a.k < 1 || a.N < 1 || a.ldb > 0x3fffffffLL) return hipErrorInvalidValue;
    if (a.N < LayerIO<T, T>::COLS) return a.nnz >= 128 * a.m ? launch_layer_few<T, 64>(a, e, s) : launch_layer_few<T, 16>(a, e, s);
    // a matrix of 2-byte elements is cut as one of half as many 4-byte ones
    RowsArgs as4 = a;
    if (sizeof(T) == 2) { as4.N = (a.N + 1) / 2; as4.ldb = (a.ldb + 1) / 2; }
    // Beyond the offsets of a buffer descriptor, or at places that its loads do not take: 64-bit addresses.
    if (odd_elements(a.B, a.ldb, a.N, e.type) || (uint64_t)a.k * (uint64_t)a.ldb * sizeof(T) > kRowsMaxBytes) return launch_layer_rows_ahead<T, 16, true, 16, 1>(a, e, as4.N, s);
    const RowsWidth w = rows_width(as4);
    switch (w.lanes) {
        case 4: return launch_layer_rows<T, 4>(a, e, as4.N, s);
        case 8: return launch_layer_rows<T, 8>(a, e, as4.N, s);
        case 16: return w.sums == 2 ? launch_layer_rows<T, 16, 2>(a, e, as4.N, s) : launch_layer_rows<T, 16>(a, e, as4.N, s);
        case 32: return launch_layer_rows<T, 32>(a, e, as4.N, s);
        default: return launch_layer_rows<T, 64>(a, e, as4.N, s);
    }
}

}  // namespace gcoo
