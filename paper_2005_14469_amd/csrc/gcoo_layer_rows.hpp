// The product with its epilogue row by row (gcoo_spdm_rows_kernel.hpp, with B in its own type and the epilogue in the place of the stores), and for few
// columns; instances by type in layer_rows_*.hip.
// Bound: the rows of B through the vector caches (8000 x 8000, 0.5 %, N = 8000, bf16, bias, gelu_tanh and residual: 296 us behind cold caches, 5.1 GB of rows of B, 18 TB/s; B, residual and C once would take 79).
#pragma once
#include "gcoo_layer_io.hpp"
#include "gcoo_layer_long.hpp"

namespace gcoo {

// (registers for four waves of a SIMD, five with eight rows of B in flight: the epilogue and a lane's eight columns do not leave enough for eight)
template <typename T, int LPR, bool WIDE, int AHEAD, int SUMS, RowsLong LONG>
__global__ __launch_bounds__(kRowsThreads, AHEAD == 16 ? (LPR == 4 || (LPR == 16 && SUMS == 2) ? 3 : 4) : 5) void layer_rows(RowsArgs a, LayerIO<T, T> io, int32_t tiles, int32_t row_wgs, int32_t rpw, int32_t wave_row)
{
    __shared__ __attribute__((aligned(16))) float part[kRowsWaves][LPR * LayerIO<T, T>::COLS];
    rows_item<LPR, WIDE, AHEAD, SUMS, LONG>(a, io, blockIdx.x, tiles, row_wgs, rpw, wave_row, RowsTurns{}, part);
}

// Few columns: LANES lanes share a row, each takes four adjacent entries at a time with one load each of columns and values, GROUPS such on their way; their sums are added up in a fixed tree.
// The elements of B lie anywhere: a lane's takes a clock of its compute unit from the vector cache, so products of many entries hold B in LDS instead (layer_held.hip).
// Long rows have workgroups of their own, `long_wgs` behind the others (us, one token: power-law rows, 16384 x 16384, of 53 entries, fp32: 28 10; ten full rows among 20000 of 20 entries: 113 14; even rows level).
template <typename T, int LANES, int N, int GROUPS>
__global__ __launch_bounds__(kRowsThreads) void layer_few(RowsArgs a, EpilogueArgs e, int32_t long_wgs)
{
    constexpr int SLOTS = kRowsThreads / LANES;
    const uint32_t kmax = (uint32_t)(a.k - 1);
    const T* B = reinterpret_cast<const T*>(a.B);
    const int n = (int)a.N;
    const int32_t wgs = (int32_t)gridDim.x - long_wgs;
    const bool shares = (int32_t)blockIdx.x >= wgs;
    const LongRows longs{a.long_rows, shares ? a.long_count : nullptr, a.long_row, shares ? a.long_room : 0};
    LongWalk<1> walk(longs, a.row_ptr, a.m, (int32_t)blockIdx.x - wgs, long_wgs);
    int32_t long_row = 0, piece;
    if (shares && !walk.next(&long_row, &piece)) return;
    const uint32_t lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    typedef uint32_t cols4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef float vals4 __attribute__((ext_vector_type(4), aligned(4)));
    for (;;) {
        // the row of these lanes, or a stretch of the workgroup's (unsigned: a step beyond the last of 2^31 entries stays a number)
        int64_t r = (int64_t)blockIdx.x * SLOTS + slot;
        uint32_t beg = 0, end = 0;
        if (shares) {
            r = long_row;
            beg = (uint32_t)a.row_ptr[r];
            end = (uint32_t)a.row_ptr[r + 1];
            const uint32_t each = (end - beg + SLOTS - 1) / SLOTS;
            beg += slot * each;
            end = beg + each < end ? beg + each : end;
        } else {
            if (r >= a.m) return;
            beg = (uint32_t)a.row_ptr[r];
            end = (uint32_t)a.row_ptr[r + 1];
            if ((int32_t)(end - beg) > a.long_row) return;
        }
        float sum[N] = {};
        for (uint32_t i = beg + 4 * lane; i < end; i += 4 * LANES * GROUPS) {
            uint32_t c[GROUPS][4];
            float v[GROUPS][4];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const uint32_t at = i + 4 * LANES * g;
                if (at + 4 <= end) {
                    const cols4 x = *reinterpret_cast<const cols4*>(a.cols + at);
                    const vals4 y = *reinterpret_cast<const vals4*>(a.vals + at);
#pragma unroll
                    for (int q = 0; q < 4; ++q) { c[g][q] = x[q]; v[g][q] = y[q]; }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const bool in = at + q < end;
                        c[g][q] = in ? (uint32_t)a.cols[at + q] : 0u;
                        v[g][q] = in ? a.vals[at + q] : 0.0f;
                    }
                }
            }
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bool in = i + 4 * LANES * g + q < end;
                    const uint32_t col = c[g][q] < kmax ? c[g][q] : kmax;
                    const T* row = B + (int64_t)col * a.ldb;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float b = in && j < n ? widen(row[j]) : 0.0f;
                        sum[j] = __builtin_fmaf(v[g][q], b, sum[j]);
                    }
                }
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int d = LANES / 2; d >= 1; d >>= 1) sum[j] += __shfl_xor(sum[j], d, LANES);
        bool stores = lane == 0;
        if (shares) {
            __shared__ float part[SLOTS][N];
            if (lane == 0)
#pragma unroll
                for (int j = 0; j < N; ++j) part[slot][j] = sum[j];
            __syncthreads();
            stores = threadIdx.x == 0;
            if (stores)
                for (int w = 1; w < SLOTS; ++w)
#pragma unroll
                    for (int j = 0; j < N; ++j) sum[j] += part[w][j];
            __syncthreads();
        }
        if (stores) {
            float res[N];
            layer_residual<T, N>(e, r, 0, 0, n, true, res);
            layer_finish<T, N>(e, r, 0, 0, n, sum, res);
        }
        if (!shares || !walk.next(&long_row, &piece)) return;
    }
}

template <typename T, int LPR, bool WIDE, int AHEAD, int SUMS>
hipError_t launch_layer_rows_ahead(const RowsArgs& a, const EpilogueArgs& e, int64_t N4, hipStream_t s)
{
    const RowsGrid g = rows_grid(a, LPR, LPR * LayerIO<T, T>::COLS, N4);
    if (too_wide(g.grid, kRowsThreads)) return hipErrorInvalidConfiguration;
    const auto kernel = !a.long_count && a.long_room > 0 ? layer_rows<T, LPR, WIDE, AHEAD, SUMS, kLongPlaces> : layer_rows<T, LPR, WIDE, AHEAD, SUMS, kLongCounted>;
    kernel<<<dim3((unsigned)g.grid), dim3(kRowsThreads), 0, s>>>(a, LayerIO<T, T>{e}, (int32_t)g.tiles, (int32_t)g.row_wgs, (int32_t)g.rpw, g.wave_row);
    return hipGetLastError();
}

template <typename T, int LPR, int SUMS = LPR <= 16 ? 1 : LPR / 16>
hipError_t launch_layer_rows(const RowsArgs& a, const EpilogueArgs& e, int64_t N4, hipStream_t s)
{
    // (2-byte elements up to 24 entries per row, whose waves have more registers to lose; us, sixteen and eight rows of B on their way: 4000 x 4000, rows of 20, N = 4000: bf16 55.4 47.3, fp16 47.7 41.3; 14000 x 14000, of 28,
    // N = 2000: 125 137.  By matrix instructions, each value as three numbers in bf16, rows of 40 took as long: the caches are the bound)
    if constexpr (LPR >= 16)
        if (a.nnz <= (sizeof(T) == 2 ? 24 : 16) * a.m) return launch_layer_rows_ahead<T, LPR, false, 8, SUMS>(a, e, N4, s);
    return launch_layer_rows_ahead<T, LPR, false, 16, SUMS>(a, e, N4, s);
}

template <typename T, int LANES, int N, int GROUPS>
hipError_t launch_layer_few(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    const int32_t long_wgs = a.long_room < 256 ? a.long_room : 256;
    const int64_t grid = (a.m + kRowsThreads / LANES - 1) / (kRowsThreads / LANES) + long_wgs;
    if (too_wide(grid, kRowsThreads)) return hipErrorInvalidConfiguration;
    layer_few<T, LANES, N, GROUPS><<<dim3((unsigned)grid), dim3(kRowsThreads), 0, s>>>(a, e, long_wgs);
    return hipGetLastError();
}
template <typename T, int LANES>
hipError_t launch_layer_few(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    if (a.N == 1) return launch_layer_few<T, LANES, 1, 4>(a, e, s);
    if (a.N <= 4) return launch_layer_few<T, LANES, 4, 2>(a, e, s);
    if constexpr (sizeof(T) == 2) return launch_layer_few<T, LANES, 8, 1>(a, e, s);
    return hipErrorInvalidValue;
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
    if (odd_rows(a.B, a.ldb, e.type) || (uint64_t)a.k * (uint64_t)a.ldb * sizeof(T) > kRowsMaxBytes) return launch_layer_rows_ahead<T, 16, true, 16, 1>(a, e, as4.N, s);
    RowsWidth w = rows_width(as4);
    // Many rows of B and more entries than a narrow wave has on their way: 16 lanes to a row, not 32, whose eight columns in two sums leave no registers for a fifth wave and whose tiles of 512 bytes have to share the L2 with
    // what the epilogue reads (us, 32 and 16: bf16, N = 8000: 5500 x 5500, 0.3 %: 128 111; 6500, 0.6 %: 222 201; 8000, 0.3 %: 218 189, 0.6 %: 324 285; N = 2000: 8000, 0.3 %: 65 60; fp16, N = 8000: 6500, 0.3 %:
    // 137 131, 8000, 0.6 %: 293 297; rows of 4 to 8 entries, bf16: 8000, N = 8000, 0.1 %: 114 146).
    if (sizeof(T) == 2 && w.lanes == 32 && a.nnz > 16 * a.m && a.k >= 5000) w = {16, 1};
    switch (w.lanes) {
        case 4: return launch_layer_rows<T, 4>(a, e, as4.N, s);
        case 8: return launch_layer_rows<T, 8>(a, e, as4.N, s);
        case 16: return w.sums == 2 ? launch_layer_rows<T, 16, 2>(a, e, as4.N, s) : launch_layer_rows<T, 16>(a, e, as4.N, s);
        case 32: return launch_layer_rows<T, 32>(a, e, as4.N, s);
        default: return launch_layer_rows<T, 64>(a, e, as4.N, s);
    }
}

}  // namespace gcoo
