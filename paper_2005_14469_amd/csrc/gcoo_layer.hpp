// Operators of a layer with sparse weights: what the host code of the entry points (gcoo_layer_api.hip) passes to the kernels (layer_*.hip), and what it
// learns of a handle from gcoo_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gcoo.h"
#include "gcoo_spdm_launch.hpp"

namespace gcoo {

// The rows of more than long_row entries as the conversion lists them: the longest from the front, the others from the back (counted), or, without counts, in places of which some hold -1.
struct LongRows {
    const int32_t* rows;       // [room]
    const int32_t* count;      // [0]: of those from the back, [2]: from the front; or null
    int32_t long_row, room;
};
// The entries of a handle in row order.
struct RowsView {
    int64_t m, k, nnz;
    const int32_t* start;      // [m + 1]
    const int32_t* cols;       // a device CSR input is not checked: whoever uses a column brings it below k
    const float* vals;
    LongRows longs;
};
RowsView rows_view(const gcoo_matrix* A);
int hip_failed(hipError_t e, const char* what);            // keeps the text for gcoo_last_hip_error()

// A launch of more threads than one takes is refused before it is made.
inline bool too_wide(int64_t workgroups, int threads) { return workgroups > 0xffffffffLL / threads; }

constexpr size_t type_bytes(int type) { return type == GCOO_F32 ? 4 : 2; }

struct EpilogueArgs {
    const float* bias;
    const void* residual;
    int64_t ldr;
    void* Z;
    int64_t ldz;
    void* C;
    int64_t ldc;
    int32_t type, activation;
};

// dst[r][0 .. N) = src[r][0 .. N) of 2-byte elements (or halves of 4-byte ones), as they are, or in fp32; ldd a multiple of 8
hipError_t launch_realign(const void* src, int64_t lds, void* dst, int64_t ldd, int64_t rows, int64_t N, hipStream_t s);
hipError_t launch_widen(const void* src, int64_t lds, int type, float* dst, int64_t ldd, int64_t rows, int64_t N, hipStream_t s);
// the epilogue of a matrix without entries
hipError_t launch_epilogue(int64_t m, int64_t N, const EpilogueArgs& e, hipStream_t s);

// Which kernel a product with its epilogue runs: none has entries, row by row (and few columns), on a few columns of B held in LDS, on tiles of B in LDS, or by the sixteen-wave kernel, for which a B of 2-byte elements is
// widened into `work` bytes of the caller's, rows ldw elements apart (and row by row, where that pays for rows at odd places or inside 128-byte lines, copied there).
enum ProductKernel { kProductNone, kProductRows, kProductHeld, kProductTile, kProductBand };
struct ProductPlan { ProductKernel kernel; int64_t ldw; size_t work; };
ProductPlan product_plan(const gcoo_matrix* A, const void* B, int64_t ldb, int64_t N, int type);
hipError_t launch_product(const gcoo_matrix* A, const ProductPlan& plan, const void* B, int64_t ldb, int64_t N, const EpilogueArgs& e, void* work, hipStream_t s);

// Rows of 2-byte elements at places that 16-byte buffer loads, which want multiples of 4, do not take: they are read by 64-bit addresses.
inline bool odd_rows(const void* B, int64_t ldb, int type) { return type != GCOO_F32 && (reinterpret_cast<uintptr_t>(B) % 4 != 0 || ldb % 2 != 0); }

// RowsArgs::B and BandArgs::B point to elements of e.type (of the bands: to fp32); C is in e.
hipError_t launch_layer_rows_f32(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s);
hipError_t launch_layer_rows_bf16(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s);
hipError_t launch_layer_rows_f16(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s);
hipError_t launch_layer_tile(const RowsArgs& a, const EpilogueArgs& e, int64_t row_wgs, bool whole, hipStream_t s);
hipError_t launch_layer_tile_halves(const RowsArgs& a, const EpilogueArgs& e, int64_t row_wgs, bool whole, hipStream_t s);      // of a product of half as many columns
hipError_t launch_layer_band_f32(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s);
hipError_t launch_layer_band_bf16(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s);
hipError_t launch_layer_band_f16(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s);

struct EpilogueGradArgs {
    const void* Z;
    int64_t ldz;
    const void* dC;
    int64_t lddc;
    void* dZ;
    int64_t lddz;
    float* dbias;
    int64_t m, N;
    int32_t type, activation;
};
// Parts of a row; part: that many times m sums where there is more than one.
int32_t epilogue_grad_parts(int64_t m, int64_t N);
hipError_t launch_epilogue_grad(const EpilogueGradArgs& a, float* part, hipStream_t s);

}  // namespace gcoo
