// Operators of a layer with sparse weights: what the host code of the entry points (gcoo_layer_api.hip) passes to the kernels (layer_*.hip), and what it
// learns of a handle from gcoo_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gcoo.h"
#include "gcoo_spdm_launch.hpp"

namespace gcoo {

// The entries of a handle in row order.
struct RowsView {
    int64_t m, k, nnz;
    const int32_t* start;      // [m + 1]
    const int32_t* cols;       // a device CSR input is not checked: whoever uses a column brings it below k
    const float* vals;
};
RowsView rows_view(const gcoo_matrix* A);
int hip_failed(hipError_t e, const char* what);            // keeps the text for gcoo_last_hip_error()

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

// dst[r][0 .. N) = src[r][0 .. N) in fp32
hipError_t launch_widen(const void* src, int64_t lds, int type, float* dst, int64_t ldd, int64_t rows, int64_t N, hipStream_t s);
// C = act(P + bias) + residual, Z = P + bias; P (m x N, fp32) may be C
hipError_t launch_epilogue(const float* P, int64_t ldp, int64_t m, int64_t N, const EpilogueArgs& e, hipStream_t s);

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
hipError_t launch_epilogue_grad(const EpilogueGradArgs& a, hipStream_t s);

}  // namespace gcoo
