// Launch interface of the gradient of the stored weights (layer_values.hip).
#pragma once
#include "gcoo_layer.hpp"

namespace gcoo {

constexpr int kValuesThreads = 256;
constexpr int64_t kValuesSums = int64_t(1) << 28;          // sums of parts that wait to be joined, at the most (1 GB); more only where eight of every entry are

struct GradValuesArgs {
    RowsView A;
    const void* dZ;
    int64_t lddz;
    const void* B;
    int64_t ldb;
    int64_t N;
    int32_t type;
    float* dvals;
};

// How the gradients are computed: `parts` of N one by one, whose sums of all entries are joined afterwards; `group` of them at a time, so that their sums do not grow with N.
enum ValuesKernel { kValuesFew, kValuesEntries, kValuesTiles };
constexpr int values_tile_cols(bool large) { return large ? 256 : 128; }
struct ValuesPlan {
    ValuesKernel kernel;
    int32_t parts, group;
    int32_t pieces;        // kValuesEntries: pieces of 16 bytes of a lane; kValuesTiles: 4 for tiles of 256 x 256, 2 of 128 x 128
    bool one;              // a wave has one row of A, not four
    bool any;              // B by addresses in 64 bits
    int64_t starts;        // kValuesTiles: words for where the tiles of a row begin
    int64_t ldw;           // not 0: B is copied first, to rows that many elements apart
};
ValuesPlan values_plan(int64_t m, int64_t k, int64_t nnz, int64_t N, int type, const void* B, int64_t ldb);
// starts: plan.starts words; part: group x nnz sums where there is more than one part; copy: k x ldw elements where ldw is not 0
hipError_t launch_grad_values(const GradValuesArgs& a, const ValuesPlan& plan, int32_t* starts, float* part, void* copy, hipStream_t s);

}  // namespace gcoo
