// Launch interface of the clipping of gradients (layer_clip.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gcoo {

constexpr int kClipThreads = 256;
constexpr int64_t kClipPiece = 4096;           // elements of a tensor; a workgroup takes a stretch of pieces
constexpr int kClipSmallThreads = 1024;
constexpr int kClipSmallPieces = 6;            // at the most, for one workgroup to do it all
constexpr int kClipTensors = 80;               // of one launch: their descriptions are its arguments
constexpr int64_t kClipSums = 2048;            // workgroups of all launches together, about: each leaves a sum, and each adds up all of them

struct ClipTensor {
    const void* data;
    void* out;
    int64_t count;
    int32_t type;
    int32_t first;                             // its first piece among those of the launch
};
struct ClipList {
    ClipTensor t[kClipTensors];                // none of them empty
    int32_t tensors, pieces;
    int32_t wgs, sum0;                         // workgroups of the launch, and of the launches before
};
// a list of kClipSmallPieces pieces at the most, none among them: all of it
hipError_t launch_clip_small(const ClipList& l, float max_norm, float* norm_out, hipStream_t s);
// sums[sum0 + i] = the squares of workgroup i's pieces
hipError_t launch_clip_sum(const ClipList& l, double* sums, hipStream_t s);
// scales the pieces by the norm that all `sums_all` sums give; norm_out may be null
hipError_t launch_clip_scale(const ClipList& l, const double* sums, int32_t sums_all, float max_norm, float* norm_out, hipStream_t s);

}  // namespace gcoo
