// The norm of many gradients and their scaling to a given one, and its launcher.
//
// Two passes: squares are summed per piece of a tensor, then every workgroup adds up all pieces in their order (so that the bits are the same in each of them and on every
// run, without a launch between the two) and scales its piece.  Squares and sums are in 64 bits: the square of an fp32 number is exact there and its sum can
// neither overflow nor lose what a long fp32 sum does.
//
// The tensors go with the launches, as arguments: nothing is copied to the device, and a captured call holds them itself.
#include "gcoo_layer_clip.hpp"
#include "gcoo_layer_device.hpp"

namespace gcoo {

// The tensor of piece `piece`: the last one that begins at or before it.
__device__ __forceinline__ int clip_tensor(const ClipList& l, int32_t piece)
{
    int lo = 0, hi = l.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (l.t[mid].first <= piece) lo = mid; else hi = mid;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ double clip_squares(const T* x, int64_t n)
{
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kClipThreads) {
        const double v = (double)widen(x[i]);
        sum = __builtin_fma(v, v, sum);
    }
    return sum;
}

__device__ __forceinline__ double clip_block_sum(double sum, double* part)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kClipThreads / 64; ++w) sum += part[w];
    return sum;
}

__global__ __launch_bounds__(kClipThreads) void clip_sum(ClipList l, double* sums)
{
    __shared__ double part[kClipThreads / 64];
    const ClipTensor& t = l.t[clip_tensor(l, (int32_t)blockIdx.x)];
    const int64_t at = (int64_t)((int32_t)blockIdx.x - t.first) * kClipPiece, n = t.count - at < kClipPiece ? t.count - at : kClipPiece;
    double sum;
    if (t.type == GCOO_F32) sum = clip_squares(static_cast<const float*>(t.data) + at, n);
    else if (t.type == GCOO_BF16) sum = clip_squares(static_cast<const bf16_t*>(t.data) + at, n);
    else sum = clip_squares(static_cast<const f16_t*>(t.data) + at, n);
    sum = clip_block_sum(sum, part);
    if (threadIdx.x == 0) sums[l.piece0 + blockIdx.x] = sum;
}

template <typename T>
__device__ __forceinline__ void clip_scaled(const T* x, T* y, int64_t n, float factor)
{
    for (int64_t i = threadIdx.x; i < n; i += kClipThreads) y[i] = narrow<T>(widen(x[i]) * factor);
}

// The workgroups behind those of the list's pieces: none, or one that only writes the norm.
__global__ __launch_bounds__(kClipThreads) void clip_scale(ClipList l, const double* sums, int32_t pieces_all, float max_norm, float* norm_out)
{
    __shared__ double part[kClipThreads / 64];
    double sum = 0.0;
    for (int32_t i = threadIdx.x; i < pieces_all; i += kClipThreads) sum += sums[i];
    const float norm = (float)sqrt(clip_block_sum(sum, part));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    if ((int32_t)blockIdx.x >= l.pieces) return;
    const bool scales = !(max_norm >= norm + 1e-6f);                // (a NaN scales)
    const ClipTensor& t = l.t[clip_tensor(l, (int32_t)blockIdx.x)];
    if (!scales && t.data == t.out) return;
    const int64_t at = (int64_t)((int32_t)blockIdx.x - t.first) * kClipPiece, n = t.count - at < kClipPiece ? t.count - at : kClipPiece;
    const float f = scales ? max_norm / (norm + 1e-6f) : 1.0f;
    if (t.type == GCOO_F32) clip_scaled(static_cast<const float*>(t.data) + at, static_cast<float*>(t.out) + at, n, f);
    else if (t.type == GCOO_BF16) clip_scaled(static_cast<const bf16_t*>(t.data) + at, static_cast<bf16_t*>(t.out) + at, n, f);
    else clip_scaled(static_cast<const f16_t*>(t.data) + at, static_cast<f16_t*>(t.out) + at, n, f);
}

hipError_t launch_clip_sum(const ClipList& l, double* sums, hipStream_t s)
{
    if (l.pieces < 1) return hipSuccess;
    clip_sum<<<dim3((unsigned)l.pieces), dim3(kClipThreads), 0, s>>>(l, sums);
    return hipGetLastError();
}
hipError_t launch_clip_scale(const ClipList& l, const double* sums, int32_t pieces_all, float max_norm, float* norm_out, hipStream_t s)
{
    if (l.pieces < 1 && !norm_out) return hipSuccess;
    clip_scale<<<dim3((unsigned)(l.pieces > 0 ? l.pieces : 1)), dim3(kClipThreads), 0, s>>>(l, sums, pieces_all, max_norm, norm_out);
    return hipGetLastError();
}

}  // namespace gcoo
