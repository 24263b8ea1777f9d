// The norm of many gradients and their scaling to a given one, and its launcher.
//
// Two passes over pieces of 4096 elements: a workgroup sums the squares of a stretch of pieces, then every workgroup adds up the sums of all (in one order, so that the bits are the same in
// each of them and on every run, without a launch between the two) and scales its stretch.  Squares and sums are in 64 bits: the square of an fp32 number is exact there, and a sum can
// neither overflow nor lose what a long fp32 sum does.
//
// Bound: memory (150 million elements in 60 tensors, fp32: 327 us; reading them twice and storing them once would take 367 at the rate of a large copy).  The second pass goes through the pieces from the last to the first, so that it begins with what the memory-side cache (256 MB) still has of the first pass, and stores past the caches.
// The tensors go with the launches, as arguments: nothing is copied to the device, and a captured call holds them itself.
#include "gcoo_layer_clip.hpp"
#include "gcoo_layer_io.hpp"

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

// f(tensor, first element, elements) for the pieces [from, to); DOWN: from the last to the first.
template <bool DOWN, typename F>
__device__ __forceinline__ void clip_stretch(const ClipList& l, int32_t from, int32_t to, F&& f)
{
    if (from >= to) return;
    int x = clip_tensor(l, DOWN ? to - 1 : from);
    for (int32_t i = 0; i < to - from; ++i) {
        const int32_t piece = DOWN ? to - 1 - i : from + i;
        if (DOWN) { while (l.t[x].first > piece) --x; }
        else { while (x + 1 < l.tensors && l.t[x + 1].first <= piece) ++x; }
        const int64_t at = (int64_t)(piece - l.t[x].first) * kClipPiece, left = l.t[x].count - at;
        f(l.t[x], at, (int)(left < kClipPiece ? left : kClipPiece));
    }
}

// the same for the pieces of the workgroup; DOWN: the workgroups from the last to the first, too
template <bool DOWN, typename F>
__device__ __forceinline__ void clip_pieces(const ClipList& l, F&& f)
{
    const int32_t wg = DOWN ? l.wgs - 1 - (int32_t)blockIdx.x : (int32_t)blockIdx.x;
    clip_stretch<DOWN>(l, (int32_t)((int64_t)l.pieces * wg / l.wgs), (int32_t)((int64_t)l.pieces * (wg + 1) / l.wgs), f);
}

template <typename T> constexpr int kClipVec = 16 / sizeof(T);
template <typename T, int THREADS> constexpr int kClipSteps = kClipPiece / (THREADS * kClipVec<T>);       // 16-byte pieces of a thread

// `t`: the thread's place among THREADS of them
template <int THREADS, typename T>
__device__ __forceinline__ double clip_squares(const T* x, int n, int t)
{
    constexpr int V = kClipVec<T>;
    double sum = 0.0;
    float v[kClipSteps<T, THREADS>][V];
#pragma unroll
    for (int s = 0; s < kClipSteps<T, THREADS>; ++s) {
        const int at = (s * THREADS + t) * V;
        if (at + V <= n) layer_load<T, V>(x, at, v[s]);
        else
#pragma unroll
            for (int u = 0; u < V; ++u) v[s][u] = at + u < n ? widen(x[at + u]) : 0.0f;
    }
#pragma unroll
    for (int s = 0; s < kClipSteps<T, THREADS>; ++s)
#pragma unroll
        for (int u = 0; u < V; ++u) sum = __builtin_fma((double)v[s][u], (double)v[s][u], sum);
    return sum;
}
template <int THREADS>
__device__ __forceinline__ double clip_squares_of(const ClipTensor& t, int64_t at, int n, int thread)
{
    if (t.type == GCOO_F32) return clip_squares<THREADS>(static_cast<const float*>(t.data) + at, n, thread);
    if (t.type == GCOO_BF16) return clip_squares<THREADS>(static_cast<const bf16_t*>(t.data) + at, n, thread);
    return clip_squares<THREADS>(static_cast<const f16_t*>(t.data) + at, n, thread);
}

template <int WAVES>
__device__ __forceinline__ double clip_block_sum(double sum, double* part)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < WAVES; ++w) sum += part[w];
    return sum;
}

__global__ __launch_bounds__(kClipThreads) void clip_sum(ClipList l, double* sums)
{
    __shared__ double part[kClipThreads / 64];
    double sum = 0.0;
    clip_pieces<false>(l, [&](const ClipTensor& t, int64_t at, int n) { sum += clip_squares_of<kClipThreads>(t, at, n, (int)threadIdx.x); });
    sum = clip_block_sum<kClipThreads / 64>(sum, part);
    if (threadIdx.x == 0) sums[l.sum0 + (int32_t)blockIdx.x] = sum;
}

// (x may be y: a thread loads what it stores itself)
template <int THREADS, typename T, typename F>
__device__ __forceinline__ void clip_scaled(const void* data, void* out, int64_t first, int n, F factor, int t)
{
    constexpr int V = kClipVec<T>;
    const T* x = static_cast<const T*>(data) + first;
    T* y = static_cast<T*>(out) + first;
    float v[kClipSteps<T, THREADS>][V];
#pragma unroll
    for (int s = 0; s < kClipSteps<T, THREADS>; ++s) {
        const int at = (s * THREADS + t) * V;
        if (at + V <= n) layer_load<T, V>(x, at, v[s]);
        else
#pragma unroll
            for (int u = 0; u < V; ++u) v[s][u] = at + u < n ? widen(x[at + u]) : 0.0f;
    }
#pragma unroll
    for (int s = 0; s < kClipSteps<T, THREADS>; ++s) {
        const int at = (s * THREADS + t) * V;
#pragma unroll
        for (int u = 0; u < V; ++u) v[s][u] = (float)(v[s][u] * factor);
        if (at + V <= n) layer_store<T, V>(y, at, v[s]);
        else
#pragma unroll
            for (int u = 0; u < V; ++u)
                if (at + u < n) y[at + u] = narrow<T>(v[s][u]);
    }
}

// What the norm of all says is to be done.  Finite elements may have a norm that fp32 has no number for, or a factor that it has none for, or one of few bits: then, which is seldom, both are in 64 bits (`wide`).
struct ClipFactor {
    bool scales, wide;
    float f;
    double norm, max_norm;
    __device__ __forceinline__ ClipFactor(double norm64, float most) : norm(norm64), max_norm(most)
    {
        const float n = (float)norm64;
        scales = !(most >= n + 1e-6f);                              // (a NaN scales)
        f = scales ? most / (n + 1e-6f) : 1.0f;
        wide = scales && f < 0x1p-100f && most > 0.0f && norm64 < (double)INFINITY;
    }
    template <int THREADS, typename F>
    __device__ __forceinline__ void apply(const ClipTensor& t, int64_t at, int n, F factor, int thread) const
    {
        if (!scales && t.data == t.out) return;
        if (t.type == GCOO_F32) clip_scaled<THREADS, float>(t.data, t.out, at, n, factor, thread);
        else if (t.type == GCOO_BF16) clip_scaled<THREADS, bf16_t>(t.data, t.out, at, n, factor, thread);
        else clip_scaled<THREADS, f16_t>(t.data, t.out, at, n, factor, thread);
    }
    // each(g): g(tensor, first element, elements) for what the thread has a part in
    template <int THREADS, typename E>
    __device__ __forceinline__ void all(int thread, E&& each) const
    {
        if (__builtin_expect(wide, 0)) {
            const double factor = max_norm / (norm + 1e-6);
            each([&](const ClipTensor& t, int64_t at, int n) { apply<THREADS>(t, at, n, factor, thread); });
        } else {
            each([&](const ClipTensor& t, int64_t at, int n) { apply<THREADS>(t, at, n, f, thread); });
        }
    }
};

__global__ __launch_bounds__(kClipThreads) void clip_scale(ClipList l, const double* sums, int32_t sums_all, float max_norm, float* norm_out)
{
    __shared__ double part[kClipThreads / 64];
    double sum = 0.0;
    for (int32_t i = threadIdx.x; i < sums_all; i += kClipThreads) sum += sums[i];
    const double norm = sqrt(clip_block_sum<kClipThreads / 64>(sum, part));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    ClipFactor(norm, max_norm).all<kClipThreads>((int)threadIdx.x, [&](auto&& f) { clip_pieces<true>(l, f); });
}

// A few pieces: one workgroup, whose quarters take a stretch each, and one launch (us, two launches and so, fp32: 2000 elements: 7.3 5.5; 16384: 6.6 5.4; 24576: 6.7 6.5; 49152: 6.9 9.3).
__global__ __launch_bounds__(kClipSmallThreads) void clip_small(ClipList l, float max_norm, float* norm_out)
{
    __shared__ double part[kClipSmallThreads / 64];
    constexpr int GROUPS = kClipSmallThreads / kClipThreads;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / kClipThreads), t = (int)threadIdx.x % kClipThreads;
    const int32_t from = l.pieces * group / GROUPS, to = l.pieces * (group + 1) / GROUPS;
    double sum = 0.0;
    clip_stretch<false>(l, from, to, [&](const ClipTensor& x, int64_t at, int n) { sum += clip_squares_of<kClipThreads>(x, at, n, t); });
    const double norm = sqrt(clip_block_sum<kClipSmallThreads / 64>(sum, part));
    if (threadIdx.x == 0) *norm_out = (float)norm;
    ClipFactor(norm, max_norm).all<kClipThreads>(t, [&](auto&& f) { clip_stretch<true>(l, from, to, f); });
}

hipError_t launch_clip_small(const ClipList& l, float max_norm, float* norm_out, hipStream_t s)
{
    clip_small<<<dim3(1), dim3(kClipSmallThreads), 0, s>>>(l, max_norm, norm_out);
    return hipGetLastError();
}
hipError_t launch_clip_sum(const ClipList& l, double* sums, hipStream_t s)
{
    clip_sum<<<dim3((unsigned)l.wgs), dim3(kClipThreads), 0, s>>>(l, sums);
    return hipGetLastError();
}
hipError_t launch_clip_scale(const ClipList& l, const double* sums, int32_t sums_all, float max_norm, float* norm_out, hipStream_t s)
{
    clip_scale<<<dim3((unsigned)l.wgs), dim3(kClipThreads), 0, s>>>(l, sums, sums_all, max_norm, norm_out);
    return hipGetLastError();
}

}  // namespace gcoo
