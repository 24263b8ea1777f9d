// The gradient of the stored weights (a scalar product of two rows for each entry), and its launcher.
#include "gcoo_layer.hpp"
#include "gcoo_layer_device.hpp"

namespace gcoo {

constexpr int kValuesThreads = 256;

// A wave per row of A, its lanes along N, one entry after the other.
template <typename T>
__global__ __launch_bounds__(kValuesThreads) void layer_values(GradValuesArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * (kValuesThreads / 64) + (threadIdx.x >> 6);
    if (r >= a.A.m) return;
    const T* z = static_cast<const T*>(a.dZ) + r * a.lddz;
    const uint32_t kmax = (uint32_t)(a.A.k - 1);
    for (int32_t e = a.A.start[r], end = a.A.start[r + 1]; e < end; ++e) {
        const uint32_t c = (uint32_t)a.A.cols[e];
        const T* b = static_cast<const T*>(a.B) + (int64_t)(c < kmax ? c : kmax) * a.ldb;
        float sum = 0.0f;
        for (int64_t j = lane; j < a.N; j += 64) sum = __builtin_fmaf(widen(z[j]), widen(b[j]), sum);
        sum = wave_sum(sum);
        if (lane == 0) a.dvals[e] = sum;
    }
}

hipError_t launch_grad_values(const GradValuesArgs& a, hipStream_t s)
{
    constexpr int64_t rows = kValuesThreads / 64;
    return with_type(a.type, [&](auto t) {
        layer_values<decltype(t)><<<dim3((unsigned)((a.A.m + rows - 1) / rows)), dim3(kValuesThreads), 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace gcoo
