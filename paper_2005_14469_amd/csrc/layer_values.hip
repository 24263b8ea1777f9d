// The gradient of the stored weights, dvals[e] = sum over n of dZ(row of e, n) B(column of e, n): its kernels and the choice among them.
#include "gcoo_layer_values.hpp"
#include "gcoo_layer_device.hpp"

#include <type_traits>

namespace gcoo {

// ---- from the caches: entry by entry ----
//
// Sixteen lanes (a slot) are on a row of A: each holds P pieces of 16 bytes of the row of dZ in registers, in fp32, and takes the same pieces of the row of B of every entry, so that an
// entry costs P loads and 16 lanes x P pieces of multiply-adds.  Sixteen entries leave sixteen partial sums in every lane; they are added up by exchanging halves (the
// lanes that keep the upper eight sums give the lower eight to those that keep these, and so on), 45 instructions for sixteen entries instead of 128, after which lane i holds the sum of entry i.
// A wave has four rows beside each other, or all four slots on one row where it is long or rows are few.
//
// Bound: the vector caches, through which every entry takes its stretch of B.  The columns of B are cut into tiles of 256 P bytes that stay in an XCD's L2 (4 MB) for as many
// rows as A has columns; the sums of a tile go to `work` and values_join adds them in the order of the tiles.
template <int I>
__device__ __forceinline__ uint32_t slot_bcast(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x150 + I, 0xf, 0xf, true); }      // row_newbcast:I

template <int CTRL>
__device__ __forceinline__ float lane_of(float x) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true)); }

// sums[i] of the slot's lanes -> the sum of all of sums[lane], in lane `lane` of the slot
template <int HALF, int CTRL>
__device__ __forceinline__ void exchange(float (&x)[16], int lane)
{
    const bool upper = lane & HALF;
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
        const float keep = upper ? x[i + HALF] : x[i], give = upper ? x[i] : x[i + HALF];
        x[i] = keep + lane_of<CTRL>(give);
    }
}
__device__ __forceinline__ float slot_sums(float (&x)[16], int lane)
{
    exchange<8, 0x140>(x, lane);          // row_mirror: lane ^ 15
    exchange<4, 0x141>(x, lane);          // row_half_mirror: lane ^ 7
    exchange<2, 0x1b>(x, lane);           // quad_perm [3,2,1,0]: lane ^ 3
    exchange<1, 0xb1>(x, lane);           // quad_perm [1,0,3,2]: lane ^ 1
    return x[0];
}

template <typename T> struct Piece {
    static constexpr int kElements = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(kElements)));
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// B for a tile: by a buffer descriptor, or (ANY) by addresses in 64 bits, which serve a B of 4 GB and more and elements at odd places.
struct ValuesB {
    __amdgpu_buffer_rsrc_t rsrc;
    const char* base;
    uint64_t pitch;
};
constexpr uint32_t kNowhere = 0xfffff000u;         // beyond every descriptor, as is a lane's place in the tile added to it

// A lane's pieces: piece q begins at byte at[q] of the tile's rows, or is nothing (none[q]: its elements are 0); bits of `keep` say which of its bytes count.
template <typename T, int P>
struct Pieces {
    uint32_t at[P];
    bool none[P];
    u32x4 keep[P];
};

// Entries FROM .. FROM + CNT - 1 of the batch.
template <typename T, int P, bool PART, bool ANY, int FROM, int CNT, int I = 0>
__device__ __forceinline__ void values_load(uint32_t off, const Pieces<T, P>& pc, const ValuesB& B, u32x4 (&b)[CNT * P])
{
    if constexpr (I < CNT) {
        const uint32_t o = slot_bcast<FROM + I>(off);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if constexpr (ANY) {
                b[I * P + q] = 0u;
                if (o != kNowhere && !(PART && pc.none[q])) __builtin_memcpy(&b[I * P + q], B.base + (uint64_t)o * B.pitch + pc.at[q], 16);
            } else {
                b[I * P + q] = __builtin_amdgcn_raw_buffer_load_b128(B.rsrc, (int)(PART && pc.none[q] ? kNowhere : o + pc.at[q]), 0, 0);
            }
        }
        values_load<T, P, PART, ANY, FROM, CNT, I + 1>(off, pc, B, b);
    }
}

template <typename T, int P, bool PART, bool ANY, int FROM, int CNT>
__device__ __forceinline__ void values_batch(uint32_t off, const Pieces<T, P>& pc, const ValuesB& B, const float (&z)[P * Piece<T>::kElements], float (&sums)[16])
{
    constexpr int E = Piece<T>::kElements;
    u32x4 b[CNT * P];
    values_load<T, P, PART, ANY, FROM, CNT>(off, pc, B, b);
#pragma unroll
    for (int i = 0; i < CNT; ++i) {
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < P; ++q) {
            u32x4 w = b[i * P + q];
            if constexpr (PART) w &= pc.keep[q];
            const typename Piece<T>::vec x = __builtin_bit_cast(typename Piece<T>::vec, w);
#pragma unroll
            for (int u = 0; u < E; ++u) s = __builtin_fmaf(z[q * E + u], widen((T)x[u]), s);
        }
        sums[FROM + i] = s;
    }
}

template <typename T, int P, bool PART, bool ANY>
struct ValuesTile {
    static constexpr int E = Piece<T>::kElements, AT_ONCE = P == 1 ? 16 : (P == 2 ? 8 : 4);
    const GradValuesArgs& a;
    float* out;
    Pieces<T, P> pc;
    ValuesB B;
    uint32_t kmax, pitch;
    int64_t j0;
    int lane;
    __device__ __forceinline__ ValuesTile(const GradValuesArgs& args, int32_t tile, float* part) : a(args)
    {
        lane = threadIdx.x & 63;
        j0 = (int64_t)tile * (16 * P * E);
        out = part ? part + (int64_t)tile * a.A.nnz : a.dvals;
        const int64_t N = a.N;
        // (a tile of fewer than E columns begins E in front of N: N is at least E)
        const int64_t first = j0 > N - E ? N - E : j0;
        const char* base = reinterpret_cast<const char*>(static_cast<const T*>(a.B) + first);
        const uint64_t bytes = ((uint64_t)(a.A.k - 1) * (uint64_t)a.ldb + (uint64_t)(N - first)) * sizeof(T);
        if constexpr (!ANY) B.rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)(uint32_t)bytes, 0x00027000);
        B.base = base;
        B.pitch = (uint64_t)a.ldb * sizeof(T);
        pitch = (uint32_t)B.pitch;
        kmax = (uint32_t)(a.A.k - 1);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int64_t want = j0 + (q * 16 + (lane & 15)) * E, begin = want > N - E ? N - E : want;
            pc.none[q] = PART && want >= N;
            pc.at[q] = (uint32_t)(begin - first) * (uint32_t)sizeof(T);
            if constexpr (PART) {
                // a piece that would reach beyond N lies in front of it instead: the elements that another lane has count 0
                const int skip = (int)(want - begin) * (int)sizeof(T);
#pragma unroll
                for (int w = 0; w < 4; ++w) pc.keep[q][w] = skip >= 4 * w + 4 ? 0u : (skip <= 4 * w ? ~0u : ~0u << (8 * (skip - 4 * w)));
            }
        }
    }
    // the row of dZ, in fp32
    __device__ __forceinline__ void row(int64_t r, float (&z)[P * E]) const
    {
        const char* src = reinterpret_cast<const char*>(static_cast<const T*>(a.dZ) + r * a.lddz + (j0 > a.N - E ? a.N - E : j0));
#pragma unroll
        for (int q = 0; q < P; ++q) {
            u32x4 w = 0u;
            if (!(PART && pc.none[q])) __builtin_memcpy(&w, src + pc.at[q], 16);
            if constexpr (PART) w &= pc.keep[q];
            const typename Piece<T>::vec x = __builtin_bit_cast(typename Piece<T>::vec, w);
#pragma unroll
            for (int u = 0; u < E; ++u) z[q * E + u] = widen((T)x[u]);
        }
    }
    __device__ __forceinline__ uint32_t offset(int32_t e, int32_t end) const
    {
        if (e >= end) return kNowhere;
        const uint32_t c = (uint32_t)a.A.cols[e], in = c < kmax ? c : kmax;
        return ANY ? in : in * pitch;
    }
    // The entries beg, beg + step, ... below end by sixteens, for each slot its own (every lane of the wave calls it); `shift`: of the slot inside a step.
    __device__ __forceinline__ void entries(int32_t beg, int32_t end, int32_t step, const float (&z)[P * E]) const
    {
        int32_t e = beg + (lane & 15);
        uint32_t next = offset(e, end);
        while (__any(e - (lane & 15) < end)) {
            const uint32_t off = next;
            const int32_t at = e;
            e += step;
            next = offset(e, end);
            float sums[16];
            if constexpr (AT_ONCE == 16) values_batch<T, P, PART, ANY, 0, 16>(off, pc, B, z, sums);
            else if constexpr (AT_ONCE == 8) {
                values_batch<T, P, PART, ANY, 0, 8>(off, pc, B, z, sums);
                values_batch<T, P, PART, ANY, 8, 8>(off, pc, B, z, sums);
            } else {
                values_batch<T, P, PART, ANY, 0, 4>(off, pc, B, z, sums);
                values_batch<T, P, PART, ANY, 4, 4>(off, pc, B, z, sums);
                values_batch<T, P, PART, ANY, 8, 4>(off, pc, B, z, sums);
                values_batch<T, P, PART, ANY, 12, 4>(off, pc, B, z, sums);
            }
            const float s = slot_sums(sums, lane);
            if (at < end) out[at] = s;
        }
    }
    // Rows r0 .. r0 + 3 of which those below `end`; ONE: row r0 by all slots.
    __device__ __forceinline__ void rows(int64_t r0, bool one) const
    {
        const int slot = lane >> 4;
        const int64_t m = a.A.m, r = one ? r0 : r0 + slot;
        int32_t beg = 0, end = 0;
        if (r < m) { beg = a.A.start[r]; end = a.A.start[r + 1]; }
        float z[P * E];
        if (!one) {
            // a row of more entries than the others of the wave together would have them wait: all slots take it
            const int32_t n = end - beg;
            int32_t all = n;
            all += __shfl_xor(all, 16, 64);
            all += __shfl_xor(all, 32, 64);
            const bool shared = n > 32 && n > 2 * (all - n);
            row(r < m ? r : m - 1, z);
            entries(beg, shared ? beg : end, 16, z);
            uint64_t todo = __ballot(shared && (lane & 15) == 0);
            while (todo) {                                       // wave-uniform
                const int s = (__ffsll((long long)todo) - 1) >> 4;
                todo &= todo - 1;
                const int32_t lb = __builtin_amdgcn_readlane(beg, 16 * s), le = __builtin_amdgcn_readlane(end, 16 * s);
                row(r0 + s, z);
                entries(lb + 16 * slot, le, 64, z);
            }
            return;
        }
        row(r < m ? r : m - 1, z);
        entries(beg + 16 * slot, end, 64, z);
    }
};

template <typename T, int P, bool ANY>
__global__ __launch_bounds__(kValuesThreads) void values_entries(GradValuesArgs a, float* part, int32_t tiles, int32_t row_wgs, int32_t one)
{
    // an XCD walks all rows of one tile before the next, eight tiles side by side; the tiles beyond the last whole eight are cut into eight slices of rows
    const int32_t block = (int32_t)blockIdx.x, xcd = block & 7, at = block >> 3, eights = tiles / 8;
    int32_t tile, wg;
    if (at < eights * row_wgs) {
        tile = at / row_wgs * 8 + xcd;
        wg = at - at / row_wgs * row_wgs;
    } else {
        const int32_t rest = (tiles - eights * 8) * row_wgs, slice = (rest + 7) / 8, x = at - eights * row_wgs, i = xcd * slice + x;
        if (x >= slice || i >= rest) return;
        tile = eights * 8 + i / row_wgs;
        wg = i - i / row_wgs * row_wgs;
    }
    const int64_t wave = (int64_t)wg * (kValuesThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r0 = one ? wave : 4 * wave;
    if (r0 >= a.A.m) return;
    if ((int64_t)(tile + 1) * (16 * P * Piece<T>::kElements) > a.N) ValuesTile<T, P, true, ANY>(a, tile, part).rows(r0, one);
    else ValuesTile<T, P, false, ANY>(a, tile, part).rows(r0, one);
}

// ---- few columns: a lane per entry ----
//
// Up to 64 bytes of a row: sixteen lanes on a row of A, each on every sixteenth entry, the row of dZ in registers of all of them.
template <typename T, int MOST>
__global__ __launch_bounds__(kValuesThreads) void values_few(GradValuesArgs a)
{
    const int64_t r = (int64_t)blockIdx.x * (kValuesThreads / 16) + (threadIdx.x >> 4);
    if (r >= a.A.m) return;
    const int N = (int)a.N;
    const T* src = static_cast<const T*>(a.dZ) + r * a.lddz;
    float z[MOST];
#pragma unroll
    for (int j = 0; j < MOST; ++j) z[j] = j < N ? widen(src[j]) : 0.0f;
    const uint32_t kmax = (uint32_t)(a.A.k - 1);
    const int32_t end = a.A.start[r + 1];
    for (int32_t e = a.A.start[r] + (int32_t)(threadIdx.x & 15); e < end; e += 16) {
        const uint32_t c = (uint32_t)a.A.cols[e];
        const T* b = static_cast<const T*>(a.B) + (int64_t)(c < kmax ? c : kmax) * a.ldb;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < MOST; ++j)
            if (j < N) s = __builtin_fmaf(z[j], widen(b[j]), s);
        a.dvals[e] = s;
    }
}

// ---- dvals[e] = the sums of the tiles or parts, in their order ----
__global__ __launch_bounds__(kValuesThreads) void values_join(const float* __restrict__ part, float* __restrict__ dvals, int64_t nnz, int32_t parts)
{
    const int64_t e = (int64_t)blockIdx.x * kValuesThreads + threadIdx.x;
    if (e >= nnz) return;
    float s = part[e];
#pragma unroll 8
    for (int32_t i = 1; i < parts; ++i) s += part[(int64_t)i * nnz + e];
    dvals[e] = s;
}

// ---- launches ----

template <typename T, int P>
static hipError_t launch_entries(const GradValuesArgs& a, const ValuesPlan& plan, float* part, hipStream_t s)
{
    constexpr int64_t waves = kValuesThreads / 64;
    const int64_t rows = plan.one ? waves : 4 * waves, row_wgs = (a.A.m + rows - 1) / rows, tiles = plan.parts;
    const int64_t rest = tiles % 8 * row_wgs, grid = tiles / 8 * 8 * row_wgs + (rest + 7) / 8 * 8;
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const auto kernel = plan.any ? values_entries<T, P, true> : values_entries<T, P, false>;
    kernel<<<dim3((unsigned)grid), dim3(kValuesThreads), 0, s>>>(a, tiles > 1 ? part : nullptr, (int32_t)tiles, (int32_t)row_wgs, plan.one ? 1 : 0);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_few(const GradValuesArgs& a, hipStream_t s)
{
    constexpr int64_t rows = kValuesThreads / 16;
    const dim3 grid((unsigned)((a.A.m + rows - 1) / rows)), threads(kValuesThreads);
    constexpr int most = 64 / sizeof(T);
    if (a.N <= 1) values_few<T, 1><<<grid, threads, 0, s>>>(a);
    else if (a.N <= 4) values_few<T, 4><<<grid, threads, 0, s>>>(a);
    else if (a.N <= most / 2) values_few<T, most / 2><<<grid, threads, 0, s>>>(a);
    else values_few<T, most><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

ValuesPlan values_plan(int64_t m, int64_t k, int64_t nnz, int64_t N, int type, const void* B, int64_t ldb)
{
    (void)nnz;
    const int64_t size = (int64_t)type_bytes(type), bytes = N * size;
    ValuesPlan p{kValuesFew, 1, 1, false, false};
    if (bytes <= 64) return p;
    p.kernel = kValuesEntries;
    p.any = (uint64_t)k * (uint64_t)ldb * (uint64_t)size > kRowsMaxBytes || reinterpret_cast<uintptr_t>(B) % 4 != 0 || ldb * size % 4 != 0 || bytes % 4 != 0;
    p.one = m < 2048;
    if (bytes <= 1024) p.pieces = bytes <= 256 ? 1 : (bytes <= 512 ? 2 : 4);
    else p.pieces = k <= 3000 ? 4 : (k <= 6000 ? 2 : 1);
    p.parts = (int32_t)((bytes + 256 * p.pieces - 1) / (256 * p.pieces));
    return p;
}

hipError_t launch_grad_values(const GradValuesArgs& a, const ValuesPlan& plan, float* part, hipStream_t s)
{
    if (plan.kernel == kValuesFew) return with_type(a.type, [&](auto t) { return launch_few<decltype(t)>(a, s); });
    hipError_t e = with_type(a.type, [&](auto t) {
        typedef decltype(t) T;
        return plan.pieces == 1 ? launch_entries<T, 1>(a, plan, part, s) : (plan.pieces == 2 ? launch_entries<T, 2>(a, plan, part, s) : launch_entries<T, 4>(a, plan, part, s));
    });
    if (e != hipSuccess || plan.parts == 1) return e;
    values_join<<<dim3((unsigned)((a.A.nnz + kValuesThreads - 1) / kValuesThreads)), dim3(kValuesThreads), 0, s>>>(part, a.dvals, a.A.nnz, plan.parts);
    return hipGetLastError();
}

}  // namespace gcoo
