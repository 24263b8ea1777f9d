// The product with its epilogue for a few tokens: B, or as many columns of it as fit, held in LDS, a row of it in one read; and its launcher.
//
// A matrix-vector product and those a little wider read every entry for a few multiply-adds, so the entries should come from memory as fast as it gives them, and everything else stay out of their way.  From the
// vector cache the elements of B, which lie anywhere, take a clock of the compute unit for every lane.  Here a workgroup of sixteen waves brings N columns of B (1, 2, 4 or 8, 16 bytes of a row at the most) to LDS
// first, the rows of B one behind the other, and takes the N elements of an entry with one read of LDS: 64 lanes theirs in five to nine clocks.
//
//   slot      64 lanes on a row of A, or 16 where rows are short; a lane takes four adjacent entries at a time with one load each of columns and values, GROUPS such on their way
//   sums      N per lane; they are added up by exchanging halves (lanes that keep the upper N/2 give the lower N/2 to their partners), after which the sums of the N columns lie in N groups
//             of lanes, one lane of each of which does the epilogue of its element
//   ends      what is behind the end of a row has the value 0 and a row of zeros behind B as its row of B
//   long rows the whole workgroup on a row, behind its own rows
//   tiles     more than N columns: several tiles, those of the same rows beside each other on one XCD, so that the entries come from memory once
//
// Bound: the entries, where one tile does (8000 x 8000, 10 %, one token, bf16: 13.3 us behind cold caches, of which reading the entries once at the rate of a large copy takes 10.4; from the vector cache 21).  Four groups of
// entries on their way, not two, leave no room for a second workgroup or spill: 10000 x 2000, 8 %, one token: 9.6 10.7.
#include "gcoo_layer_held.hpp"
#include "gcoo_layer_io.hpp"
#include "gcoo_layer_long.hpp"

namespace gcoo {

constexpr int kHeldThreads = 1024;

template <typename T, int LANES, int N>
__global__ __launch_bounds__(kHeldThreads, N == 8 ? 4 : 8) void layer_held(RowsArgs a, EpilogueArgs e, int32_t tiles, int32_t wgs, int32_t rows)
{
    constexpr int SLOTS = kHeldThreads / LANES, GROUPS = 2, V = 16 / sizeof(T);
    const int32_t block = (int32_t)(blockIdx.x >> 3), tile = block % tiles, wg = block / tiles * 8 + (int32_t)(blockIdx.x & 7u);
    if (wg >= wgs) return;                                                 // the whole workgroup
    const int64_t j0 = (int64_t)tile * N;
    const int n = a.N - j0 < N ? (int)(a.N - j0) : N, t = (int)threadIdx.x;
    const uint32_t k = (uint32_t)a.k, lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const T* B = reinterpret_cast<const T*>(a.B) + j0;

    const LongRows longs{a.long_rows, a.long_count, a.long_row, a.long_room};
    LongWalk<1> walk(longs, a.row_ptr, a.m, wg, wgs);

    // the row of these lanes, or, when its own are done, a stretch of the workgroup's long row (unsigned: a step beyond the last of 2^31 entries stays a number)
    bool shares = false;
    int64_t r = ((int64_t)wg * rows) * SLOTS + slot;
    uint32_t beg = 0, end = 0;
    auto bounds = [&] {
        beg = end = 0;
        if (r >= a.m) return;
        beg = (uint32_t)a.row_ptr[r];
        end = (uint32_t)a.row_ptr[r + 1];
        if (shares) {
            const uint32_t each = (end - beg + SLOTS - 1) / SLOTS;
            beg += slot * each;
            end = beg + each < end ? beg + each : end;
        }
    };
    bounds();

    extern __shared__ __attribute__((aligned(16))) char held_smem[];
    typedef T vec __attribute__((ext_vector_type(N)));
    vec* held = reinterpret_cast<vec*>(held_smem);
    if (n == N && a.ldb == N) {
        // (the last bytes of B by elements)
        const uint32_t all = k * N, vecs = all / V;
        for (uint32_t i = t; i < vecs; i += kHeldThreads) {
            const typename Adjacent<T, V>::vec x = *reinterpret_cast<const typename Adjacent<T, V>::vec*>(B + i * V);
            typedef T piece16 __attribute__((ext_vector_type(V)));
            *reinterpret_cast<piece16*>(reinterpret_cast<T*>(held) + i * V) = x;
        }
        for (uint32_t i = vecs * V + t; i < all; i += kHeldThreads) reinterpret_cast<T*>(held)[i] = B[i];
    } else {
        for (uint32_t c = t; c < k; c += kHeldThreads) {
            vec x = (T)0.0f;
            const T* from = B + (int64_t)c * a.ldb;
            // (columns behind the last lie in what nothing is made of: they may be those of the next row)
            if (n == N || (int64_t)(k - 1 - c) * a.ldb + n >= N) x = *reinterpret_cast<const typename Adjacent<T, N>::vec*>(from);
            else
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (j < n) x[j] = from[j];
            held[c] = x;
        }
    }
    if (t == 0) held[k] = (T)0.0f;
    __syncthreads();

    // the column whose sum this lane comes to hold
    int col = 0;
#pragma unroll
    for (int h = N / 2, d = LANES / 2; h >= 1; h /= 2, d /= 2) col += lane & d ? h : 0;
    const bool owner = (lane & (LANES / N - 1)) == 0 && col < n;

    typedef uint32_t cols4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef float vals4 __attribute__((ext_vector_type(4), aligned(4)));
    for (int32_t row = 0;;) {
        const bool own = !shares && r < a.m && (int32_t)(end - beg) <= a.long_row;
        if (!shares && !own) end = beg;
        float res[1];
        layer_residual<T, 1>(e, r, j0 + col, 0, 1, own && owner, res);
        float bias = own && owner && e.bias ? e.bias[r] : 0.0f;

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
                    for (int q = 0; q < 4; ++q) { c[g][q] = x[q] < k ? x[q] : k - 1; v[g][q] = y[q]; }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const bool in = at + q < end;
                        const uint32_t x = in ? (uint32_t)a.cols[at + q] : 0u;
                        c[g][q] = in ? (x < k ? x : k - 1) : k;
                        v[g][q] = in ? a.vals[at + q] : 0.0f;
                    }
                }
            }
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const vec b = held[c[g][q]];
#pragma unroll
                    for (int j = 0; j < N; ++j) sum[j] = __builtin_fmaf(v[g][q], widen((T)b[j]), sum[j]);
                }
        }
#pragma unroll
        for (int h = N / 2, d = LANES / 2; h >= 1; h /= 2, d /= 2)
#pragma unroll
            for (int j = 0; j < h; ++j) {
                const bool upper = lane & d;
                const float keep = upper ? sum[j + h] : sum[j], give = upper ? sum[j] : sum[j + h];
                sum[j] = keep + __shfl_xor(give, d, LANES);
            }
#pragma unroll
        for (int d = LANES / N / 2; d >= 1; d >>= 1) sum[0] += __shfl_xor(sum[0], d, LANES);

        if (shares) {
            __shared__ float part[SLOTS][N];
            if ((lane & (LANES / N - 1)) == 0) part[slot][col] = sum[0];
            __syncthreads();
            if (slot == 0 && owner)
                for (int w = 1; w < SLOTS; ++w) sum[0] += part[w][col];
            __syncthreads();
            if (slot == 0 && owner) {
                layer_residual<T, 1>(e, r, j0 + col, 0, 1, true, res);
                bias = e.bias ? e.bias[r] : 0.0f;
            }
        }
        if (owner && (shares ? slot == 0 : own)) {
            float x[1] = {sum[0]};
            layer_finish<T, 1>(e, bias, r, j0 + col, 0, 1, x, res);
        }
        if (++row < rows) r += SLOTS;
        else {
            shares = true;
            int32_t long_row, piece;
            if (!walk.next(&long_row, &piece)) return;
            r = long_row;
        }
        bounds();
    }
}

int held_cols(int64_t k, int64_t N, int type)
{
    const int64_t size = (int64_t)type_bytes(type);
    int cols = 1;
    while (cols * size < 16 && cols < N && (k + 1) * (2 * cols) * size <= kHeldLdsBytes) cols *= 2;
    return (k + 1) * cols * size <= kHeldLdsBytes ? cols : 0;
}

template <typename T, int LANES, int N>
static hipError_t launch_held(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    constexpr int SLOTS = kHeldThreads / LANES;
    const int64_t lds = (a.k + 1) * N * (int64_t)sizeof(T), tiles = (a.N + N - 1) / N, all = (a.m + SLOTS - 1) / SLOTS;
    // as many workgroups of a tile as an XCD, of 32 compute units, has room for beside those of the other tiles, all of them with as many rows
    const int64_t room = 8 * ((N < 8 && lds <= 78 * 1024 ? 64 : 32) / tiles), rows = (all + room - 1) / (room > 0 ? room : 1), wgs = (all + rows - 1) / rows;
    const int64_t grid = (wgs + 7) / 8 * 8 * tiles;
    if (tiles > 32 || too_wide(grid, kHeldThreads) || rows > INT32_MAX) return hipErrorInvalidConfiguration;
    static LdsLimit limit;
    const hipError_t err = limit.raise(reinterpret_cast<const void*>(&layer_held<T, LANES, N>), (int)kHeldLdsBytes);
    if (err != hipSuccess) return err;
    layer_held<T, LANES, N><<<dim3((unsigned)grid), dim3(kHeldThreads), (size_t)lds, s>>>(a, e, (int32_t)tiles, (int32_t)wgs, (int32_t)rows);
    return hipGetLastError();
}
template <typename T, int LANES>
static hipError_t launch_held(const RowsArgs& a, const EpilogueArgs& e, int cols, hipStream_t s)
{
    switch (cols) {
        case 1: return launch_held<T, LANES, 1>(a, e, s);
        case 2: return launch_held<T, LANES, 2>(a, e, s);
        case 4: return launch_held<T, LANES, 4>(a, e, s);
        case 8:
            if constexpr (sizeof(T) == 2) return launch_held<T, LANES, 8>(a, e, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_layer_held(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    if (a.m < 1 || a.k < 1 || a.N < 1 || a.ldb > 0x3fffffffLL) return hipErrorInvalidValue;
    const int cols = held_cols(a.k, a.N, e.type);
    return with_type(e.type, [&](auto t) {
        typedef decltype(t) T;
        return a.nnz >= 128 * a.m ? launch_held<T, 64>(a, e, cols, s) : launch_held<T, 16>(a, e, cols, s);
    });
}

}  // namespace gcoo
