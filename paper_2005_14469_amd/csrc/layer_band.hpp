// The sixteen-wave product with its epilogue: the kernel of gcoo_spdm_band_kernel.hpp, whose sums go through LDS to the epilogue; instances by type in layer_band_*.hip.
// Bound: vector instructions, as without the epilogue (8000 x 8000, 10 %, N = 8000, fp32: 2010 us; with bias, gelu, residual and Z, 0.77 GB more: 2171, the kernel alone 2145 to 2200 where pass follows pass).
#pragma once
#include "gcoo_layer_io.hpp"
#include "gcoo_spdm_band_launch.hpp"

namespace gcoo {

// The arguments of the kernel as they lie in memory.
template <typename T>
struct BandLayerArgs {
    BandArgs a;
    RowsArgs rows;
    BandRowsGrid grid;
    LayerIO<float, T> io;
};

// The sums lie in registers that only an instruction can name, 24 or 48 rows of them: with the epilogue behind each the code would not fit the cache.  They go to LDS, to the ten kilobytes that the wave
// itself has fetched bands into (nobody reads them behind the last barrier, and the wave's own requests have landed), ten or twenty rows at a time, and from there row by row.  A lane reads
// what it wrote: no wait for other waves.
template <typename T>
struct BandLayer {
    typedef LayerIO<float, T> Rows;
    static constexpr bool kRowsToo = false;
    template <int V>
    static __device__ __forceinline__ void store(const BandAcc& acc, uint32_t lane_at, uint32_t fillw)
    {
        constexpr int32_t kTile = BandCut<V>::kTile;
        constexpr int kRowBytes = 256 * V, kHalf = kBandFillBytes / kRowBytes, kStride = BandCut<V>::kMaxH + 1;
        typedef const __attribute__((address_space(4))) char* arg_ptr;
        arg_ptr args = (arg_ptr)__builtin_amdgcn_kernarg_segment_ptr();
        uint32_t bid = blockIdx.x;
        asm volatile("" : "+s"(args), "+s"(bid));
        const __attribute__((address_space(4))) BandLayerArgs<T>* z = (const __attribute__((address_space(4))) BandLayerArgs<T>*)args;
        const int32_t blocks = z->a.blocks, item = (int32_t)(bid & 7u) * (int32_t)(z->a.grid >> 3) + (int32_t)(bid >> 3), tile = item / blocks, Q = item - tile * blocks;
        const int32_t N = (int32_t)z->a.N, from = tile * kTile, base = from > N - kTile && N >= kTile ? N - kTile : from;
        const int32_t jc = base + (int32_t)(lane_at >> 2);                 // the lane's first column; it stores those from `from` on
        const int32_t h = z->a.h, row0 = (Q * kBandWaves + (int32_t)(fillw / (uint32_t)kBandFillBytes)) * h, m = (int32_t)z->a.m;
        const int32_t rows = __builtin_amdgcn_readfirstlane(m - row0 < h ? m - row0 : h);
        extern __shared__ __attribute__((aligned(16))) uint32_t band_smem[];
        typedef float vec __attribute__((ext_vector_type(V)));
        char* at = reinterpret_cast<char*>(band_smem) + fillw + lane_at;
#pragma unroll
        for (int c = 0; c < BandCut<V>::kMaxH; c += 2 * kHalf) {
            if (c >= rows) break;
#pragma unroll
            for (int i = 0; i < 2 * kHalf; ++i)
                if (c + i < BandCut<V>::kMaxH) {
                    vec o;
#pragma unroll
                    for (int v = 0; v < V; ++v) o[v] = band_acc_get(acc, v * kStride + c + i);
                    *reinterpret_cast<vec*>(at + (i >= kHalf ? kBandBufferBytes - kHalf * kRowBytes : 0) + i * kRowBytes) = o;
                }
            const int32_t n = rows - c < 2 * kHalf ? rows - c : 2 * kHalf;
            if (jc + V > from && jc < N) {
                char* p = at;
                float ahead[V];                    // what the residual holds in the next row (fp32, 8000 x 8000, 0.5 %, N = 8000, with Z: 560 505 us)
                {
                    EpilogueArgs e;
                    e.residual = z->io.e.residual; e.ldr = z->io.e.ldr;
                    layer_residual<T, V>(e, row0 + c, jc, from - jc, V, true, ahead);
                }
#pragma unroll 1
                for (int i = 0; i < n; ++i) {
                    if (i == kHalf) p += kBandBufferBytes - kHalf * kRowBytes;
                    // (the arguments are read anew for every row: there are no registers to keep them)
                    const __attribute__((address_space(4))) BandLayerArgs<T>* again = z;
                    asm volatile("" : "+s"(again));
                    EpilogueArgs e;
                    e.bias = again->io.e.bias; e.residual = again->io.e.residual; e.ldr = again->io.e.ldr; e.Z = again->io.e.Z; e.ldz = again->io.e.ldz; e.C = again->io.e.C; e.ldc = again->io.e.ldc; e.activation = again->io.e.activation;
                    const vec o = *reinterpret_cast<vec*>(p);
                    p += kRowBytes;
                    float x[V], res[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) x[v] = o[v];
#pragma unroll
                    for (int v = 0; v < V; ++v) res[v] = ahead[v];
                    layer_residual<T, V>(e, row0 + c + i + 1, jc, from - jc, V, i + 1 < n, ahead);
                    layer_finish<T, V>(e, row0 + c + i, jc, from - jc, V, x, res);
                }
            }
        }
    }
};

template <typename T, int V, bool SPREAD, bool LATE>
__global__ __launch_bounds__(64 * kBandWaves) void layer_band(BandArgs a, RowsArgs by_rows, BandRowsGrid rg, LayerIO<float, T> io)
{
    band_item<V, SPREAD, LATE, BandLayer<T>>(a, by_rows, rg, io);
}

// Uneven rows, one by one, in a launch of their own, which ends at once where there are none (2 to 5 us): with both in one kernel the scalar registers do not suffice.  (128 vector registers, and 14 to 18 spilled.)
template <typename T>
__global__ __launch_bounds__(64 * kBandWaves) void layer_rows_all(const uint32_t* uneven, RowsArgs by_rows, BandRowsGrid rg, LayerIO<float, T> io)
{
    __shared__ RowsAllLds lds;
    if (*uneven != 0u) rows_all<16>(by_rows, io, rg.tiles, rg.rpw, rg.wave_row, lds);
}

template <typename T>
struct LayerBand {
    BandLaunch l;
    EpilogueArgs e;
    template <int V, bool SPREAD, bool LATE>
    hipError_t launch(hipStream_t s) const
    {
        static LdsLimit limit;
        const hipError_t err = limit.raise(reinterpret_cast<const void*>(&layer_band<T, V, SPREAD, LATE>), kBandLdsBytes);
        if (err != hipSuccess) return err;
        layer_band<T, V, SPREAD, LATE><<<l.blocks(), dim3(64 * kBandWaves), kBandLdsBytes, s>>>(l.a, l.rows, l.grid, LayerIO<float, T>{e});
        return hipGetLastError();
    }
};

template <typename T>
hipError_t launch_layer_band_of(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s)
{
    LayerBand<T> b;
    const hipError_t err = band_launch(a, rows, &b.l);
    if (err != hipSuccess) return err;
    b.l.rows.moved = 0;                       // (the rows of fp32 sums are not what is stored)
    b.l.grid.tiles = (int32_t)((rows.N + 63) / 64);
    b.e = e;
    layer_rows_all<T><<<dim3(kRowsAllWgs), dim3(64 * kBandWaves), 0, s>>>(a.uneven, b.l.rows, b.l.grid, LayerIO<float, T>{e});
    const hipError_t first = hipGetLastError();
    return first == hipSuccess ? launch_band_kind(b, s) : first;
}

}  // namespace gcoo
