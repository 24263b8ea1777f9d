// The product with its epilogue by the kernel that works row by row on a tile of B in LDS (gcoo_spdm_tile_kernel.hpp), and its launcher: B comes to LDS in fp32, or, 32 columns of fp16, as it is.
// Bound: bank conflicts, as without the epilogue (1777 x 2301, 3 %, N = 1117, fp32, without residual and Z: 20 to 22 us).
#include "gcoo_layer_io.hpp"
#include "gcoo_spdm_tile_kernel.hpp"

namespace gcoo {

template <typename T>
struct TileLayer {
    typedef TileFloats In;
    const T* B;
    int64_t ldb;
    const EpilogueArgs& e;
    __device__ __forceinline__ tile_u32x4 piece(int32_t row, int32_t q) const
    {
        float x[4];
        layer_load<T, 4>(B, (int64_t)row * ldb + q * 4, x);
        return {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
    __device__ __forceinline__ void store(const RowsArgs&, int64_t r, int32_t jc, int32_t j0, float (&acc)[4]) const
    {
        float res[4];
        layer_residual<T, 4>(e, r, jc, j0 - jc, 4, true, res);
        layer_finish<T, 4>(e, r, jc, j0 - jc, 4, acc, res);
    }
};

// Tiles of 32 columns of fp16, a row of B 64 bytes in LDS as one of sixteen fp32 ones: half as many reads of LDS, and the multiply-add widens its operand itself (us, fp32 in LDS and so:
// 1777 x 2301, 3 %, N = 1117: 22.4 19.4, 10 %: 49 36; 12000 x 1500, 10 %, N = 512: 76 53).  bf16 would take as many instructions more as it saves.
struct TileHalves {
    static constexpr int kCols = 8;
    typedef tile_u32x4 Read;
    static __device__ __forceinline__ void add(const Read& x, float w, float (&acc)[8])
    {
        typedef f16_t pair __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t word = x[u];
            const pair h = __builtin_bit_cast(pair, word);
            acc[2 * u] = __builtin_fmaf(w, (float)h[0], acc[2 * u]);
            acc[2 * u + 1] = __builtin_fmaf(w, (float)h[1], acc[2 * u + 1]);
        }
    }
};
struct TileLayerHalves {
    typedef TileHalves In;
    const f16_t* B;
    int64_t ldb;
    const EpilogueArgs& e;
    __device__ __forceinline__ tile_u32x4 piece(int32_t row, int32_t q) const
    {
        tile_u32x4 x;
        __builtin_memcpy(&x, B + (int64_t)row * ldb + q * 8, 16);
        return x;
    }
    __device__ __forceinline__ void store(const RowsArgs&, int64_t r, int32_t jc, int32_t j0, float (&acc)[8]) const
    {
        if (j0 - jc >= 8) return;
        float res[8];
        layer_residual<f16_t, 8>(e, r, jc, j0 - jc, 8, true, res);
        layer_finish<f16_t, 8>(e, r, jc, j0 - jc, 8, acc, res);
    }
};
__global__ __launch_bounds__(kTileThreads, 4) void layer_tile_halves(RowsArgs a, EpilogueArgs e, int32_t row_wgs, int32_t rows, int32_t total, int32_t long_steps)
{
    tile_item(a, row_wgs, rows, total, long_steps, [&](int32_t jb) { return TileLayerHalves{reinterpret_cast<const f16_t*>(a.B) + jb, a.ldb, e}; });
}

hipError_t launch_layer_tile_halves(const RowsArgs& a, const EpilogueArgs& e, int64_t row_wgs, bool whole, hipStream_t s)
{
    TileGrid g;
    RowsArgs as4 = a;                                                     // cut as half as many columns of fp32
    as4.N = (a.N + 1) / 2;
    if (e.type != GCOO_F16 || a.N < 2 * kTileCols || a.ldb > 0x3fffffffLL || !tile_grid(as4, row_wgs, whole, &g)) return hipErrorInvalidValue;
    static LdsLimit limit;
    const hipError_t err = limit.raise(reinterpret_cast<const void*>(&layer_tile_halves), (int)kTileLdsBytes);
    if (err != hipSuccess) return err;
    layer_tile_halves<<<dim3((unsigned)((g.total + 7) / 8 * 8)), dim3(kTileThreads), (size_t)g.lds, s>>>(a, e, (int32_t)g.wgs, (int32_t)g.rows, (int32_t)g.total, g.long_steps);
    return hipGetLastError();
}

template <typename T>
__global__ __launch_bounds__(kTileThreads, 4) void layer_tile(RowsArgs a, EpilogueArgs e, int32_t row_wgs, int32_t rows, int32_t total, int32_t long_steps)
{
    tile_item(a, row_wgs, rows, total, long_steps, [&](int32_t jb) { return TileLayer<T>{reinterpret_cast<const T*>(a.B) + jb, a.ldb, e}; });
}

hipError_t launch_layer_tile(const RowsArgs& a, const EpilogueArgs& e, int64_t row_wgs, bool whole, hipStream_t s)
{
    TileGrid g;
    if (a.ldb > 0x3fffffffLL || !tile_grid(a, row_wgs, whole, &g)) return hipErrorInvalidValue;
    return with_type(e.type, [&](auto t) {
        typedef decltype(t) T;
        static LdsLimit limit;
        const hipError_t err = limit.raise(reinterpret_cast<const void*>(&layer_tile<T>), (int)kTileLdsBytes);
        if (err != hipSuccess) return err;
        layer_tile<T><<<dim3((unsigned)((g.total + 7) / 8 * 8)), dim3(kTileThreads), (size_t)g.lds, s>>>(a, e, (int32_t)g.wgs, (int32_t)g.rows, (int32_t)g.total, g.long_steps);
        return hipGetLastError();
    });
}

}  // namespace gcoo
