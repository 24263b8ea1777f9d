// The product with its epilogue by the kernel that works row by row on a tile of B in LDS (gcoo_spdm_tile_kernel.hpp), and its launcher: B comes to LDS in fp32, whatever it is in memory.
// Bound: bank conflicts, as without the epilogue (1777 x 2301, 3 %, N = 1117, fp16, bias, silu, residual and Z: 22 us; fp32 without them 20 to 22).
#include "gcoo_layer_io.hpp"
#include "gcoo_spdm_tile_kernel.hpp"

namespace gcoo {

template <typename T>
struct TileLayer {
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
