// The SpDM kernel that works row by row on a tile of B in LDS, and its launcher.
#include "gcoo_spdm_tile_kernel.hpp"

namespace gcoo {

__global__ __launch_bounds__(kTileThreads, 8) void spdm_rows_tile(RowsArgs a, int32_t row_wgs, int32_t rows, int32_t total, int32_t long_steps)
{
    tile_item(a, row_wgs, rows, total, long_steps, [&](int32_t jb) { return TilePlain(a, jb); });
}

bool tile_grid(const RowsArgs& a, int64_t row_wgs, bool whole, TileGrid* g)
{
    if (a.m < 1 || a.k < 1 || a.N < kTileCols || row_wgs < 1 || a.nnz > kTileMaxNnz) return false;
    const int64_t tiles = (a.N + kTileCols - 1) / kTileCols, rows = (a.m + row_wgs - 1) / row_wgs, wgs = (a.m + rows - 1) / rows, total = tiles * wgs;
    const int64_t lds = tile_lds(a.k, rows);
    if (rows > kTileMaxRows || lds > kTileLdsBytes || total > 0x7ffffff0LL) return false;
    // A row of three times the mean keeps its slot busy while the others of the wave have ended; rows of the open bin are not put in order among each other.
    const int64_t steps = (3 * (a.nnz / a.m) + 64) / 4;
    *g = {rows, wgs, total, lds, (int32_t)(whole ? -1 : (steps < kTileBins - 2 ? steps : kTileBins - 2))};
    return true;
}

hipError_t launch_spdm_rows_tile(const RowsArgs& a, int64_t row_wgs, bool whole, hipStream_t s)
{
    TileGrid g;
    if ((uint64_t)a.k * (uint64_t)a.ldb * 4u > kRowsMaxBytes || !tile_grid(a, row_wgs, whole, &g)) return hipErrorInvalidValue;
    static LdsLimit limit;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(&spdm_rows_tile), (int)kTileLdsBytes);
    if (e != hipSuccess) return e;
    spdm_rows_tile<<<dim3((unsigned)((g.total + 7) / 8 * 8)), dim3(kTileThreads), (size_t)g.lds, s>>>(a, (int32_t)g.wgs, (int32_t)g.rows, (int32_t)g.total, g.long_steps);
    return hipGetLastError();
}

}  // namespace gcoo
