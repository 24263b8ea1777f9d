// The sixteen-wave product with its epilogue, bf16.
#include "layer_band.hpp"

namespace gcoo {
hipError_t launch_layer_band_bf16(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s) { return launch_layer_band_of<bf16_t>(a, rows, e, s); }
}  // namespace gcoo
