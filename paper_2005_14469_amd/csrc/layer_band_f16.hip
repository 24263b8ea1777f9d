// The sixteen-wave product with its epilogue, f16.
#include "layer_band.hpp"

namespace gcoo {
hipError_t launch_layer_band_f16(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s) { return launch_layer_band_of<f16_t>(a, rows, e, s); }
}  // namespace gcoo
