// The sixteen-wave product with its epilogue, f32.
#include "layer_band.hpp"

namespace gcoo {
hipError_t launch_layer_band_f32(const BandArgs& a, const RowsArgs& rows, const EpilogueArgs& e, hipStream_t s) { return launch_layer_band_of<float>(a, rows, e, s); }
}  // namespace gcoo
