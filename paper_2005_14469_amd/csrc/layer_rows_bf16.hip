// The row-by-row product with its epilogue, bf16.
#include "gcoo_layer_rows.hpp"

namespace gcoo {
hipError_t launch_layer_rows_bf16(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s) { return launch_layer_rows_of<bf16_t>(a, e, s); }
}  // namespace gcoo
