// Launch interface of the product that holds B in LDS (layer_held.hip).
#pragma once
#include "gcoo_layer.hpp"

namespace gcoo {

constexpr int64_t kHeldLdsBytes = 156 * 1024;            // beside the kernel's own
// Columns of B that are held at a time, 16 bytes of a row at the most; 0: not one fits.
int held_cols(int64_t k, int64_t N, int type);
hipError_t launch_layer_held(const RowsArgs& a, const EpilogueArgs& e, hipStream_t s);

}  // namespace gcoo
