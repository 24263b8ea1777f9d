// Host side of the launches of the sixteen-wave kernel and of its instances for a layer with sparse weights.
#pragma once
#include "gcoo_spdm_band_kernel.hpp"

namespace gcoo {

// The instances: the cut, and how the rows of B are requested (gcoo_spdm_band_kernel.hpp).
enum BandKind { kBandTallSpread, kBandTallFirst, kBandTallSecond, kBandWideSpread, kBandWideStep, kBandWideFirst, kBandWideSecond };
struct BandLaunch {
    BandArgs a;
    RowsArgs rows;
    BandRowsGrid grid;
    BandKind kind;
    dim3 blocks() const { return dim3((unsigned)(a.grid > kRowsAllWgs ? a.grid : kRowsAllWgs)); }
};
// Checks what the kernel assumes and fills in the rest.
hipError_t band_launch(const BandArgs& a, const RowsArgs& rows, BandLaunch* out);

// b.launch<V, SPREAD, LATE>(stream) of b.l.kind
template <class B>
hipError_t launch_band_kind(const B& b, hipStream_t s)
{
    switch (b.l.kind) {
        case kBandTallSpread: return b.template launch<2, true, false>(s);
        case kBandTallFirst: return b.template launch<2, false, false>(s);
        case kBandTallSecond: return b.template launch<2, false, true>(s);
        case kBandWideSpread: return b.template launch<4, true, false>(s);
        case kBandWideStep: return b.template launch<4, true, true>(s);
        case kBandWideFirst: return b.template launch<4, false, false>(s);
        default: return b.template launch<4, false, true>(s);
    }
}

}  // namespace gcoo
