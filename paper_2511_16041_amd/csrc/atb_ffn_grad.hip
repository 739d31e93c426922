// The gated block's backward products.
#include "atb_tiles.h"

namespace atb {

hipError_t launch_tiles_dx(TileParams p, int epilogue, hipStream_t stream)
{
    if (epilogue == kGatedGrad) return launch_tiles<false, true, kGatedGrad>(p, stream);
    return launch_tiles<false, true, kStore>(p, stream);
}

hipError_t launch_tiles_dw(TileParams p, hipStream_t stream) { return launch_tiles<true, true, kStore>(p, stream); }

}  // namespace atb
