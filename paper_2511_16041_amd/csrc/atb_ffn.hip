// The gated block's forward products: act(x Wg^T) o (x Wu^T), and the down projection.
#include "atb_tiles.h"

namespace atb {

hipError_t launch_tiles_forward(TileParams p, int epilogue, hipStream_t stream)
{
    if (epilogue == kGated) return launch_tiles<false, false, kGated>(p, stream);
    if (epilogue == kGatedKeep) return launch_tiles<false, false, kGatedKeep>(p, stream);
    return launch_tiles<false, false, kStore>(p, stream);
}

}  // namespace atb
