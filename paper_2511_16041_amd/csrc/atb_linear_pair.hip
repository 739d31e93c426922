// Both products of a linear layer's backward pass in one launch: dx = dz W, and behind it dW = dz^T x.
//
// Where each by itself would leave CUs idle at its end, or has fewer tiles than there is room for, the tiles of the second take their place; the ones of dx, whose reductions are the longer ones (of N, not of
// M), come first.  Bound: as the tiles (atb_tiles.h).
// Measured: M = 8192, N = 14336, K = 4096 1566 us, 1230 TFLOP/s, MFMAs busy 62 % (two launches 1563: level); 1500 x 5001 x 2056 85 to 90, 34 % (99), its tail one long reduction of 79 K-steps per CU.
#include "atb_block.h"
#include "atb_tiles.h"

namespace atb {
namespace {

template <class S>
__global__ void __launch_bounds__(S::NT, 2) pair_kernel(const TileParams dx, const TileParams dw, int first)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS_BYTES];
    int m0 = 0, n0 = 0, share = 0;
    if ((int)blockIdx.x < first) {
        if (!tile_of<S, false>(dx, blockIdx.x, m0, n0, share)) return;
        Tile<S, false, true, kStore> tile(dx, lds, m0, n0, 0);
        tile.multiply(0, dx.steps);
        tile.finish(0);
    } else {
        if (!tile_of<S, false>(dw, blockIdx.x - first, m0, n0, share)) return;
        Tile<S, true, true, kStore> tile(dw, lds, m0, n0, 0);
        tile.multiply(0, dw.steps);
        tile.finish(0);
    }
}

template <class S>
hipError_t launch(TileParams &dx, TileParams &dw, hipStream_t stream)
{
    int64_t blocks[2];
    TileParams *of[2] = {&dx, &dw};
    for (int i = 0; i < 2; ++i) {
        TileParams &p = *of[i];
        const TilePlan plan = tile_plan(p.M, p.N, S::TM, false);
        p.tiles_m = plan.tiles_m;
        p.tiles_n = plan.tiles_n;
        p.group_m = 2048 / S::TM;
        p.steps = (p.K + 63) / 64;
        p.planes = p.parts = 1;
        p.edge = p.N;
        blocks[i] = round_up((int64_t)p.tiles_m * p.tiles_n, 8);           // (whole eights: a workgroup's XCD is its tile's)
    }
    if (blocks[0] + blocks[1] > 0xffffff00u / S::NT) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(pair_kernel<S>, dim3((unsigned)(blocks[0] + blocks[1])), dim3(S::NT), 0, stream, dx, dw, (int)blocks[0]);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tiles_pair(TileParams dx, TileParams dw, int tile, hipStream_t stream) { return tile == 256 ? launch<Tile256>(dx, dw, stream) : launch<Tile128>(dx, dw, stream); }

}  // namespace atb
