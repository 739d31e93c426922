// Internal declarations of the feed-forward sublayer's operators: layer norm, the gated block in bf16, products with 4-bit weights.
// Not part of the public C ABI (see include/atb.h).
#pragma once

#include "atb_internal.h"

#include <algorithm>

namespace atb {

// ---- layer norm (atb_norm.hip)

struct NormParams {
    const void *x, *dy;          // rows of D elements, ldx / lddy elements apart
    void *y, *dx;
    int64_t ldx, lddy, ldy, lddx;
    const void *weight, *bias;   // null: 1 and 0
    void *dweight, *dbias;       // null: not asked for
    float *mean, *rstd;          // written by the forward pass if not null, read by the backward pass
    float *partial;              // norm_partials(M, D) x 2 D floats, where dweight or dbias is asked for
    int64_t M, D;
    float eps;
    int x_type, w_type;          // atb_type
};
hipError_t launch_norm(const NormParams &p, hipStream_t stream);
hipError_t launch_norm_backward(const NormParams &p, hipStream_t stream);

constexpr int kNormPerThread = 16;                 // elements of a row that a thread holds
constexpr int kNormGradThreads = 512;              // workgroup of the backward pass: 256 registers per thread
constexpr int kNormMaxGradRow = kNormGradThreads * kNormPerThread;       // of longer rows the parameters' gradients are a pass of their own

// Threads per row: the power of two, 64 to 1024, that holds it.
static inline int norm_threads(int64_t D)
{
    int t = 64;
    while (t < 1024 && (int64_t)t * kNormPerThread < D) t *= 2;
    return t;
}

// Partial sums of the parameters' gradients that the backward pass makes, one of each of its workgroups: one per CU of the 256 (of longer rows 64, times the column blocks),
// fewer where there are not as many row groups (a workgroup takes kNormGradThreads / norm_threads(D) rows at a time), and as many times more as it takes for none to
// add more than 512 of them one after another: every addition may err by 2^-24 of the sum, and where all err one way 4096 of them made it 6e-5.
static inline int64_t norm_partials(int64_t M, int64_t D)
{
    if (M <= 0) return 0;
    const int64_t rows = D > kNormMaxGradRow ? 1 : kNormGradThreads / norm_threads(D), most = D > kNormMaxGradRow ? 64 : 256;
    const int64_t groups = (M + rows - 1) / rows;
    return groups < most ? groups : most * ((groups + most * 512 - 1) / (most * 512));
}

// ---- bf16 products in tiles (atb_ffn.hip, atb_ffn_grad.hip)

// What a lane does with its sums.
enum Epilogue {
    kStore = 0,          // C = sum, bf16
    kGated = 1,          // C = act(gate sum) * up sum; B is both weights, their columns side by side in a wave's tile
    kGatedKeep = 2,      // ... and writes what the backward pass needs of both sums
    kGatedGrad = 3,      // the sum is dh: writes dg = dh u act'(g) and du = dh act(g)
    kShare = 4,          // the sum of a share of the reduction, in fp32; what it is for is done where the shares are joined
    kGatedShare = 5,     // ... of both weights
    kLinear = 6,         // C = act(sum + bias) + residual
    kLinearKeep = 7,     // ... and writes act'(sum + bias)
};
constexpr bool is_gated(int epilogue) { return epilogue == kGated || epilogue == kGatedKeep || epilogue == kGatedShare; }
constexpr bool is_share(int epilogue) { return epilogue == kShare || epilogue == kGatedShare; }
constexpr bool is_linear(int epilogue) { return epilogue == kLinear || epilogue == kLinearKeep; }

struct TileParams {
    // A: M x K, K contiguous, or (transposed) K x M, M contiguous; B: N x K, K contiguous, or (rows) K x N, N contiguous.
    // Two of each: the two halves of a longer reduction (segments = 2), two problems (problems = 2; B[1] = B[0]), or the two weights (kGated, kGatedKeep)
    const uint16_t *A[2], *B[2];
    int64_t lda[2], ldb[2];
    uint16_t *C[2];              // [1]: the second problem's; kGatedGrad: dg, du
    int64_t ldc;
    uint16_t *kept;              // kGatedKeep: written; kGatedGrad: read.  Three planes of M x N (see Tile::keep)
    int M, N, K;
    int segments, problems;
    int act;                     // atb_activation
    float *shares;               // room for tile_shares() floats, or null: reductions are not shared out
    // a product with its epilogue: N is a multiple of 8, of whose columns the first `edge` exist (0: all); C and residual begin at any element
    int edge;
    const void *bias;            // edge elements of bias_type, or null
    int bias_type;               // atb_type
    const uint16_t *residual;    // M x edge, ldr apart, or null
    int64_t ldr;
    uint16_t *slope;             // kLinearKeep: M rows of round_up(edge, 8) in fp16, 16-byte aligned
    // set by the launch
    int tiles_m, tiles_n, group_m;
    int steps;                   // K-steps of a segment
    int parts, planes;           // shares of the reduction; planes of M x N in each
};

struct TilePlan { int tiles_m, tiles_n; };
static inline TilePlan tile_plan(int64_t M, int64_t N, int tile, bool gated)
{
    const int64_t cols = gated ? tile / 2 : tile;
    return {(int)((M + tile - 1) / tile), (int)((N + cols - 1) / cols)};
}
// Tiles of 256 x 256, one workgroup per CU, where there are nearly as many as CUs (192 of 256; forward pass of D = 4096, F = 14336, M = 512, 224 of them in the
// gated product, us: 195, with 128 x 128 230; M = 2048, 128 of them in the down projection: 670 with small ones there, 717 with large ones).  Otherwise the reduction
// is split into shares, whose sums go to memory in fp32 and are joined by a second kernel, so that there are nearly as many workgroups as CUs: in large
// tiles where a share has 28 K-steps or more (more than 128 rows, which would leave half of a tile empty; not gated products, whose reduction is the short one: D = 8192,
// F = 2048, M = 512 68 without, 70 with), else in tiles of 128 x 128 where these are at most half as many as CUs.  A workgroup alone on its CU takes 0.74 us
// per K-step whatever the others do, so at few tokens the length of the reduction is the time.  A share has at least 8 K-steps: below, the second launch
// costs what it saves.  What is left, tiles of 128 x 128, two per CU.
// Whole / in shares, us, forward and backward (the sum of the kernels and launches):
//   M 33, D 1024, F 4096    44 /  24    94 /  39        M 33, D 4096, F 14336   225 /  92    492 / 208
//   M 256                   47 /  35   102 /  52        M 512                   275 / 206    661 / 522
//   M 2048                  67 /  61   164 / 153        M 512, D 8192, F 2048    92 /  67    214 / 157
// Large tiles in shares / small ones: D 4096, F 14336, M 640 276 / 348 and 538 / 689, M 1024 318 / 370 and 692 / 799, M 2048 593 / 659 and 1259 / 1404; D 2048, F 5504,
// M 2048 148 / 145 and 340 / 374.  With shares of 24 K-steps D 5120, F 1536, M 1500 takes 199 backward instead of 174.
// Two workgroups per CU with small tiles write twice the sums and are slower from M = 128 on (D 8192, F 2048, M 128: 48 forward, 98 backward; with one 40 and 87).
// Without room for shares (`room`) what is left takes their place: M = 500, D = 4096, F = 14336 275 us forward and 650 backward, with whole reductions in
// the large tiles that their shares would have had 417 and 973.
// Products with an epilogue (`linear`) have tiles of 128 x 256 too, one per CU, where these are no more than CUs and small ones would be two to some of them.  us, these / what the rules above choose: 2048 x 4096 x 4096 62
// / 80 (large ones in two shares), 1500 x 5008 x 2056 39 / 47, 1100 x 4096 x 4096 54 / 57, 2048 x 3500 x 1024 20.8 / 21.8.
struct TileChoice { bool large; int parts; bool wide = false; };
static inline TileChoice choose_tiles(int64_t M, int64_t N, int64_t K, int segments, int problems, bool gated, bool room, bool linear = false)
{
    const TilePlan large = tile_plan(M, N, 256, gated), small = tile_plan(M, N, 128, gated);
    if ((int64_t)large.tiles_m * large.tiles_n * problems >= 192) return {true, 1};
    if (linear && (int64_t)small.tiles_m * small.tiles_n > 256 && (int64_t)small.tiles_m * large.tiles_n <= 256) return {false, 1, true};
    if (!room) return {false, 1};
    const int64_t steps = (K + 63) / 64 * segments, tiles = (int64_t)small.tiles_m * small.tiles_n * problems;
    const int64_t few = (int64_t)large.tiles_m * large.tiles_n * problems, each = 256 / std::max<int64_t>(few, 1);
    if (!gated && M > 128 && few > 0 && few * each >= 192 && steps >= 28 * each) return {true, (int)each};
    const int64_t parts = std::min(256 / std::max<int64_t>(tiles, 1), steps / 8);
    return {false, parts > 1 ? (int)parts : 1};
}
static inline int64_t tile_shares(int64_t M, int64_t N, int64_t K, int segments, int problems, bool gated, bool linear = false)
{
    const TileChoice c = choose_tiles(M, N, K, segments, problems, gated, true, linear);
    return c.parts > 1 ? c.parts * (gated ? 2 : problems) * M * N : 0;
}
// The products of the forward pass (A and B with K contiguous): epilogue kStore, kGated or kGatedKeep.
hipError_t launch_tiles_forward(TileParams p, int epilogue, hipStream_t stream);
// A product with its epilogue (atb_linear.hip): kLinear or kLinearKeep.
hipError_t launch_tiles_linear(TileParams p, int epilogue, hipStream_t stream);
// dh with its epilogue, and dx = dg Wg + du Wu: B in rows.
hipError_t launch_tiles_dx(TileParams p, int epilogue, hipStream_t stream);
// Gradients of weights: A transposed, B in rows.
hipError_t launch_tiles_dw(TileParams p, hipStream_t stream);

// ---- products of few rows (atb_stream.hip, atb_q4_stream.hip)

// Whether the gated block of M tokens in bf16 runs on the kernel for few rows, whose waves hold at most 32: forward at M = 32, us, 11.9 there and 23 in
// tiles with D = 1024 and F = 4096, 78 and 92 with D = 4096 and F = 14336.  More would read the weights twice.
static inline bool ffn_streams(int64_t M) { return M <= 32; }

struct StreamWeight {
    const void *w;               // bf16 N x K (row pitch ldw elements), or 4-bit codes N x K/2 bytes
    const uint16_t *scales;      // 4 bits: bf16 N x K/group
    const uint8_t *zeros;        // 4 bits: N x K/group, or null for 8
    int64_t ldw;
};
struct StreamParams {
    StreamWeight w[2];           // [1]: the up projection of a gated product
    const uint16_t *x;           // bf16 M x K
    void *y;                     // M x N
    int64_t ldx, ldy;
    int M, N, K;
    int group;                   // 0: bf16 weights
    int gated, act;
    int y_type;                  // atb_type
    // bf16 weights, not gated: y = act(x W^T + bias) + residual if `linear` is set
    int linear;
    const void *bias;            // N elements of bias_type, or null
    int bias_type;
    const uint16_t *residual;    // M x N, ldr apart, or null
    int64_t ldr;
    uint16_t *slope;             // M rows of round_up(N, 8) in fp16: act'(x W^T + bias), or null
};
hipError_t launch_stream(const StreamParams &p, hipStream_t stream);
hipError_t launch_q4_stream(const StreamParams &p, hipStream_t stream);      // 4 bits; launch_stream calls it

// ---- 4-bit storage (atb_q4.hip)

hipError_t launch_q4_quantize(const void *w, int w_type, int64_t ldw, uint8_t *packed, uint16_t *scales, uint8_t *zeros,
                              int64_t N, int64_t K, int group, hipStream_t stream);
hipError_t launch_q4_decode(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, void *out, int out_type,
                            int64_t N, int64_t K, int group, hipStream_t stream);

}  // namespace atb
