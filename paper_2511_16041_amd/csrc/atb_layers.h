// Internal declarations of the feed-forward sublayer's operators: layer norm, the gated block in bf16, products with 4-bit weights.
// Not part of the public C ABI (see include/atb.h).
#pragma once

#include "atb_internal.h"

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
int64_t norm_partials(int64_t M, int64_t D);       // partial sums of the parameters' gradients that the backward pass makes

// ---- bf16 products in tiles (atb_ffn.hip, atb_ffn_grad.hip)

// What a lane does with its sums.
enum Epilogue {
    kStore = 0,          // C = sum, bf16
    kGated = 1,          // C = act(gate sum) * up sum; B is both weights, their columns side by side in a wave's tile
    kGatedKeep = 2,      // ... and writes what the backward pass needs of both sums
    kGatedGrad = 3,      // the sum is dh: writes dg = dh u act'(g) and du = dh act(g)
};

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
    int tiles_m, tiles_n, group_m;
};
// The products of the forward pass (A and B with K contiguous): epilogue kStore, kGated or kGatedKeep.
hipError_t launch_tiles_forward(TileParams p, int epilogue, hipStream_t stream);
// dh with its epilogue, and dx = dg Wg + du Wu: B in rows.
hipError_t launch_tiles_dx(TileParams p, int epilogue, hipStream_t stream);
// Gradients of weights: A transposed, B in rows.
hipError_t launch_tiles_dw(TileParams p, hipStream_t stream);

// ---- products of few rows (atb_stream.hip, atb_q4_stream.hip)

// Whether the gated block of M tokens in bf16 runs on the kernel for few rows.
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
};
hipError_t launch_stream(const StreamParams &p, hipStream_t stream);
hipError_t launch_q4_stream(const StreamParams &p, hipStream_t stream);      // 4 bits; launch_stream calls it

// ---- 4-bit storage (atb_q4.hip)

hipError_t launch_q4_quantize(const void *w, int w_type, int64_t ldw, uint8_t *packed, uint16_t *scales, uint8_t *zeros,
                              int64_t N, int64_t K, int group, hipStream_t stream);
hipError_t launch_q4_decode(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, void *out, int out_type,
                            int64_t N, int64_t K, int group, hipStream_t stream);

}  // namespace atb
