// Internal declarations of what a transformer's block has around its feed-forward sublayer: a product with its epilogue, norms on both sides of a residual sum, a mixture of experts
// for few tokens.
// Not part of the public C ABI (see include/atb.h).
#pragma once

#include "atb_layers.h"

namespace atb {

// ---- a product with its epilogue (atb_linear.hip)

// dz = dy o act'(z) and its column sums
struct LinearGradParams {
    const uint16_t *dy;          // M x N bf16, lddy apart, at any element
    int64_t lddy;
    const uint16_t *slope;       // M rows of round_up(N, 8) in fp16, of which N count, or null: 1
    uint16_t *dz;                // M x round_up(N, 8) bf16, the padding written as zero, or null: not wanted
    float *partial;              // linear_parts(M, N) x N column sums, where dbias is wanted
    void *dbias;                 // N elements of bias_type, or null
    int bias_type;
    int64_t M;
    int N;
};
hipError_t launch_linear_grad(const LinearGradParams &p, hipStream_t stream);

// Runs of rows whose column sums are taken apart: one of up to 16 rows (which needs no second kernel), else of 4 rows, which are loaded at once, and as many more as it takes for about 1024 workgroups of 2048 columns; for
// no sum to have a chain of more than 512 additions, of at most 512.
static inline int64_t linear_parts(int64_t M, int64_t N)
{
    if (M <= 16) return M > 0;
    const int64_t blocks = (N + 2047) / 2048, wanted = std::max<int64_t>(1, std::min(1024 / std::min<int64_t>(blocks, 1024), (M + 3) / 4));
    return std::max(wanted, (M + 511) / 512);
}

// The tiles in which both products of the backward pass of M rows, N columns and K inputs run in one launch (atb_linear_pair.hip), or 0: each in its own.  A launch of tiles takes as long as its longest reduction
// or as all K-steps of 64 over 256 CUs, us per K-step of a tile of 256 x 256 1.3 and 1.65, of 128 x 128 0.6 and 0.53: the smaller time chooses the tiles.  By themselves the products may have their reductions in
// shares, and where dx has few tiles and a long reduction that is faster: up to 1.35 times what large tiles take without idle CUs, or 32 K-steps, the pair is.  us, in one launch / by themselves: 1500 x 5000 x 2056
// 92 / 102, 5000 x 5000 x 1000 116 / 168, 4096 x 4096 x 2048 108 / 152, 2048 x 2048 x 2048 37 / 44, 1000 x 2000 x 1000 21 / 39, 100 x 1000 x 4000 14 / 19, 1024 x 11008 x 4096 183 / 196, 2048 x 8192 x 2048 141 / 133,
// 5000 x 5000 x 4096 357 / 443, 4096 x 4096 x 4096 205 / 209, 8192 x 14336 x 4096 1566 / 1563; not taken: 1024 x 8192 x 2048 84 / 79, 512 x 14336 x 4096 162 / 156, 64 x 4096 x 4096 36 / 26.
static inline int linear_pair(int64_t M, int64_t N, int64_t K)
{
    const double dx = (double)((N + 63) / 64), dw = (double)((M + 63) / 64), longest = std::max(dx, dw);
    auto all = [&](int tile) {
        const TilePlan x = tile_plan(M, K, tile, false), w = tile_plan(N, K, tile, false);
        return ((double)x.tiles_m * x.tiles_n * dx + (double)w.tiles_m * w.tiles_n * dw) / 256;
    };
    const double large = std::max(1.3 * longest, 1.65 * all(256)), small = std::max(0.6 * longest, 0.53 * all(128));
    if (longest > 32 && std::min(large, small) > 1.35 * 1.65 * all(256)) return 0;
    return large <= small ? 256 : 128;
}
hipError_t launch_tiles_pair(TileParams dx, TileParams dw, int tile, hipStream_t stream);

// ---- norms on both sides of a residual sum (atb_residual.hip)

struct NormSpec {
    int kind;                    // atb_norm_kind
    const void *weight, *bias;   // null: 1 and 0
    float eps;
};
struct ResidualParams {
    const void *x, *z;           // M x D: the residual stream and the block's result
    void *r, *h;                 // the sum, and (a norm `pre`) its norm
    const void *dr, *dh;         // their gradients (dr may be null: 0)
    void *dx, *dz;               // null: not asked for
    int64_t ldx, ldz, ldr, ldh, lddr, lddh, lddx, lddz;
    NormSpec post, pre;
    const void *gate;            // groups x D, or null
    int64_t groups;              // 1 without a gate; M is a multiple
    float scale;
    float *stats;                // 4 x M: mean and 1 / size of post, of pre
    void *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;       // null: not asked for
    float *workspace;            // residual_room(M, D, groups).total floats, where one of them is asked for
    int64_t M;
    int D;
    int x_type, z_type, w_type;  // atb_type
    int parts;                   // set by the launch: workgroups that share the sums over a group's rows
};
hipError_t launch_residual(const ResidualParams &p, hipStream_t stream);
hipError_t launch_residual_backward(const ResidualParams &p, hipStream_t stream);

constexpr int kResidualPerThread = 8;              // elements of a row that a thread holds, of long rows a few times as many
constexpr int kResidualThreads = 512;              // workgroup of the backward pass: 256 registers per thread
constexpr int kResidualMaxGradRow = 2 * kResidualThreads * kResidualPerThread;       // longer rows are read again for every sum

// ... and rows of less than a chunk with them
static inline bool residual_is_long(int64_t D) { return D > kResidualMaxGradRow || D < kResidualPerThread; }
// Rows of up to twice as many elements in 16 bits are held for dx and dz; their sums are a pass of their own, as those of longer rows.  (The kernels have 123 to 199 of 256 registers: two sums, 48 or 64 more, would fit some of
// them; not tried.)  us without the sums, held / read again: 4096 x 12000 138 / 225, 512 x 16384 28 / 36, 9 x 11066 7.6 / 19.5.  With x in fp32, whose rows are read again, 4096 x 12000 takes 294.
static inline bool residual_is_wide(int64_t D) { return D > kResidualMaxGradRow && D <= 2 * kResidualMaxGradRow; }

// Threads per row: the power of two, 64 to 512, that holds it.
static inline int residual_threads(int64_t D)
{
    int t = 64;
    while (t < kResidualThreads && (int64_t)t * kResidualPerThread < D) t *= 2;
    return t;
}

// The backward pass's workspace in floats.  Sums over the rows of a group are taken by `parts` workgroups, one per CU of the 256 in all (of rows that residual_is_long, whose sums are a pass of their own, 64 times the
// column blocks), with chains of at most 512 rows as in norm_partials.  (Two per CU, for which 128 registers do in 16 bits and without biases: 8192 x 4096 84 us instead of 81, and twice the parts to add.)
struct ResidualRoom { int64_t parts, sums, totals, rows, total; };
static inline ResidualRoom residual_room(int64_t M, int64_t D, int64_t groups)
{
    ResidualRoom r = {};
    const bool is_long = residual_is_long(D);
    const int64_t rows = M / groups, at_once = is_long ? 1 : kResidualThreads / residual_threads(D), most = std::max<int64_t>(1, (is_long ? 64 : 256) / groups);
    const int64_t turns = (rows + at_once - 1) / at_once;
    r.parts = M == 0 ? 0 : turns < most ? turns : most * ((turns + most * 512 - 1) / (most * 512));
    r.sums = round_up(groups * r.parts * 4 * D, 4);
    r.totals = groups > 1 ? round_up(groups * 4 * D, 4) : 0;
    r.rows = is_long ? round_up(2 * M, 4) : 0;
    r.total = r.sums + r.totals + r.rows;
    return r;
}

// ---- a mixture of experts for few tokens (atb_moe.hip, atb_moe_q4.hip)

constexpr int kMoeTokens = 64, kMoeExperts = 256, kMoeTopK = 16, kMoePlaces = kMoeTokens * kMoeTopK;
constexpr int kMoeSegments = kMoeExperts + kMoePlaces / 16;

// What the tokens chose, in device memory.  A place is a token's choice; places are sorted by expert, of one expert by token.  A segment is a run of places of one expert that a workgroup takes at a
// time: at most 16 or 32.
struct MoePlan {
    int segments;
    int expert[kMoeSegments], first[kMoeSegments], rows[kMoeSegments];
    int token[kMoePlaces];
    float weight[kMoePlaces];
};

struct MoeParams {
    const uint16_t *x, *router;  // bf16, M x D and E x D
    int64_t ldx, ld_router;
    StreamWeight gate, up, down; // of all experts, one after the other's: E F x D, E F x D, E D x F, contiguous
    uint16_t *y;                 // bf16 M x D
    int64_t ldy;
    int *experts;                // M x k, or null
    float *weights;              // M x k, or null
    int M, D, F, E, k;
    int group;                   // 0: bf16 weights
    int act, renormalize;
    int few;                     // moe_is_few
    // workspace
    double *logits;              // M x E
    MoePlan *plan;
    uint16_t *h;                 // M k x F: the inner activations, by place
    int shares;                  // of the down product's reduction; 1: no partial sums
    float *partial;              // shares x M x D
};
hipError_t launch_moe(const MoeParams &p, hipStream_t stream);
hipError_t launch_moe_q4(const MoeParams &p, hipStream_t stream);        // the products, with weights in 4 bits; launch_moe calls it

// Rows of x that a workgroup of the products takes: 32 where an expert gets more than 12 on average, so that few get more than 16 and read their weights twice.
static inline int moe_rows(int64_t M, int64_t E, int64_t k) { return M > 16 && M * k > 12 * E ? 32 : 16; }
// Whether the products of up to 8 tokens choose the experts themselves, instead of a launch before them: where there are no more of the router's products than a workgroup has threads, and their workgroups, of 16 columns of
// an expert, run at once, four per CU, or have little to choose from.  us, with / without that launch, 4 bits: 2 tokens through 8 of 8 experts of 2304 x 1856 40 / 37.5, 4 through one of 41 of 1280 x 640 21.3 / 19.5,
// 8 through 2 of 8 of 2048 x 1536 30.5 / 28.2, 2 through 8 of 128 of 2048 x 768 30.2 / 28.8, 2 through 2 of 8 of 4096 x 14336 82.7 / 82.7; not taken: 2 through 8 of 64 of 2048 x 1536 38.3 / 40.0, 8 through 2 of 8 of 4096 x 14336
// 178 / 183, 8 through 2 of 16 of 2048 x 8192 83 / 102.
static inline bool moe_is_few(int64_t M, int64_t E, int64_t k, int64_t F)
{
    return M <= 8 && M * E <= 256 && (M * E <= 16 || std::min(E, M * k) * ((F + 15) / 16) <= 1024);
}
// The most segments that the choices can have
static inline int moe_segments(int64_t M, int64_t E, int64_t k, int rows) { return (int)(std::min(E, M * k) + M * k / rows); }

// Shares of the down product's reduction, the chosen experts' panels of 64 (4 bits: 256) one after the other, which a third kernel adds: as many as make 512 workgroups of 16 columns (4 bits: 32) where there
// would be fewer than CUs, and a panel or more for each of their 8 waves (4 bits, whose waves take longer to begin: one and a half).  us, 1 / 2 / 3 / 4 / 6 shares without joining them, which takes 2.5 to 4.8: 21
// tokens over 60 experts of 2056 x 1416 143 / 108 / 79 / 91 / 79, one token through 2 experts of 4096 x 14336 (256 workgroups) 44 / 44 / 43 / 43 / 43; 4 bits, 4 / 8 shares: one token through 8 of 2048 x 1536 7.5 / 9.7,
// 2 / 4 / 8: 32 tokens over 8 of 4096 x 14336 81 / 76 / 77.
static inline int moe_shares(int64_t M, int64_t D, int64_t F, int64_t E, int64_t k, int group)
{
    const int64_t blocks = group ? (D + 31) / 32 : (D + 15) / 16, experts = std::min(E, M * k);
    if (blocks >= 256) return 1;
    return (int)std::max<int64_t>(1, std::min(512 / blocks, group ? experts * ((F + 255) / 256) / 12 : experts * ((F + 63) / 64) / 8));
}

// The workspace, in bytes
struct MoeRoom { int64_t logits, plan, h, partial, total; };
static inline MoeRoom moe_room(int64_t M, int64_t D, int64_t F, int64_t E, int64_t k, int group)
{
    MoeRoom r;
    const int64_t shares = M > 0 ? moe_shares(M, D, F, E, k, group) : 1;
    r.logits = round_up(M * E * (int64_t)sizeof(double), 256);
    r.plan = round_up((int64_t)sizeof(MoePlan), 256);
    r.h = round_up(M * k * F * 2, 256);
    r.partial = shares > 1 ? round_up(shares * M * D * (int64_t)sizeof(float), 256) : 0;
    r.total = r.logits + r.plan + r.h + r.partial;
    return r;
}

}  // namespace atb
