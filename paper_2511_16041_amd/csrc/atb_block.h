// Internal declarations of what a transformer's block has around its feed-forward sublayer: a product with its epilogue.
// Not part of the public C ABI (see include/atb.h).
#pragma once

#include "atb_layers.h"

namespace atb {

// ---- a product with its epilogue (atb_linear.hip)

// dz = dy o act'(z) and its column sums
struct LinearGradParams {
    const uint16_t *dy;          // M x N bf16, lddy apart, at any element
    int64_t lddy;
    const uint16_t *slope;       // M x N fp16, or null: 1
    uint16_t *dz;                // M x round_up(N, 8) bf16, the padding written as zero, or null: not wanted
    float *partial;              // linear_parts(M, N) x N column sums, or null
    void *dbias;                 // N elements of bias_type, or null
    int bias_type;
    int64_t M;
    int N;
};
hipError_t launch_linear_grad(const LinearGradParams &p, hipStream_t stream);

// Runs of rows whose column sums are taken apart: about 1024 workgroups of 2048 columns, runs of 16 rows or more and, for no sum to have a chain of more than 512 additions,
// of at most 512.
static inline int64_t linear_parts(int64_t M, int64_t N)
{
    if (M <= 0) return 0;
    const int64_t blocks = (N + 2047) / 2048, wanted = std::max<int64_t>(1, std::min(1024 / std::min<int64_t>(blocks, 1024), (M + 15) / 16));
    return std::max(wanted, (M + 511) / 512);
}

}  // namespace atb
