// What the products of a mixture of experts share (atb_moe.hip: weights in bf16, atb_moe_q4.hip: in 4 bits).
#pragma once

#include "atb_block.h"
#include "atb_stream.h"

namespace atb {

struct MoeSegment { int expert, first, rows; };
ATB_DEV MoeSegment moe_segment(const MoePlan *plan, int i)
{
    return {__builtin_amdgcn_readfirstlane(plan->expert[i]), __builtin_amdgcn_readfirstlane(plan->first[i]), __builtin_amdgcn_readfirstlane(plan->rows[i])};
}

// The product of a segment's gate and up weights, as finish_rows stores it: rows of h
ATB_DEV StreamParams moe_inner(const MoeParams &p, const MoeSegment &s)
{
    StreamParams h = {};
    h.y = p.h + (int64_t)s.first * p.F;
    h.ldy = p.F;
    h.M = s.rows;
    h.act = p.act;
    h.y_type = ATB_TYPE_BF16;
    return h;
}

// A wave's sums of a segment, times the router's weights, onto its part of y: totals[token][16 NB].  No other wave touches it, and within a segment every row is another token's.
template <int MB, int NB>
ATB_DEV void moe_add(const MoePlan *plan, const MoeSegment &s, const floatx4 (&acc)[MB][NB], float *totals)
{
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = 16 * i + 4 * q + e;
            if (row >= s.rows) continue;
            float *to = totals + plan->token[s.first + row] * (16 * NB) + c;
            const float weight = plan->weight[s.first + row];
#pragma unroll
            for (int j = 0; j < NB; ++j) to[16 * j] += weight * acc[i][j][e];
        }
}

// A wave's way through its share of the down product: every W-th panel of the segments', one after the other
template <int W>
struct MoePlace {
    int panels, at, segment, panel;            // of a segment; of all; the segment's
    ATB_DEV MoePlace(int panels_, int first) : panels(panels_), at(first), segment(first / panels_), panel(first - segment * panels_) {}
    ATB_DEV void next()
    {
        at += W;
        panel += W;
        while (panel >= panels) {
            panel -= panels;
            ++segment;
        }
    }
};

// The waves' parts of y, added in wave order: `cols` columns from n0 on; of a reduction in shares the share's part, in fp32.
template <int NB, int W>
ATB_DEV void moe_finish(const MoeParams &p, const float *totals, int n0, int cols)
{
    __syncthreads();
    for (int o = threadIdx.x; o < p.M * 16 * NB; o += W * 64) {
        const int token = o / (16 * NB), col = o % (16 * NB);
        if (col >= cols) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += totals[w * p.M * 16 * NB + o];
        if (p.shares > 1) p.partial[((int64_t)blockIdx.y * p.M + token) * p.D + n0 + col] = v;
        else reinterpret_cast<__bf16 *>(p.y)[token * p.ldy + n0 + col] = (__bf16)v;
    }
}

}  // namespace atb
