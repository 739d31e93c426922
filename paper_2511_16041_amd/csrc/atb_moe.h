// What the products of a mixture of experts share (atb_moe.hip: weights in bf16, atb_moe_q4.hip: in 4 bits).
#pragma once

#include "atb_block.h"
#include "atb_row.h"
#include "atb_stream.h"

namespace atb {

struct MoeSegment { int expert, first, rows; };
ATB_DEV MoeSegment moe_segment(const MoePlan *plan, int i)
{
    return {__builtin_amdgcn_readfirstlane(plan->expert[i]), __builtin_amdgcn_readfirstlane(plan->first[i]), __builtin_amdgcn_readfirstlane(plan->rows[i])};
}

// The plan in LDS, fetched by all threads at once: what a wave reads of it later does not wait for memory, with other requests on their way.
struct MoeCopy { int *expert, *first, *rows, *token; float *weight; };
static inline size_t moe_copy_bytes(int segments, int places) { return (size_t)(3 * segments + 2 * places) * 4; }
ATB_DEV MoeCopy moe_copy(const MoePlan *plan, int *to, int segments, int places)
{
    const MoeCopy c = {to, to + segments, to + 2 * segments, to + 3 * segments, reinterpret_cast<float *>(to + 3 * segments + places)};
    for (int i = threadIdx.x; i < segments; i += blockDim.x) {
        c.expert[i] = plan->expert[i];
        c.first[i] = plan->first[i];
        c.rows[i] = plan->rows[i];
    }
    for (int i = threadIdx.x; i < places; i += blockDim.x) {
        c.token[i] = plan->token[i];
        c.weight[i] = plan->weight[i];
    }
    return c;
}
ATB_DEV MoeSegment moe_segment(const MoeCopy &c, int i)
{
    return {__builtin_amdgcn_readfirstlane(c.expert[i]), __builtin_amdgcn_readfirstlane(c.first[i]), __builtin_amdgcn_readfirstlane(c.rows[i])};
}

// A token's router weights from its products, lane l's of the experts 64 i + l, and their ranks: exp(l - the largest l) over its sum over all experts or over the chosen ones.  A NaN or an infinity among the
// summands gives what the formula gives.
template <int PER>
ATB_DEV void moe_weights(const MoeParams &p, const double (&mine)[PER], const int (&rank)[PER], float (&weight)[PER])
{
    const int lane = threadIdx.x & 63;
    double top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) top = fmax(top, mine[i]);        // (of a NaN and a number the number)
    top = lanes_max(top);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool live = 64 * i + lane < p.E, taken = live && rank[i] < p.k;
        weight[i] = live ? expf((float)(mine[i] - top)) : 0.0f;
        if (p.renormalize ? taken : live) sum += weight[i];
    }
    sum = lanes_sum(sum);
#pragma unroll
    for (int i = 0; i < PER; ++i) weight[i] /= sum;
}

// The choice of a single token, by every workgroup of its gate and up products for itself, without a launch for it (which took 6 us, 5 more than this, of one token through 8 of 64 experts of 2048 x 1536 in 4 bits: 30 / 25.3 in all):
// the experts ahead of each are counted by all 256 threads.  Returns this workgroup's segment; those of the first columns write their part of the plan.  `lds`: 12 bytes for each of kMoeExperts.
ATB_DEV MoeSegment moe_choose_one(const MoeParams &p, char *lds)
{
    double *l = reinterpret_cast<double *>(lds);
    int *ahead = reinterpret_cast<int *>(l + kMoeExperts);
    const int t = threadIdx.x, lane = t & 63, place = blockIdx.y;
    const double mine = t < p.E ? p.logits[t] : -INFINITY;
    l[t] = mine == mine ? mine : -INFINITY;                        // NaN is behind all numbers
    ahead[t] = 0;
    __syncthreads();
    const int width = p.E <= 64 ? 64 : p.E <= 128 ? 128 : 256, e = t & (width - 1), part = t / width, per = width * width / 256;
    const double key = l[e];
    int n = 0;
#pragma unroll 4
    for (int j = part * per; j < (part + 1) * per; ++j) n += j < p.E && (l[j] > key || (l[j] == key && j < e));
    atomicAdd(&ahead[e], n);
    __syncthreads();
    // every wave finds the place-th of the chosen by itself
    int expert = 0, before = 0, rank[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        rank[i] = ahead[64 * i + lane];
        const unsigned long long taken = __ballot(64 * i + lane < p.E && rank[i] < p.k), to = (taken >> lane & 1) == 0 ? 0 : __popcll(taken & ((1ull << lane) - 1)) + before == place;
        const unsigned long long found = __ballot(to);
        if (found) expert = 64 * i + __ffsll(found) - 1;
        before += __popcll(taken);
    }
    if (blockIdx.x == 0 && t < 64) {
        double raw[4];
        float weight[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = 64 * i + lane < p.E ? p.logits[64 * i + lane] : -INFINITY;
        moe_weights(p, raw, rank, weight);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (64 * i + lane != expert) continue;
            p.plan->expert[place] = expert;
            p.plan->first[place] = place;
            p.plan->rows[place] = 1;
            p.plan->token[place] = 0;
            p.plan->weight[place] = weight[i];
            if (place == 0) p.plan->segments = p.k;
            if (p.experts) p.experts[rank[i]] = expert;
            if (p.weights) p.weights[rank[i]] = weight[i];
        }
    }
    __syncthreads();                                               // `lds` is free again
    return {expert, place, 1};
}

// Whether the workgroup has a segment, and which.  FEW: there may be one token alone
template <bool FEW>
ATB_DEV bool moe_open(const MoeParams &p, char *lds, MoeSegment &segment)
{
    const bool one = FEW && p.M == 1;
    if ((int)blockIdx.y >= (one ? p.k : p.plan->segments)) return false;
    segment = one ? moe_choose_one(p, lds) : moe_segment(p.plan, blockIdx.y);
    return true;
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
ATB_DEV void moe_add(const MoeCopy &plan, const MoeSegment &s, const floatx4 (&acc)[MB][NB], float *totals)
{
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = 16 * i + 4 * q + e;
            if (row >= s.rows) continue;
            float *to = totals + plan.token[s.first + row] * (16 * NB) + c;
            const float weight = plan.weight[s.first + row];
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
