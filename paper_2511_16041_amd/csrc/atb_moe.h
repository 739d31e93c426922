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

// What experts are ordered by: l, of -infinity less than all that sums of bf16 products can be (2^278), and NaN behind that
ATB_DEV double moe_key(double l) { return l == l ? fmax(l, -0x1p1000) : -INFINITY; }

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

// A segment of up to 8 tokens, which are the bits of `tokens`
struct MoeFew { MoeSegment segment; unsigned tokens; };

// The choice of few tokens (moe_is_few), by every workgroup of their gate and up products for itself, without a launch for it, which took 6 us, 5 more than this does of one token over 64 experts (one token
// through 8 of them, 2048 x 1536 in 4 bits, 30 / 25.3 in all): the experts ahead of each are counted by all 256 threads.  Workgroup y has the y-th of the chosen experts; the one of its first columns
// writes its part of the plan.  rows 0: there is none.  `lds`: 12 bytes for each of 256 products.
ATB_DEV MoeFew moe_choose_few(const MoeParams &p, char *lds)
{
    double *l = reinterpret_cast<double *>(lds);
    int *ahead = reinterpret_cast<int *>(l + 256);
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, all = p.M * p.E;
    const double mine = t < all ? p.logits[t] : -INFINITY;
    l[t] = moe_key(mine);
    ahead[t] = 0;
    __syncthreads();
    const int width = all <= 64 ? 64 : all <= 128 ? 128 : 256, o = t & (width - 1), per = (p.E * width + 255) / 256, from = t / width * per;
    if (o < all) {
        const int base = o / p.E * p.E;
        const double key = l[o];
        int n = 0;
#pragma unroll 4
        for (int j = base + from; j < base + min(from + per, p.E); ++j) n += l[j] > key || (l[j] == key && j < o);
        atomicAdd(&ahead[o], n);
    }
    __syncthreads();
    // every wave finds the chosen expert and its tokens by itself
    unsigned chose[4];                                             // tokens of expert 64 i + lane
    int expert = -1, experts = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 64 * i + lane;
        chose[i] = 0;
        for (int m = 0; m < p.M; ++m) chose[i] |= e < p.E && ahead[min(m * p.E + e, 255)] < p.k ? 1u << m : 0;
        const unsigned long long taken = __ballot(chose[i] != 0), found = __ballot(chose[i] != 0 && __popcll(taken & ((1ull << lane) - 1)) + experts == (int)blockIdx.y);
        if (found) expert = 64 * i + __ffsll(found) - 1;
        experts += __popcll(taken);
    }
    MoeFew few = {{max(expert, 0), 0, 0}, 0};
    if (expert >= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (64 * i <= expert)
                for (int m = 0; m < p.M; ++m) few.segment.first += __popcll(__ballot((chose[i] >> m & 1) != 0 && 64 * i + lane < expert));
            if (expert >> 6 == i) few.tokens = __builtin_amdgcn_readlane(chose[i], expert & 63);
        }
        few.segment.rows = __popc(few.tokens);
        if (blockIdx.x == 0) {
            if (t == 0) {
                p.plan->expert[blockIdx.y] = expert;
                p.plan->first[blockIdx.y] = few.segment.first;
                p.plan->rows[blockIdx.y] = few.segment.rows;
                if (blockIdx.y == 0) p.plan->segments = experts;
            }
            int place = few.segment.first;
            for (int m = 0; m < p.M; ++m) {
                if ((few.tokens >> m & 1) == 0) continue;
                if (place % 4 == wave) {
                    double raw[4];
                    float weight[4];
                    int rank[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool live = 64 * i + lane < p.E;
                        raw[i] = live ? p.logits[m * p.E + 64 * i + lane] : -INFINITY;
                        rank[i] = live ? ahead[m * p.E + 64 * i + lane] : p.E;
                    }
                    moe_weights(p, raw, rank, weight);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (64 * i + lane != expert) continue;
                        p.plan->token[place] = m;
                        p.plan->weight[place] = weight[i];
                        if (p.experts) p.experts[m * p.k + rank[i]] = expert;
                        if (p.weights) p.weights[m * p.k + rank[i]] = weight[i];
                    }
                }
                ++place;
            }
        }
    }
    __syncthreads();                                               // `lds` is free again
    return few;
}

// The workgroup's segment; rows 0: none.  FEW: moe_is_few
template <bool FEW>
ATB_DEV MoeFew moe_open(const MoeParams &p, char *lds)
{
    if constexpr (FEW) return moe_choose_few(p, lds);
    if ((int)blockIdx.y >= p.plan->segments) return {};
    return {moe_segment(p.plan, blockIdx.y), 0};
}

// The token of a segment's row
template <bool FEW>
ATB_DEV int moe_token(const MoeParams &p, const MoeFew &few, int row)
{
    if (!FEW) return p.plan->token[few.segment.first + row];
    int token = 0;
#pragma unroll
    for (int m = 0; m < 8; ++m)
        if (few.tokens >> m & 1 && row-- == 0) token = m;
    return token;
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
