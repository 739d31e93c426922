// The products of a mixture of experts with weights in 4 bits (atb_moe.hip has the whole, atb_q4_stream.hip how the weights are multiplied).
#include "atb_moe.h"
#include "atb_q4_rows.h"

namespace atb {
namespace {

template <class S>
__global__ void __launch_bounds__(S::W * 64, 4) moe_q4_gated_kernel(const MoeParams p)
{
    __shared__ float lds[S::W * S::NB * 256];
    if ((int)blockIdx.y >= p.plan->segments) return;
    const MoeSegment seg = moe_segment(p.plan, blockIdx.y);
    const int n0 = blockIdx.x * 16 * S::COLS, cols = min(p.F - n0, 16 * S::COLS);
    const int64_t n = (int64_t)seg.expert * p.F + n0;
    const Q4View view = {p.x, p.ldx, p.M, seg.rows, {q4_columns(p.gate, n, p.D, S::G), q4_columns(p.up, n, p.D, S::G)}, cols, p.D};
    const int *tokens = p.plan->token + seg.first;
    Q4Stream<S> s(view, [&](int row) { return tokens[row]; });
    s.run();
    finish_rows<1, S::NB, S::W, true>(moe_inner(p, seg), s.acc, lds, 0, n0, cols);
}

template <class S, int MOST>
__global__ void __launch_bounds__(S::W * 64, 4) moe_q4_down_kernel(const MoeParams p)
{
    __shared__ float totals[S::W * MOST * 16 * S::NB];
    const MoePlan *plan = p.plan;
    const int n0 = blockIdx.x * 16 * S::COLS, cols = min(p.D - n0, 16 * S::COLS);
    auto view_of = [&](const MoeSegment &seg) {
        return Q4View{p.h + (int64_t)seg.first * p.F, p.F, seg.rows, seg.rows, {q4_columns(p.down, (int64_t)seg.expert * p.D + n0, p.F, S::G), {}}, cols, p.F};
    };
    auto row_of = [](int row) { return row; };
    const int panels = (p.F + kQ4PanelK - 1) / kQ4PanelK, segments = __builtin_amdgcn_readfirstlane(plan->segments);
    Q4Stream<S> s(view_of(moe_segment(plan, 0)), row_of);
    float *mine = totals + s.wave * p.M * 16 * S::NB;
    for (int i = s.lane; i < p.M * 16 * S::NB; i += 64) mine[i] = 0.0f;
    // this wave's panels: every W-th of all segments'
    struct Place { int segment, panel; };
    auto next = [&](Place at) {
        at.panel += S::W;
        while (at.panel >= panels && at.segment < segments) {
            at.panel -= panels;
            ++at.segment;
        }
        return at;
    };
    Place at = next({0, s.wave - S::W});
    int loaded = 0, summed = at.segment;
    typename Q4Stream<S>::Panel a, b;
    auto load = [&](typename Q4Stream<S>::Panel &to, const Place &place) {
        if (place.segment >= segments) return;
        if (place.segment != loaded) {
            loaded = place.segment;
            s.open_weight(view_of(moe_segment(plan, loaded)), 0);
        }
        s.load(to, place.panel);
    };
    int rows_of = 0;
    auto multiply = [&](const typename Q4Stream<S>::Panel &panel) {
        if (at.segment != summed) {
            moe_add(plan, moe_segment(plan, summed), s.acc, mine);
            s.clear();
            summed = at.segment;
        }
        if (at.segment != rows_of) {
            rows_of = at.segment;
            s.open_rows(view_of(moe_segment(plan, rows_of)), row_of);
        }
        s.multiply(panel, at.panel);
    };
    load(a, at);
    while (at.segment < segments) {
        Place then = next(at);
        load(b, then);
        multiply(a);
        at = then;
        if (at.segment >= segments) break;
        then = next(at);
        load(a, then);
        multiply(b);
        at = then;
    }
    if (summed < segments) moe_add(plan, moe_segment(plan, summed), s.acc, mine);
    __syncthreads();
    moe_finish<S::NB, S::W>(p, totals, n0, cols);
}

template <int G, bool ZEROS>
hipError_t launch_group(const MoeParams &p, hipStream_t stream)
{
    typedef Q4Shape<G, 2, 8, true, ZEROS> Gated;
    typedef Q4Shape<G, 1, 16, false, ZEROS> Down;
    typedef Q4Shape<G, 1, 8, false, ZEROS> DownMany;                // (the totals of 16 waves take 64 KiB for 64 tokens)
    hipLaunchKernelGGL((moe_q4_gated_kernel<Gated>), dim3((unsigned)((p.F + 15) / 16), (unsigned)moe_segments(p.M, p.E, p.k, 16)), dim3(Gated::W * 64), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((p.D + 15) / 16));
    if (p.M <= 16) hipLaunchKernelGGL((moe_q4_down_kernel<Down, 16>), grid, dim3(Down::W * 64), 0, stream, p);
    else hipLaunchKernelGGL((moe_q4_down_kernel<DownMany, kMoeTokens>), grid, dim3(DownMany::W * 64), 0, stream, p);
    return hipGetLastError();
}

template <int G>
hipError_t launch_zeros(const MoeParams &p, hipStream_t stream)
{
    return p.gate.zeros ? launch_group<G, true>(p, stream) : launch_group<G, false>(p, stream);
}

}  // namespace

hipError_t launch_moe_q4(const MoeParams &p, hipStream_t stream)
{
    return p.group == 32 ? launch_zeros<32>(p, stream) : p.group == 64 ? launch_zeros<64>(p, stream) : launch_zeros<128>(p, stream);
}

}  // namespace atb
