// The products of a mixture of experts with weights in 4 bits (atb_moe.hip has the whole, atb_q4_stream.hip how the weights are multiplied).
#include "atb_moe.h"
#include "atb_q4_rows.h"

namespace atb {
namespace {

template <class S, bool FEW>
__global__ void __launch_bounds__(S::W * 64, S::NB > 2 ? 2 : 4) moe_q4_gated_kernel(const MoeParams p)
{
    __shared__ __attribute__((aligned(16))) float lds[S::W * S::NB * 256];
    static_assert(S::W == 4 && sizeof(lds) >= 12 * 256, "moe_choose_few");
    const MoeFew few = moe_open<FEW>(p, reinterpret_cast<char *>(lds));
    const MoeSegment &seg = few.segment;
    if (seg.rows == 0) return;
    const int n0 = blockIdx.x * 16 * S::COLS, cols = min(p.F - n0, 16 * S::COLS);
    const int64_t n = (int64_t)seg.expert * p.F + n0;
    const Q4View view = {p.x, p.ldx, p.M, seg.rows, {q4_columns(p.gate, n, p.D, S::G), q4_columns(p.up, n, p.D, S::G)}, cols, p.D};
    Q4Stream<S> s(view);
    s.run([&] { s.open_rows(view, [&](int row) { return moe_token<FEW>(p, few, row); }); });
    finish_rows<1, S::NB, S::W, true>(moe_inner(p, seg), s.acc, lds, 0, n0, cols);
}

template <class S>
__global__ void __launch_bounds__(S::W * 64, 2) moe_q4_down_kernel(const MoeParams p, int segments)
{
    extern __shared__ float totals[];                              // [W][M][16 NB], and the plan of at most `segments`
    const MoeCopy plan = moe_copy(p.plan, reinterpret_cast<int *>(totals + S::W * p.M * 16 * S::NB), segments, p.M * p.k);
    const int n0 = blockIdx.x * 16 * S::COLS, cols = min(p.D - n0, 16 * S::COLS);
    auto view_of = [&](const MoeSegment &seg) {
        return Q4View{p.h + (int64_t)seg.first * p.F, p.F, seg.rows, seg.rows, {q4_columns(p.down, (int64_t)seg.expert * p.D + n0, p.F, S::G), {}}, cols, p.F};
    };
    auto row_of = [](int row) { return row; };
    const int panels = (p.F + kQ4PanelK - 1) / kQ4PanelK, all = __builtin_amdgcn_readfirstlane(p.plan->segments) * panels;
    __syncthreads();
    const int first = (int)((int64_t)all * blockIdx.y / p.shares), end = (int)((int64_t)all * (blockIdx.y + 1) / p.shares);
    Q4Stream<S> s(view_of(moe_segment(plan, 0)));
    float *mine = totals + s.wave * p.M * 16 * S::NB;
    for (int i = s.lane; i < p.M * 16 * S::NB; i += 64) mine[i] = 0.0f;
    MoePlace<S::W> at(panels, first + s.wave), to = at;             // the panel that is multiplied, the next one that is asked for
    int loaded = 0, taken = -1, summed = at.segment;                // segments of the weight that is asked for, of x, of the sums
    typename Q4Stream<S>::Panel a, b;
    auto load = [&](typename Q4Stream<S>::Panel &panel) {
        if (to.at >= end) return;
        if (to.segment != loaded) {
            loaded = to.segment;
            s.open_weight(view_of(moe_segment(plan, loaded)), 0);
        }
        s.load(panel, to.panel);
        to.next();
    };
    typename Q4Stream<S>::Rows r;
    auto multiply = [&](const typename Q4Stream<S>::Panel &panel, typename Q4Stream<S>::Panel &behind) {
        if (at.segment != summed) {
            moe_add(plan, moe_segment(plan, summed), s.acc, mine);
            s.clear();
            summed = at.segment;
        }
        if (at.segment != taken) {
            taken = at.segment;
            s.open_rows(view_of(moe_segment(plan, taken)), row_of);
        }
        s.load_rows(r, at.panel);
        load(behind);
        s.multiply(panel, r);
        at.next();
    };
    load(a);
    while (at.at < end) {
        multiply(a, b);
        if (at.at >= end) break;
        multiply(b, a);
    }
    if (first + s.wave < end) moe_add(plan, moe_segment(plan, summed), s.acc, mine);
    moe_finish<S::NB, S::W>(p, totals, n0, cols);
}

// Columns of a workgroup: 16 + 16 of a gated product for up to 8 tokens, beyond 32 + 32, so that x, which takes as many bytes as the weights from 8 rows on, is read half as often (us, one token through
// 8 of 64 experts of 2048 x 1536 12.0 / 14.0, 32 tokens over 8 of 4096 x 14336 134 / 123); 32 of the down product, whose shares make up for the fewer workgroups (7.4 in 16 with as many
// shares as make 512 workgroups and 7.5 in 32; 108 and 80, joining included).
template <int G, bool ZEROS>
hipError_t launch_group(const MoeParams &p, hipStream_t stream)
{
    typedef Q4Shape<G, 2, 4, true, ZEROS> Gated;
    typedef Q4Shape<G, 4, 4, true, ZEROS> GatedWide;
    typedef Q4Shape<G, 2, 8, false, ZEROS> Down;
    const unsigned segments = (unsigned)moe_segments(p.M, p.E, p.k, 16);
    const dim3 narrow((unsigned)((p.F + 15) / 16), segments);
    if (p.few) hipLaunchKernelGGL((moe_q4_gated_kernel<Gated, true>), narrow, dim3(Gated::W * 64), 0, stream, p);
    else if (p.M <= 8) hipLaunchKernelGGL((moe_q4_gated_kernel<Gated, false>), narrow, dim3(Gated::W * 64), 0, stream, p);
    else hipLaunchKernelGGL((moe_q4_gated_kernel<GatedWide, false>), dim3((unsigned)((p.F + 31) / 32), segments), dim3(GatedWide::W * 64), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((moe_q4_down_kernel<Down>), dim3((unsigned)((p.D + 31) / 32), (unsigned)p.shares), dim3(Down::W * 64), (size_t)Down::W * p.M * 32 * sizeof(float) + moe_copy_bytes((int)segments, p.M * p.k), stream, p, (int)segments);
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
