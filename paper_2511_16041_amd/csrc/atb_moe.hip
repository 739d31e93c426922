// A mixture of experts for few tokens: l = x R^T, the k experts with the largest l and their shares of softmax(l), y = sum over them of share * Wd (act(Wg x) o (Wu x)).
// Floor: the bytes of the chosen experts' weights.
//
// Four launches.  (1) The router's products in fp64, a wave for one expert and a few tokens: which experts are taken hangs on the order of the l, and in fp32 two that lie close could change places.
// (2) One workgroup: every token's experts, their shares, and the plan, the choices sorted by expert; that of few tokens is part
// of the products.  (3) Gate and up
// products of every expert and its tokens, as the kernel for few rows does them, with the rows of x gathered by the plan; h by place.  (4) The down product: a workgroup has 16 columns of y and
// all experts in turn; its waves take the panels of all of them as one long reduction, and at an expert's end each adds its sums, times the tokens' shares, to its own part of y in LDS.  So every expert's weights
// are read once (of more tokens than a segment's 16 or 32 again), those of no token not at all, the sum over a token's experts is in fp32, in the order of the experts, without atomics, and no token's values meet another's.
// Bound: the bytes of the weights; one token in 4 bits: latency, in the gate and up kernel that of what it waits for in a row (the router's products, the choice, weights, x), and four launches.
// Measured, gate and up / down, us: one token through 2 of 8 experts of 4096 x 14336 80.0 / 43.9, 5.9 and 5.3 TB/s; 21 tokens over 60 of 2056 x 1416 106 / 74, 5.9 and 4.2 (of the 53.4 experts that they choose on average); in 4 bits one token through 8 of 64 of 2048 x 1536
// 14.1 / 7.2, with the router 2.9 and the join 2.7, 32 tokens over 8 of 4096 x 14336 123 / 76, 3.9 and 3.2 TB/s (VALU busy 51 and 44 %; every 16 tokens of an expert decode its weights again).
#include "atb_moe.h"
#include "atb_stream_rows.h"

namespace atb {
namespace {

// ---- the router

// A workgroup for one expert and T tokens, a quarter of every 2048 elements to each wave
template <int T>
__global__ void __launch_bounds__(256) moe_logits_kernel(const MoeParams p)
{
    __shared__ double parts[4][T];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x, m0 = blockIdx.y * T;
    const __bf16 *r = reinterpret_cast<const __bf16 *>(p.router) + e * p.ld_router, *x[T];
#pragma unroll
    for (int t = 0; t < T; ++t) x[t] = reinterpret_cast<const __bf16 *>(p.x) + min(m0 + t, p.M - 1) * p.ldx;
    double sum[T] = {};
#pragma unroll 2
    for (int at = threadIdx.x * 8; at < p.D; at += 2048) {         // D is a multiple of 8
        const bf16x8 w = *reinterpret_cast<const bf16x8 *>(r + at);
        bf16x8 v[T];
#pragma unroll
        for (int t = 0; t < T; ++t) v[t] = *reinterpret_cast<const bf16x8 *>(x[t] + at);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int t = 0; t < T; ++t) sum[t] = fma((double)(float)w[i], (double)(float)v[t][i], sum[t]);
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) sum[t] += __shfl_xor(sum[t], d);
        if (lane == 0) parts[wave][t] = sum[t];
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t < T && m0 + t < p.M) p.logits[(int64_t)(m0 + t) * p.E + e] = parts[0][t] + parts[1][t] + parts[2][t] + parts[3][t];
}

// Every token's choice and the plan.  PER: experts of a lane.  `rows`: of a segment at most.
template <int PER>
__global__ void __launch_bounds__(1024) moe_plan_kernel(const MoeParams p, int rows)
{
    __shared__ unsigned long long tokens[kMoeExperts];             // of an expert, a bit each
    __shared__ int first[kMoeExperts + 1], segment[kMoeExperts + 1];
    __shared__ int chosen[kMoeTokens][kMoeTopK];
    __shared__ float share[kMoeTokens][kMoeTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x < kMoeExperts) tokens[threadIdx.x] = 0;
    __syncthreads();
    // a wave takes a token, and the next one's products are on their way
    double next[PER];
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) next[i] = t < p.M && 64 * i + lane < p.E ? p.logits[(int64_t)t * p.E + 64 * i + lane] : -INFINITY;
    };
    fetch(wave);
    for (int t = wave; t < p.M; t += 16) {
        double mine[PER], left[PER];                               // left: what has not been taken
        int rank[PER];
        bool open[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            mine[i] = next[i];
            rank[i] = p.E;
            open[i] = 64 * i + lane < p.E;
            left[i] = open[i] ? moe_key(mine[i]) : -INFINITY;
        }
        fetch(t + 16);
        // the greatest, of equal ones the first, k times (to count for every expert those ahead of it took 11 us of 21 tokens over 60 experts, this 6)
        for (int c = 0; c < p.k; ++c) {
            double top = -INFINITY;
#pragma unroll
            for (int i = 0; i < PER; ++i) top = fmax(top, left[i]);
            top = lanes_max(top);
            bool found = false;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const unsigned long long equal = found ? 0 : __ballot(open[i] && left[i] == top);
                if (equal && lane == __ffsll(equal) - 1) {
                    rank[i] = c;
                    open[i] = false;
                    left[i] = -INFINITY;
                }
                found = found || equal;
            }
        }
        float weight[PER];
        moe_weights(p, mine, rank, weight);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = 64 * i + lane;
            if (e >= p.E || rank[i] >= p.k) continue;
            chosen[t][rank[i]] = e;
            share[t][rank[i]] = weight[i];
            atomicOr(&tokens[e], 1ull << t);                   // (bits: no order)
            if (p.experts) p.experts[t * p.k + rank[i]] = e;
            if (p.weights) p.weights[t * p.k + rank[i]] = weight[i];
        }
    }
    __syncthreads();
    // first place and segment of every expert, by a sum over the experts before it
    if (wave == 0) {
        int places = 0, segments = 0;
        for (int e0 = 0; e0 < p.E; e0 += 64) {
            const int e = e0 + lane, n = e < p.E ? __popcll(tokens[e]) : 0, s = (n + rows - 1) / rows;
            int at = n, seg = s;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int a = __shfl_up(at, d), b = __shfl_up(seg, d);
                if (lane >= d) { at += a; seg += b; }
            }
            if (e < p.E) {
                first[e] = places + at - n;
                segment[e] = segments + seg - s;
            }
            places += __shfl(at, 63);
            segments += __shfl(seg, 63);
        }
        if (lane == 0) p.plan->segments = segments;
    }
    __syncthreads();
    if (threadIdx.x < p.E) {
        const int e = threadIdx.x, n = __popcll(tokens[e]);
        for (int i = 0; i * rows < n; ++i) {
            p.plan->expert[segment[e] + i] = e;
            p.plan->first[segment[e] + i] = first[e] + i * rows;
            p.plan->rows[segment[e] + i] = min(rows, n - i * rows);
        }
    }
    for (int o = threadIdx.x; o < p.M * p.k; o += 1024) {
        const int t = o / p.k, c = o - t * p.k, e = chosen[t][c], place = first[e] + __popcll(tokens[e] & ((1ull << t) - 1));
        p.plan->token[place] = t;
        p.plan->weight[place] = share[t][c];
    }
}

// ---- the products

template <class S, bool FEW>
__global__ void __launch_bounds__(S::W * 64) moe_gated_kernel(const MoeParams p)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS_BYTES];
    static_assert(S::W == 4 && S::LDS_BYTES >= 12 * 256, "moe_choose_few");
    const MoeFew few = moe_open<FEW>(p, lds);
    const MoeSegment &seg = few.segment;
    if (seg.rows == 0) return;
    const int n0 = blockIdx.x * 16 * S::COLS, cols = min(p.F - n0, 16 * S::COLS);
    const int64_t at = ((int64_t)seg.expert * p.F + n0) * p.D;
    const StreamView view = {p.x, p.ldx, p.M, seg.rows, {static_cast<const uint16_t *>(p.gate.w) + at, static_cast<const uint16_t *>(p.up.w) + at}, {p.D, p.D}, cols, p.D};
    Stream<S> s(view, (unsigned)reinterpret_cast<uintptr_t>(lds), [&](int row) { return moe_token<FEW>(p, few, row); });
    s.run();
    finish_rows<S::MB, S::NB, S::W, true>(moe_inner(p, seg), s.acc, reinterpret_cast<float *>(lds), 0, n0, cols);
}

// Workgroup (x, y): 16 columns of y, share y of the reduction.
template <class S>
__global__ void __launch_bounds__(S::W * 64) moe_down_kernel(const MoeParams p, int segments)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS_BYTES];
    extern __shared__ float totals[];                              // [W][M][16 NB], and the plan of at most `segments`
    const MoeCopy plan = moe_copy(p.plan, reinterpret_cast<int *>(totals + S::W * p.M * 16 * S::NB), segments, p.M * p.k);
    const int n0 = blockIdx.x * 16 * S::COLS, cols = min(p.D - n0, 16 * S::COLS);
    auto view_of = [&](const MoeSegment &seg) {
        return StreamView{p.h + (int64_t)seg.first * p.F, p.F, seg.rows, seg.rows, {static_cast<const uint16_t *>(p.down.w) + ((int64_t)seg.expert * p.D + n0) * p.F, nullptr}, {p.F, 0}, cols, p.F};
    };
    auto row_of = [](int row) { return row; };
    const int panels = (p.F + S::K - 1) / S::K, all = __builtin_amdgcn_readfirstlane(p.plan->segments) * panels;
    __syncthreads();
    const int first = (int)((int64_t)all * blockIdx.y / p.shares), end = (int)((int64_t)all * (blockIdx.y + 1) / p.shares);
    Stream<S> s(view_of(moe_segment(plan, 0)), (unsigned)reinterpret_cast<uintptr_t>(lds), row_of);
    float *mine = totals + s.wave * p.M * 16 * S::NB;
    for (int i = s.lane; i < p.M * 16 * S::NB; i += 64) mine[i] = 0.0f;
    MoePlace<S::W> at(panels, first + s.wave), to = at;             // the panel that is multiplied, the next one that is asked for
    int opened = 0;
    auto request = [&](int slot) {
        if (to.segment != opened) {
            opened = to.segment;
            const StreamView view = view_of(moe_segment(plan, opened));
            s.open_rows(view, row_of);
            s.open_weight(view, 0);
        }
        s.request(to.panel, slot);
        to.next();
    };
    int summed = at.segment, slot = 0;
    if (to.at < end) request(0);
    bool ahead = to.at < end;                                      // whether the panel behind the next one has been asked for
    if (ahead) request(1);
    while (at.at < end) {
        if (at.segment != summed) {
            moe_add(plan, moe_segment(plan, summed), s.acc, mine);
            s.clear();
            summed = at.segment;
        }
        // (what the compiler loads of the plan in between only makes this wait longer)
        if (ahead) Stream<S>::template wait<S::REQS>();
        else Stream<S>::template wait<0>();
        s.multiply(slot);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the buffer is in registers
        ahead = to.at < end;
        if (ahead) request(slot);
        slot ^= 1;
        at.next();
    }
    if (first + s.wave < end) moe_add(plan, moe_segment(plan, summed), s.acc, mine);
    moe_finish<S::NB, S::W>(p, totals, n0, cols);
}

// The shares of y added in order: four columns per thread.  (The workgroup of a column that is done last could add them, without this launch: the fence that its sight of the others' parts takes writes back
// an XCD's whole L2, and two shares of 32 tokens over 8 experts of 4096 x 14336 then took 220 us, one 124.)
__global__ void __launch_bounds__(256) moe_join_kernel(const MoeParams p)
{
    const int pieces = p.D / 4, at = blockIdx.x * 256 + threadIdx.x;
    if (at >= p.M * pieces) return;
    const int token = at / pieces, col = (at - token * pieces) * 4;
    const float *from = p.partial + (int64_t)token * p.D + col;
    floatx4 sum = {};
#pragma unroll 8
    for (int s = 0; s < p.shares; ++s, from += (int64_t)p.M * p.D) sum += *reinterpret_cast<const floatx4 *>(from);
    __bf16 *to = reinterpret_cast<__bf16 *>(p.y) + token * p.ldy + col;
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = (__bf16)sum[e];
}

template <int MB, int XQ>
hipError_t launch_products(const MoeParams &p, hipStream_t stream)
{
    typedef StreamShape<MB, 2, XQ, 4, true> Gated;
    typedef StreamShape<MB, 1, XQ, 8, false> Down;
    const int segments = moe_segments(p.M, p.E, p.k, 16 * MB);
    const dim3 grid((unsigned)((p.F + 15) / 16), (unsigned)segments);
    if (XQ == 1 && p.few) hipLaunchKernelGGL((moe_gated_kernel<Gated, XQ == 1>), grid, dim3(Gated::W * 64), 0, stream, p);
    else hipLaunchKernelGGL((moe_gated_kernel<Gated, false>), grid, dim3(Gated::W * 64), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((moe_down_kernel<Down>), dim3((unsigned)((p.D + 15) / 16), (unsigned)p.shares), dim3(Down::W * 64), (size_t)Down::W * p.M * 16 * sizeof(float) + moe_copy_bytes(segments, p.M * p.k), stream, p, segments);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_moe(const MoeParams &p, hipStream_t stream)
{
    if (p.M == 0) return hipSuccess;
    if (p.M * p.E <= 1024) hipLaunchKernelGGL(moe_logits_kernel<1>, dim3((unsigned)p.E, (unsigned)p.M), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(moe_logits_kernel<4>, dim3((unsigned)p.E, (unsigned)((p.M + 3) / 4)), dim3(256), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = p.group ? 16 : moe_rows(p.M, p.E, p.k);
    if (!p.few) {
        if (p.E <= 64) hipLaunchKernelGGL(moe_plan_kernel<1>, dim3(1), dim3(1024), 0, stream, p, rows);
        else if (p.E <= 128) hipLaunchKernelGGL(moe_plan_kernel<2>, dim3(1), dim3(1024), 0, stream, p, rows);
        else hipLaunchKernelGGL(moe_plan_kernel<4>, dim3(1), dim3(1024), 0, stream, p, rows);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.group) e = launch_moe_q4(p, stream);
    else if (rows == 32) e = launch_products<2, 4>(p, stream);
    else e = p.M <= 8 ? launch_products<1, 1>(p, stream) : launch_products<1, 2>(p, stream);
    if (e != hipSuccess || p.shares == 1) return e;
    hipLaunchKernelGGL(moe_join_kernel, dim3((unsigned)(((int64_t)p.M * (p.D / 4) + 255) / 256)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace atb
