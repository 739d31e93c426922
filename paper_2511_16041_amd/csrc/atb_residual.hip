// Norms on both sides of a residual sum for gfx950, forward and backward: r = a x + g o N1(z), h = N2(r).  Bound: HBM; a small call is its launch.
//
// With xh the normed row before weight and bias (of the root-mean-square norm v / size, without a norm v itself), n1 = xh1 w1 + b1, t the whole gradient of r:
//     t = dr + s2 (dh w2 - [mean(dh w2)] - xh2 mean(dh w2 xh2)),       dx = a t,
//     g1 = t g w1,   dz = s1 (g1 - [mean(g1)] - xh1 mean(g1 xh1)),     [..] of layer norms only,
//     dgate = w1 S1 + b1 S0,   dw1 = sum over groups g S1,   db1 = sum over groups g S0,   S1 = sum t xh1, S0 = sum t over the rows of a gate's group,
//     dw2 = sum dh xh2,   db2 = sum dh,
// so gate, w1 and b1 share two sums, and all parameters need four, of which two fall away without biases.  Rows of up to 8192 elements (forward, and in 16 bits without the sums, 16384) are held in registers and read once; r is computed again in the
// backward pass, which reads x in its place.  A workgroup of the backward pass walks rows of one group and keeps its share of the sums in registers; a second kernel adds them in order,
// a third one the groups.  No atomics: the same bits every time.
// Measured, bf16, root-mean-square norms on both sides: 8192 x 4096 forward 49.5 us, 5.4 TB/s (part of x and z in the memory-side cache), backward 79.3, 5.1 TB/s (waves waiting 44 %), sums 4.8; 2048 x 8192 with one norm 23.0;
// one row of 4096 2.9.  fp32 stream, layer norms with biases, 3000 x 5001, six gates: 44.8, 65.5, sums 7.7 + 4.8 (rows that begin at any element; a workgroup of 640 threads per CU).
#include "atb_block.h"
#include "atb_row.h"

namespace atb {
namespace {

constexpr int E = kResidualPerThread;          // elements of a chunk: 16 bytes of bf16

// A chunk as it lies in memory; 0 past the row's end
template <class T>
struct Raw {
    static constexpr int N = E / Chunk<T>::E;
    typename Chunk<T>::vec v[N];
    ATB_DEV void fetch(const T *row, int at, int D)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = load_chunk<T>(row, at + n * Chunk<T>::E, D);
    }
    // ... of a chunk that lies inside the row
    ATB_DEV void fetch(const T *chunk)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = *reinterpret_cast<const typename Chunk<T>::any *>(chunk + n * Chunk<T>::E);
    }
    ATB_DEV void fill(float x)
    {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e / Chunk<T>::E][e % Chunk<T>::E] = (T)x;
    }
    ATB_DEV float operator[](int e) const { return (float)v[e / Chunk<T>::E][e % Chunk<T>::E]; }
};

// x, which the compiler is not to know ahead of this place: it would keep every comparison with the row's end for the whole kernel, in more registers than there are
ATB_DEV int here(int x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(x));
#endif
    return x;
}

template <class T>
ATB_DEV void store_row(T *row, int at, int D, const float (&v)[E])
{
    constexpr int N = Chunk<T>::E;
#pragma unroll
    for (int n = 0; n < E; n += N) {
        float part[N];
#pragma unroll
        for (int e = 0; e < N; ++e) part[e] = v[n + e];
        if (at + n < D) store<T, N>(row, at + n, D, part);
    }
}

// A parameter's chunk: `other` where there is none, 0 past the row's end
template <class P>
ATB_DEV Raw<P> param(const void *w, int64_t row, int at, int D, float other)
{
    Raw<P> v;
    if (w) v.fetch(static_cast<const P *>(w) + row * D, at, D);
    else v.fill(other);
    return v;
}

// Threads of a row: T, or as many of T as the launch asks for where a row has a workgroup to itself.
template <int T> ATB_DEV int row_threads() { return T >= kResidualThreads ? (int)blockDim.x : T; }

// A thread's chunk c of a row of D >= E elements.  The row's last chunk is moved back to end with the row, and what follows lies in the same place: all chunks are loaded whole, without a branch (a wave in which some
// lanes load and others do not waits for its loads where the two ways meet: the next row was not on its way then, and 3000 x 5000 took 86 us backward where 3000 x 5120 took 57).  Elements before `first` are another
// thread's, or none's.
struct Span {
    int at, first;
    ATB_DEV bool own(int e) const { return e >= first; }
};
template <int T>
ATB_DEV Span span(int c, int t, int D)
{
    const int from = here((c * row_threads<T>() + t) * E), at = min(from, D - E);
    return {at, from - at};
}
template <class T>
ATB_DEV void store_span(T *row, const Span &s, const float (&v)[E])
{
    constexpr int N = Chunk<T>::E;
    if (s.first == 0) {
#pragma unroll
        for (int n = 0; n < E; n += N) {
            typename Chunk<T>::vec w;
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = (T)v[n + e];
            *reinterpret_cast<typename Chunk<T>::any *>(row + s.at + n) = w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (s.own(e)) row[s.at + e] = (T)v[e];
    }
}
// A parameter's chunk: `other` where there is none
template <class P>
ATB_DEV Raw<P> param(const void *w, int64_t row, const Span &s, int D, float other)
{
    Raw<P> v;
    if (w) v.fetch(static_cast<const P *>(w) + row * D + s.at);
    else v.fill(other);
    return v;
}

// The sums of a row over its threads; two areas of scratch in turns, so that one barrier is enough
template <int T, int NT>
struct RowSums {
    float (*scratch)[2 * NT / 64];
    int turn = 0;
    ATB_DEV RowSums(float (*scratch_)[2 * NT / 64]) : scratch(scratch_)
    {
        if constexpr (T >= kResidualThreads) {                // waves that are not there add nothing
            for (int i = threadIdx.x; i < 2 * 2 * NT / 64; i += blockDim.x) scratch[0][i] = 0.0f;
            __syncthreads();
        }
    }
    template <int N>
    ATB_DEV void operator()(float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i]);
        if constexpr (T > 64) {
            constexpr int W = T / 64;
            const int wave = threadIdx.x >> 6;
            float *here = scratch[turn];
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) here[wave * N + i] = v[i];
            __syncthreads();
            const float *mine = here + (T >= kResidualThreads ? 0 : wave / W * W * N);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) s += mine[w * N + i];
                v[i] = s;
            }
            turn ^= 1;
        }
    }
};

// Elements that are not this thread's own, as 0: in the few waves that have any
ATB_DEV void clear_before(float (&v)[E], int first)
{
    if (first > 0) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < first) v[e] = 0.0f;
    }
}

// v becomes the normed row, without weight and bias; what is not this thread's is 0 before and anything behind
template <int T, int NT, int C>
ATB_DEV void normalise(float (&v)[C][E], int kind, float eps, int t, int D, RowSums<T, NT> &sums, float &mean, float &rstd)
{
    mean = 0.0f;
    float s[1] = {0.0f};
    if (kind == ATB_NORM_LAYER) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) s[0] += v[c][e];
        sums(s);
        mean = s[0] / (float)D;
        s[0] = 0.0f;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const Span own = span<T>(c, t, D);
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] -= mean;
        clear_before(v[c], own.first);
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] += v[c][e] * v[c][e];
    }
    sums(s);
    rstd = 1.0f / sqrtf(s[0] / (float)D + eps);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] *= rstd;
}

// T threads per row with C chunks each, NT / T rows of a workgroup at a time.  Rows of one chunk: the parameters are held, and the next row is on its way while one is normed.
template <class X, class Z, class P, int T, int C>
__global__ void __launch_bounds__(T < 256 ? 256 : T) residual_kernel(const ResidualParams p, int rounds)
{
    constexpr int NT = T < 256 ? 256 : T, R = NT / T;
    constexpr bool HOLD = C == 1;
    __shared__ float scratch[2][2 * NT / 64];
    RowSums<T, NT> sums(scratch);
    const int t = T >= kResidualThreads ? threadIdx.x : threadIdx.x % T, group = T >= kResidualThreads ? 0 : threadIdx.x / T, D = p.D;
    const int64_t per_gate = p.M / p.groups;
    Raw<X> next_x[C];
    Raw<Z> next_z[C];
    Raw<P> w1[HOLD ? C : 1], b1[HOLD ? C : 1], w2[HOLD ? C : 1], b2[HOLD ? C : 1], next_gate[HOLD ? C : 1];
    auto fetch = [&](int64_t row) {
        row = row < p.M ? row : 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Span own = span<T>(c, t, D);
            next_z[c].fetch(static_cast<const Z *>(p.z) + row * p.ldz + own.at);
            next_x[c].fetch(static_cast<const X *>(p.x) + row * p.ldx + own.at);
        }
        if (HOLD && p.groups > 1) {
#pragma unroll
            for (int c = 0; c < (HOLD ? C : 1); ++c) next_gate[c] = param<P>(p.gate, row / per_gate, span<T>(c, t, D), D, 1.0f);
        }
    };
    if constexpr (HOLD) {
#pragma unroll
        for (int c = 0; c < C; ++c) next_gate[c] = param<P>(p.gate, 0, span<T>(c, t, D), D, 1.0f);
    }
    fetch((int64_t)blockIdx.x * R + group);
    if constexpr (HOLD) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Span own = span<T>(c, t, D);
            w1[c] = param<P>(p.post.weight, 0, own, D, 1.0f);
            b1[c] = param<P>(p.post.bias, 0, own, D, 0.0f);
            w2[c] = param<P>(p.pre.weight, 0, own, D, 1.0f);
            b2[c] = param<P>(p.pre.bias, 0, own, D, 0.0f);
        }
    }
    for (int n = 0; n < rounds; ++n) {                        // the same number for every thread of the workgroup
        const int64_t row = ((int64_t)n * gridDim.x + blockIdx.x) * R + group;
        Raw<X> x[C];
        Raw<P> gate[HOLD ? C : 1];
        float v[C][E];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Span own = span<T>(c, t, D);
            x[c] = next_x[c];
            if constexpr (HOLD) gate[c] = next_gate[c];
#pragma unroll
            for (int e = 0; e < E; ++e) v[c][e] = next_z[c][e];
            clear_before(v[c], own.first);
        }
        if (HOLD && n + 1 < rounds) fetch(row + (int64_t)gridDim.x * R);
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (p.post.kind != ATB_NORM_NONE) normalise<T, NT, C>(v, p.post.kind, p.post.eps, t, D, sums, mean1, rstd1);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Span own = span<T>(c, t, D);
            const Raw<P> w = HOLD ? w1[HOLD ? c : 0] : param<P>(p.post.weight, 0, own, D, 1.0f), b = HOLD ? b1[HOLD ? c : 0] : param<P>(p.post.bias, 0, own, D, 0.0f);
            const Raw<P> g = HOLD ? gate[HOLD ? c : 0] : param<P>(p.gate, p.groups > 1 && row < p.M ? row / per_gate : 0, own, D, 1.0f);
#pragma unroll
            for (int e = 0; e < E; ++e) v[c][e] = p.scale * x[c][e] + g[e] * (v[c][e] * w[e] + b[e]);
            clear_before(v[c], own.first);
            if (row < p.M) store_span(static_cast<X *>(p.r) + row * p.ldr, own, v[c]);
            if (C > 1) __builtin_amdgcn_sched_barrier(0);     // chunk by chunk: registers
        }
        if (p.pre.kind != ATB_NORM_NONE) {
            normalise<T, NT, C>(v, p.pre.kind, p.pre.eps, t, D, sums, mean2, rstd2);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const Span own = span<T>(c, t, D);
                const Raw<P> w = HOLD ? w2[HOLD ? c : 0] : param<P>(p.pre.weight, 0, own, D, 1.0f), b = HOLD ? b2[HOLD ? c : 0] : param<P>(p.pre.bias, 0, own, D, 0.0f);
#pragma unroll
                for (int e = 0; e < E; ++e) v[c][e] = v[c][e] * w[e] + b[e];
                if (row < p.M) store_span(static_cast<Z *>(p.h) + row * p.ldh, own, v[c]);
                if (C > 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (p.stats && t == 0 && row < p.M) {
            p.stats[row] = mean1;
            p.stats[p.M + row] = rstd1;
            p.stats[2 * p.M + row] = mean2;
            p.stats[3 * p.M + row] = rstd2;
        }
        if (!HOLD && n + 1 < rounds) fetch(row + (int64_t)gridDim.x * R);
    }
}

// The statistics of a row
struct RowStats {
    float mean1, rstd1, mean2, rstd2;
    ATB_DEV void fetch(const ResidualParams &p, int64_t row)
    {
        mean1 = p.stats[row];
        rstd1 = p.stats[p.M + row];
        mean2 = p.stats[2 * p.M + row];
        rstd2 = p.stats[3 * p.M + row];
    }
};

// dx, dz and (SUMS) the workgroup's part of the sums over rows, [group][part][SUMS][D]: S1, dw2's, S0, db2's.  T threads per row with C chunks each.
// rows: of rows whose sums residual_columns_kernel takes (C > 2), where their two means go, or null.
template <class X, class Z, class P, int T, int C, int SUMS>
__global__ void __launch_bounds__(T > kResidualThreads ? T : kResidualThreads) residual_grad_kernel(const ResidualParams p, int parts, int rounds, float *rows)
{
    constexpr int NT = T > kResidualThreads ? T : kResidualThreads, R = NT / T;
    // registers: the next row's operands (dr, which is used last, on its own) and the parameters are held unless they would not fit
    constexpr bool TIGHT = T > kResidualThreads && sizeof(X) == 4, LARGE = TIGHT && sizeof(Z) == 4;
    constexpr bool AHEAD = C == 1 ? !LARGE : C == 2 && sizeof(X) == 2 && SUMS < 4, DR_AHEAD = AHEAD && !TIGHT, HOLD = C == 1 ? !TIGHT || sizeof(P) == 2 : C == 2 && sizeof(P) == 2;
    __shared__ float scratch[2][2 * NT / 64];
    RowSums<T, NT> sums(scratch);
    const int t = T >= kResidualThreads ? threadIdx.x : threadIdx.x % T, group = T >= kResidualThreads ? 0 : threadIdx.x / T, D = p.D;
    const int64_t per_gate = p.M / p.groups, gate_row = blockIdx.x / parts, part = blockIdx.x % parts;
    const bool normed1 = p.post.kind != ATB_NORM_NONE, normed2 = p.pre.kind != ATB_NORM_NONE;
    const bool centred1 = p.post.kind == ATB_NORM_LAYER, centred2 = p.pre.kind == ATB_NORM_LAYER;
    const float inv = 1.0f / (float)D;
    struct Params { Raw<P> w1, b1, w2, gate; };
    Params held[HOLD ? C : 1];
    auto params = [&](int c) {
        const Span own = span<T>(c, t, D);
        return Params{param<P>(p.post.weight, 0, own, D, 1.0f), param<P>(p.post.bias, 0, own, D, 0.0f), param<P>(p.pre.weight, 0, own, D, 1.0f), param<P>(p.gate, gate_row, own, D, 1.0f)};
    };
    if constexpr (HOLD) {
#pragma unroll
        for (int c = 0; c < C; ++c) held[c] = params(c);
    }
    float sum[SUMS > 0 ? SUMS : 1][C][E] = {};
    Raw<X> next_x[C], next_dr[C];
    Raw<Z> next_z[C], next_dh[C];
    RowStats next;
    // the row that turn n brings to this thread's row group; past the group's end its first one, which is not used
    auto row_of = [&](int n, bool &live) {
        const int64_t in_group = ((int64_t)n * parts + part) * R + group;
        live = in_group < per_gate;
        return gate_row * per_gate + (live ? in_group : 0);
    };
    auto fetch = [&](int64_t row) {
        next.fetch(p, row);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Span own = span<T>(c, t, D);
            next_x[c].fetch(static_cast<const X *>(p.x) + row * p.ldx + own.at);
            next_z[c].fetch(static_cast<const Z *>(p.z) + row * p.ldz + own.at);
            if (normed2) next_dh[c].fetch(static_cast<const Z *>(p.dh) + row * p.lddh + own.at);
            else next_dh[c].fill(0.0f);
        }
    };
    auto fetch_dr = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (p.dr) next_dr[c].fetch(static_cast<const X *>(p.dr) + row * p.lddr + span<T>(c, t, D).at);
            else next_dr[c].fill(0.0f);
        }
    };
    bool next_live = false;
    int64_t next_row = row_of(0, next_live);
    if (AHEAD) fetch(next_row);
    if (DR_AHEAD) fetch_dr(next_row);
    for (int n = 0; n < rounds; ++n) {                        // the same number for every thread of the workgroup
        const int64_t row = next_row;
        const bool live = next_live;
        if (!AHEAD) fetch(row);
        if (!DR_AHEAD) fetch_dr(row);
        const RowStats st = next;
        float xh1[C][E], xh2[C][E], g[C][E], s[2] = {0.0f, 0.0f};
        Raw<X> dr[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Params k = HOLD ? held[HOLD ? c : 0] : params(c);
            const Span own = span<T>(c, t, D);
            dr[c] = next_dr[c];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float dh = next_dh[c][e];
                xh1[c][e] = (next_z[c][e] - st.mean1) * st.rstd1;
                const float r = p.scale * next_x[c][e] + k.gate[e] * (xh1[c][e] * k.w1[e] + k.b1[e]);
                xh2[c][e] = (r - st.mean2) * st.rstd2;
                if constexpr (SUMS > 0) {
                    if (live) {
                        sum[1][c][e] += dh * xh2[c][e];
                        if constexpr (SUMS > 2) sum[SUMS - 1][c][e] += dh;
                    }
                }
                g[c][e] = dh * k.w2[e];
            }
            clear_before(g[c], own.first);                    // (the products: a weight may be infinite)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                s[0] += g[c][e];
                s[1] += g[c][e] * xh2[c][e];
            }
            if (C > 1) __builtin_amdgcn_sched_barrier(0);     // chunk by chunk: registers
        }
        if (n + 1 < rounds) {                                 // the next row is on its way while this one is summed
            next_row = row_of(n + 1, next_live);
            if (AHEAD) fetch(next_row);
            if (DR_AHEAD) fetch_dr(next_row);
        }
        if (normed2) sums(s);
        const float m0 = centred2 ? s[0] * inv : 0.0f, m1 = s[1] * inv;       // (selected: a sum that is not needed may be infinite, and times 0 NaN)
        if (C > 2 && rows && live && t == 0) {
            rows[row] = m0;
            rows[p.M + row] = m1;
        }
        float q[2] = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Params k = HOLD ? held[HOLD ? c : 0] : params(c);
            const Span own = span<T>(c, t, D);
            float d[E], out[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                d[e] = dr[c][e];
                if (normed2) d[e] += st.rstd2 * (g[c][e] - m0 - xh2[c][e] * m1);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if constexpr (SUMS > 0) {
                    if (live) {
                        sum[0][c][e] += d[e] * xh1[c][e];
                        if constexpr (SUMS > 2) sum[SUMS - 2][c][e] += d[e];
                    }
                }
                out[e] = p.scale * d[e];
                g[c][e] = d[e] * k.gate[e] * k.w1[e];
            }
            clear_before(g[c], own.first);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                q[0] += g[c][e];
                q[1] += g[c][e] * xh1[c][e];
            }
            if (live && p.dx) store_span(static_cast<X *>(p.dx) + row * p.lddx, own, out);
            if (C > 1) __builtin_amdgcn_sched_barrier(0);
        }
        if (normed1) {
            sums(q);
            const float n0 = centred1 ? q[0] * inv : 0.0f, n1 = q[1] * inv;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) g[c][e] = st.rstd1 * (g[c][e] - n0 - xh1[c][e] * n1);
        }
        if (live && p.dz) {
#pragma unroll
            for (int c = 0; c < C; ++c) store_span(static_cast<Z *>(p.dz) + row * p.lddz, span<T>(c, t, D), g[c]);
        }
    }
    if constexpr (SUMS > 0) {
        // the row groups' sums, the upper half of the groups onto the lower one in every step
        if constexpr (R > 1) {
            static_assert(C == 1, "longer rows have a workgroup to themselves");
            __shared__ float room[R / 2 * SUMS * E * T];                     // [R / 2][SUMS][E][T]
#pragma unroll
            for (int half = R / 2; half >= 1; half /= 2) {
                __syncthreads();
                if (group >= half && group < 2 * half) {
#pragma unroll
                    for (int i = 0; i < SUMS; ++i)
#pragma unroll
                        for (int e = 0; e < E; ++e) room[(((group - half) * SUMS + i) * E + e) * T + t] = sum[i][0][e];
                }
                __syncthreads();
                if (group < half) {
#pragma unroll
                    for (int i = 0; i < SUMS; ++i)
#pragma unroll
                        for (int e = 0; e < E; ++e) sum[i][0][e] += room[((group * SUMS + i) * E + e) * T + t];
                }
            }
            if (group > 0) return;
        }
        float *to = p.workspace + (int64_t)blockIdx.x * SUMS * D;
#pragma unroll
        for (int i = 0; i < SUMS; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c) store_span(to + (int64_t)i * D, span<T>(c, t, D), sum[i][c]);
    }
}

// ---- rows of more than kResidualMaxGradRow elements, or of less than a chunk: read again for every sum, from the second time on out of a cache

// This thread's share of sums over a row: f(at, sums) adds the chunk at `at`; 16 chunks at a time, so that no chain of additions is longer than 128 and D / 2^16
template <int N, class F>
ATB_DEV void add_chunks(int D, float (&sums)[N], F f)
{
    constexpr int RUN = 16 * kResidualThreads * E;
#pragma unroll
    for (int n = 0; n < N; ++n) sums[n] = 0.0f;
    for (int from = 0; from < D; from += RUN) {
        float run[N] = {};
        const int end = min(D, from + RUN);
        for (int at = from + threadIdx.x * E; at < end; at += kResidualThreads * E) f(at, run);
#pragma unroll
        for (int n = 0; n < N; ++n) sums[n] += run[n];
    }
}

// The statistics of a row whose elements f(at, v) gives, a chunk at a time
template <class F>
ATB_DEV void long_stats(int kind, float eps, int D, RowSums<kResidualThreads, kResidualThreads> &sums, F f, float &mean, float &rstd)
{
    float s[1];
    mean = 0.0f;
    if (kind == ATB_NORM_LAYER) {
        add_chunks(D, s, [&](int at, float (&sum)[1]) {
            float v[E];
            f(at, v);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += at + e < D ? v[e] : 0.0f;
        });
        sums(s);
        mean = s[0] / (float)D;
    }
    add_chunks(D, s, [&](int at, float (&sum)[1]) {
        float v[E];
        f(at, v);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[0] += at + e < D ? (v[e] - mean) * (v[e] - mean) : 0.0f;
    });
    sums(s);
    rstd = 1.0f / sqrtf(s[0] / (float)D + eps);
}

// A chunk of r, in fp32, and of the normed z
template <class X, class Z, class P>
ATB_DEV void long_sum(const ResidualParams &p, int64_t row, int64_t gate_row, int at, float mean1, float rstd1, float (&xh1)[E], float (&r)[E])
{
    const int D = p.D;
    Raw<X> x;
    Raw<Z> z;
    x.fetch(static_cast<const X *>(p.x) + row * p.ldx, at, D);
    z.fetch(static_cast<const Z *>(p.z) + row * p.ldz, at, D);
    const Raw<P> w = param<P>(p.post.weight, 0, at, D, 1.0f);
    const Raw<P> b = param<P>(p.post.bias, 0, at, D, 0.0f);
    const Raw<P> g = param<P>(p.gate, gate_row, at, D, 1.0f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        xh1[e] = (z[e] - mean1) * rstd1;
        r[e] = p.scale * x[e] + g[e] * (xh1[e] * w[e] + b[e]);
    }
}

template <class X, class Z, class P>
__global__ void __launch_bounds__(kResidualThreads) residual_long_kernel(const ResidualParams p)
{
    __shared__ float scratch[2][2 * kResidualThreads / 64];
    RowSums<kResidualThreads, kResidualThreads> sums(scratch);
    const int D = p.D;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        const int64_t gate_row = row / (p.M / p.groups);
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (p.post.kind != ATB_NORM_NONE)
            long_stats(p.post.kind, p.post.eps, D, sums, [&](int at, float (&v)[E]) {
                Raw<Z> z;
                z.fetch(static_cast<const Z *>(p.z) + row * p.ldz, at, D);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = z[e];
            }, mean1, rstd1);
        if (p.pre.kind != ATB_NORM_NONE)
            long_stats(p.pre.kind, p.pre.eps, D, sums, [&](int at, float (&v)[E]) {
                float xh1[E];
                long_sum<X, Z, P>(p, row, gate_row, at, mean1, rstd1, xh1, v);
            }, mean2, rstd2);
        for (int at = threadIdx.x * E; at < D; at += kResidualThreads * E) {
            float xh1[E], v[E];
            long_sum<X, Z, P>(p, row, gate_row, at, mean1, rstd1, xh1, v);
            store_row<X>(static_cast<X *>(p.r) + row * p.ldr, at, D, v);
            if (p.pre.kind != ATB_NORM_NONE) {
                const Raw<P> w = param<P>(p.pre.weight, 0, at, D, 1.0f);
                const Raw<P> b = param<P>(p.pre.bias, 0, at, D, 0.0f);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = (v[e] - mean2) * rstd2 * w[e] + b[e];
                store_row<Z>(static_cast<Z *>(p.h) + row * p.ldh, at, D, v);
            }
        }
        if (p.stats && threadIdx.x == 0) {
            p.stats[row] = mean1;
            p.stats[p.M + row] = rstd1;
            p.stats[2 * p.M + row] = mean2;
            p.stats[3 * p.M + row] = rstd2;
        }
    }
}

// The gradient of r but for its means, and what they are taken of
struct LongGrad { float xh1[E], xh2[E], g[E], dr[E], dh[E]; };
template <class X, class Z, class P>
ATB_DEV void long_grad(const ResidualParams &p, const RowStats &st, int64_t row, int64_t gate_row, int at, bool normed2, LongGrad &l)
{
    const int D = p.D;
    float r[E];
    long_sum<X, Z, P>(p, row, gate_row, at, st.mean1, st.rstd1, l.xh1, r);
    Raw<X> dr;
    Raw<Z> dh;
    dr.fill(0.0f);
    dh.fill(0.0f);
    if (p.dr) dr.fetch(static_cast<const X *>(p.dr) + row * p.lddr, at, D);
    if (normed2) dh.fetch(static_cast<const Z *>(p.dh) + row * p.lddh, at, D);
    const Raw<P> u = param<P>(p.pre.weight, 0, at, D, 1.0f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        l.xh2[e] = (r[e] - st.mean2) * st.rstd2;
        l.dr[e] = dr[e];
        l.dh[e] = dh[e];
        l.g[e] = l.dh[e] * u[e];
    }
}

// dx, dz, and the two means of a row's dh w2 to `rows` for the pass that takes the sums over rows.
template <class X, class Z, class P>
__global__ void __launch_bounds__(kResidualThreads) residual_grad_long_kernel(const ResidualParams p, float *rows)
{
    __shared__ float scratch[2][2 * kResidualThreads / 64];
    RowSums<kResidualThreads, kResidualThreads> sums(scratch);
    const int D = p.D;
    const bool normed1 = p.post.kind != ATB_NORM_NONE, normed2 = p.pre.kind != ATB_NORM_NONE;
    const bool centred1 = p.post.kind == ATB_NORM_LAYER, centred2 = p.pre.kind == ATB_NORM_LAYER;
    const float inv = 1.0f / (float)D;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        const int64_t gate_row = row / (p.M / p.groups);
        RowStats st;
        st.fetch(p, row);
        float m0 = 0.0f, m1 = 0.0f, n0 = 0.0f, n1 = 0.0f;
        if (normed2) {
            float s[2];
            add_chunks(D, s, [&](int at, float (&sum)[2]) {
                LongGrad l;
                long_grad<X, Z, P>(p, st, row, gate_row, at, true, l);
#pragma unroll
                for (int e = 0; e < E; ++e) {                  // (0 past the end)
                    sum[0] += l.g[e];
                    sum[1] += l.g[e] * l.xh2[e];
                }
            });
            sums(s);
            m0 = centred2 ? s[0] * inv : 0.0f;
            m1 = s[1] * inv;
        }
        if (rows && threadIdx.x == 0) {
            rows[row] = m0;
            rows[p.M + row] = m1;
        }
        // dx, and dz but for its means
        auto inner = [&](int at, float (&d)[E], float (&g1)[E], float (&xh1)[E]) {
            LongGrad l;
            long_grad<X, Z, P>(p, st, row, gate_row, at, normed2, l);
            const Raw<P> w = param<P>(p.post.weight, 0, at, D, 1.0f);
            const Raw<P> k = param<P>(p.gate, gate_row, at, D, 1.0f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                d[e] = l.dr[e];
                if (normed2) d[e] += st.rstd2 * (l.g[e] - m0 - l.xh2[e] * m1);
                if (at + e >= D) d[e] = 0.0f;
                g1[e] = d[e] * k[e] * w[e];
                xh1[e] = l.xh1[e];
            }
        };
        if (normed1 && p.dz) {
            float q[2];
            add_chunks(D, q, [&](int at, float (&sum)[2]) {
                float d[E], g1[E], xh1[E];
                inner(at, d, g1, xh1);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    sum[0] += g1[e];
                    sum[1] += g1[e] * xh1[e];
                }
            });
            sums(q);
            n0 = centred1 ? q[0] * inv : 0.0f;
            n1 = q[1] * inv;
        }
        if (!p.dx && !p.dz) continue;
        for (int at = threadIdx.x * E; at < D; at += kResidualThreads * E) {
            float d[E], g1[E], xh1[E];
            inner(at, d, g1, xh1);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                d[e] *= p.scale;
                if (normed1) g1[e] = st.rstd1 * (g1[e] - n0 - xh1[e] * n1);
            }
            if (p.dx) store_row<X>(static_cast<X *>(p.dx) + row * p.lddx, at, D, d);
            if (p.dz) store_row<Z>(static_cast<Z *>(p.dz) + row * p.lddz, at, D, g1);
        }
    }
}

// The sums over rows: a thread has a chunk of columns of a part of a group's rows, one after the other.
template <class X, class Z, class P, int SUMS>
__global__ void __launch_bounds__(256) residual_columns_kernel(const ResidualParams p, int blocks, const float *rows)
{
    const int D = p.D, at = (blockIdx.x % blocks * 256 + threadIdx.x) * E, mine = blockIdx.x / blocks;
    if (at >= D) return;
    const int64_t per_gate = p.M / p.groups, gate_row = mine / p.parts, part = mine % p.parts;
    const bool normed2 = p.pre.kind != ATB_NORM_NONE;
    float sum[SUMS][E] = {};
    for (int64_t i = part; i < per_gate; i += p.parts) {
        const int64_t row = gate_row * per_gate + i;
        RowStats st;
        st.fetch(p, row);
        const float m0 = rows[row], m1 = rows[p.M + row];
        LongGrad l;
        long_grad<X, Z, P>(p, st, row, gate_row, at, normed2, l);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float d = l.dr[e];
            if (normed2) d += st.rstd2 * (l.g[e] - m0 - l.xh2[e] * m1);
            sum[0][e] += d * l.xh1[e];
            sum[1][e] += l.dh[e] * l.xh2[e];
            if constexpr (SUMS > 2) {
                sum[SUMS - 2][e] += d;
                sum[SUMS - 1][e] += l.dh[e];
            }
        }
    }
    float *out = p.workspace + (int64_t)mine * SUMS * D;
#pragma unroll
    for (int i = 0; i < SUMS; ++i) store_row<float>(out + (int64_t)i * D, at, D, sum[i]);
}

// ---- the sums' parts

// Sums over `count` numbers that lie `pitch` floats apart, N of them `apart` floats from sum to sum.  A workgroup of 1024 threads has COLS columns, each of its groups of COLS threads a run of the numbers, 64 at a time
// (shorter chains); the groups' parts are added in order.  What comes back belongs to column threadIdx.x of the first COLS threads.
template <int COLS, int N>
ATB_DEV void sum_columns(const float *from, int64_t pitch, int64_t apart, int count, bool live, float (&s)[N], float (*scratch)[N][COLS])
{
    constexpr int GROUPS = 1024 / COLS;
    const int lane = threadIdx.x % COLS, part = threadIdx.x / COLS, run = (count + GROUPS - 1) / GROUPS, first = part * run, end = live ? min(first + run, count) : 0;
    from += first * pitch;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.0f;
    for (int at = first; at < end; at += 64) {
        const int stop = min(end, at + 64);
        float chain[N] = {};
#pragma unroll 8
        for (int n = at; n < stop; ++n, from += pitch)
#pragma unroll
            for (int i = 0; i < N; ++i) chain[i] += from[i * apart];
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += chain[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) scratch[part][i][lane] = s[i];
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = 0.0f;
        for (int from_group = 0; from_group < GROUPS; from_group += 16) {
            float sixteen = 0.0f;
#pragma unroll
            for (int n = 0; n < 16; ++n) sixteen += scratch[from_group + n][i][lane];
            s[i] += sixteen;
        }
    }
}

// The parts of a group's sums, and its gate's gradient; with one group the other parameters' too, else their terms for residual_groups_kernel.
template <class P, int SUMS, int COLS>
__global__ void __launch_bounds__(1024) residual_params_kernel(const ResidualParams p, float *totals)
{
    __shared__ float scratch[1024 / COLS][SUMS][COLS];
    const int D = p.D, col = blockIdx.x * COLS + threadIdx.x % COLS;
    const int64_t g = blockIdx.y;
    float run[SUMS];
    sum_columns<COLS, SUMS>(p.workspace + g * p.parts * SUMS * D + col, (int64_t)SUMS * D, D, p.parts, col < D, run, scratch);
    if (threadIdx.x >= COLS || col >= D) return;
    float s[4] = {};
#pragma unroll
    for (int i = 0; i < SUMS; ++i) s[i] = run[i];
    const bool normed1 = p.post.kind != ATB_NORM_NONE;
    auto value = [&](const void *w, int64_t at, float other) { return w ? (float)static_cast<const P *>(w)[at] : other; };
    if (p.dgate) {
        // (a factor of 0 takes its sum out: that may be infinite, and times 0 NaN, where sum t n1 is not)
        const float w = value(normed1 ? p.post.weight : nullptr, col, 1.0f), b = value(normed1 ? p.post.bias : nullptr, col, 0.0f);
        static_cast<P *>(p.dgate)[g * D + col] = (P)(b == 0.0f ? w * s[0] : w == 0.0f ? b * s[2] : w * s[0] + b * s[2]);
    }
    const float gate = value(p.gate, g * D + col, 1.0f);
    s[0] *= gate;
    s[2] *= gate;
    if (totals) {
#pragma unroll
        for (int i = 0; i < SUMS; ++i) totals[(g * SUMS + i) * D + col] = s[i];
        return;
    }
    if (p.dpost_weight) static_cast<P *>(p.dpost_weight)[col] = (P)s[0];
    if (p.dpre_weight) static_cast<P *>(p.dpre_weight)[col] = (P)s[1];
    if (p.dpost_bias) static_cast<P *>(p.dpost_bias)[col] = (P)s[2];
    if (p.dpre_bias) static_cast<P *>(p.dpre_bias)[col] = (P)s[3];
}

// The groups' terms, one sum to a workgroup.
template <class P, int SUMS>
__global__ void __launch_bounds__(1024) residual_groups_kernel(const ResidualParams p, const float *totals)
{
    __shared__ float scratch[16][1][64];
    const int D = p.D, col = blockIdx.x * 64 + threadIdx.x % 64, i = blockIdx.y;
    P *out = static_cast<P *>(i == 0 ? p.dpost_weight : i == 1 ? p.dpre_weight : i == 2 ? p.dpost_bias : p.dpre_bias);
    if (!out) return;                                         // the whole workgroup
    float s[1];
    sum_columns<64, 1>(totals + (int64_t)i * D + col, (int64_t)SUMS * D, 0, (int)p.groups, col < D, s, scratch);
    if (threadIdx.x < 64 && col < D) out[col] = (P)s[0];
}

// ---- launches

constexpr int64_t kMostWorkgroups = 1 << 20;        // of a launch; each walks rows a grid apart

// Threads of a workgroup: where a row has it to itself as many waves as the row fills
template <int T, int C>
int workgroup(int D, int least) { return T >= kResidualThreads ? (D + C * E * 64 - 1) / (C * E * 64) * 64 : std::max(T, least); }

// Rows of one chunk per thread: workgroups of 16 waves per CU in all walk the rows (8192 x 4096 in bf16, 16 waves 57 us, 8 77, a workgroup for every row 75, as the rest was then).  Of longer rows, with twice the registers for
// the row alone, one per workgroup (2048 x 8192 in bf16 25 us either way, 3000 x 5001 with an fp32 stream 47, walking with 12 waves 62).
template <class X, class Z, class P, int T, int C>
hipError_t forward_of(const ResidualParams &p, hipStream_t stream)
{
    constexpr int NT = T < 256 ? 256 : T, R = NT / T;
    const int64_t all = (p.M + R - 1) / R, grid = std::min(all, C == 1 ? (int64_t)256 * (1024 / NT) : kMostWorkgroups);
    hipLaunchKernelGGL((residual_kernel<X, Z, P, T, C>), dim3((unsigned)grid), dim3(workgroup<T, C>(p.D, 256)), 0, stream, p, (int)((all + grid - 1) / grid));
    return hipGetLastError();
}

template <class X, class Z, class P, int T, int C, int SUMS>
hipError_t backward_of(const ResidualParams &p, hipStream_t stream, float *rows = nullptr)
{
    constexpr int NT = T > kResidualThreads ? T : kResidualThreads, R = NT / T;
    const int64_t per_gate = p.M / p.groups, turns = (per_gate + R - 1) / R;
    const int64_t parts = SUMS > 0 ? p.parts : std::min<int64_t>(turns, std::max<int64_t>(1, 2048 / p.groups));
    hipLaunchKernelGGL((residual_grad_kernel<X, Z, P, T, C, SUMS>), dim3((unsigned)(p.groups * parts)), dim3(workgroup<T, C>(p.D, NT)), 0, stream, p, (int)parts, (int)((turns + parts - 1) / parts), rows);
    return hipGetLastError();
}

template <class X, class Z, class P, int SUMS>
hipError_t backward_rows(const ResidualParams &p, hipStream_t stream)
{
    switch (residual_threads(p.D)) {
        case 64: return backward_of<X, Z, P, 64, 1, SUMS>(p, stream);
        case 128: return backward_of<X, Z, P, 128, 1, SUMS>(p, stream);
        case 256: return backward_of<X, Z, P, 256, 1, SUMS>(p, stream);
        default:
            if (p.D <= 512 * E) return backward_of<X, Z, P, 512, 1, SUMS>(p, stream);
            return p.D <= 768 * E ? backward_of<X, Z, P, 768, 1, SUMS>(p, stream) : backward_of<X, Z, P, 512, 2, SUMS>(p, stream);
    }
}

template <class X, class Z, class P, int SUMS>
hipError_t sums_of(const ResidualParams &p, float *rows, float *totals, hipStream_t stream)
{
    if (p.M > 0 && residual_is_long(p.D)) {
        const int64_t blocks = (p.D + 256 * E - 1) / (256 * E);
        if (blocks * p.groups * p.parts > 0xffffff) return hipErrorInvalidConfiguration;       // (2^32 threads: operands of 64 GiB each)
        hipLaunchKernelGGL((residual_columns_kernel<X, Z, P, SUMS>), dim3((unsigned)(blocks * p.groups * p.parts)), dim3(256), 0, stream, p, (int)blocks, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // 16 columns to a workgroup where there would be fewer than 32 of 64 columns (us, 64 / 16 columns: 256 parts of 4 sums of 706 columns 18.6 / 6.0, of 2 sums of 4096 5.1 / 9.8; six times 42 parts of 4 sums of 5001 8.5 / 35.8)
    if ((p.D + 63) / 64 * p.groups < 32)
        hipLaunchKernelGGL((residual_params_kernel<P, SUMS, 16>), dim3((unsigned)((p.D + 15) / 16), (unsigned)p.groups), dim3(1024), 0, stream, p, totals);
    else
        hipLaunchKernelGGL((residual_params_kernel<P, SUMS, 64>), dim3((unsigned)((p.D + 63) / 64), (unsigned)p.groups), dim3(1024), 0, stream, p, totals);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !totals) return e;
    hipLaunchKernelGGL((residual_groups_kernel<P, SUMS>), dim3((unsigned)((p.D + 63) / 64), SUMS), dim3(1024), 0, stream, p, totals);
    return hipGetLastError();
}

template <class X, class Z, class P>
hipError_t forward(const ResidualParams &p, hipStream_t stream)
{
    if (p.D > 4 * kResidualThreads * E || p.D < E) {
        hipLaunchKernelGGL((residual_long_kernel<X, Z, P>), dim3((unsigned)std::min(p.M, kMostWorkgroups)), dim3(kResidualThreads), 0, stream, p);
        return hipGetLastError();
    }
    switch (residual_threads(p.D)) {
        case 64: return forward_of<X, Z, P, 64, 1>(p, stream);
        case 128: return forward_of<X, Z, P, 128, 1>(p, stream);
        case 256: return forward_of<X, Z, P, 256, 1>(p, stream);
        default:
            if (p.D <= 512 * E) return forward_of<X, Z, P, 512, 1>(p, stream);
            return p.D <= 1024 * E ? forward_of<X, Z, P, 512, 2>(p, stream) : forward_of<X, Z, P, 512, 4>(p, stream);
    }
}

template <class X, class Z, class P>
hipError_t backward(const ResidualParams &p, hipStream_t stream)
{
    const bool asked = p.dgate || p.dpost_weight || p.dpost_bias || p.dpre_weight || p.dpre_bias, is_long = residual_is_long(p.D);
    const int sums = !asked ? 0 : p.dpost_bias || p.dpre_bias || (p.dgate && p.post.kind != ATB_NORM_NONE && p.post.bias) ? 4 : 2;
    const ResidualRoom room = residual_room(p.M, p.D, p.groups);
    float *totals = asked && p.groups > 1 ? p.workspace + room.sums : nullptr, *rows = asked && is_long ? p.workspace + room.sums + room.totals : nullptr;
    if (p.M > 0 && (asked || p.dx || p.dz)) {
        hipError_t e = hipSuccess;
        if (is_long) {
            bool held = false;
            if constexpr (sizeof(X) == 2) {
                held = residual_is_wide(p.D);
                if (held) e = p.D <= 3 * kResidualThreads * E ? backward_of<X, Z, P, 512, 3, 0>(p, stream, rows) : backward_of<X, Z, P, 512, 4, 0>(p, stream, rows);
            }
            if (!held) {
                hipLaunchKernelGGL((residual_grad_long_kernel<X, Z, P>), dim3((unsigned)std::min(p.M, kMostWorkgroups)), dim3(kResidualThreads), 0, stream, p, rows);
                e = hipGetLastError();
            }
        } else {
            e = sums == 0 ? backward_rows<X, Z, P, 0>(p, stream) : sums == 2 ? backward_rows<X, Z, P, 2>(p, stream) : backward_rows<X, Z, P, 4>(p, stream);
        }
        if (e != hipSuccess) return e;
    }
    if (!asked) return hipSuccess;
    return sums == 2 ? sums_of<X, Z, P, 2>(p, rows, totals, stream) : sums_of<X, Z, P, 4>(p, rows, totals, stream);
}

// f, called with the types of p as template arguments
template <class F>
hipError_t with_types(const ResidualParams &p, F f)
{
    const bool wide = p.w_type == ATB_TYPE_F32;
    if (p.x_type == ATB_TYPE_BF16) return wide ? f(__bf16(), __bf16(), float()) : f(__bf16(), __bf16(), __bf16());
    if (p.z_type == ATB_TYPE_BF16) return wide ? f(float(), __bf16(), float()) : f(float(), __bf16(), __bf16());
    return wide ? f(float(), float(), float()) : f(float(), float(), __bf16());
}

}  // namespace

hipError_t launch_residual(const ResidualParams &p, hipStream_t stream)
{
    return with_types(p, [&](auto x, auto z, auto w) { return forward<decltype(x), decltype(z), decltype(w)>(p, stream); });
}

hipError_t launch_residual_backward(const ResidualParams &p, hipStream_t stream)
{
    ResidualParams q = p;
    q.parts = (int)residual_room(p.M, p.D, p.groups).parts;
    return with_types(q, [&](auto x, auto z, auto w) { return backward<decltype(x), decltype(z), decltype(w)>(q, stream); });
}

}  // namespace atb
