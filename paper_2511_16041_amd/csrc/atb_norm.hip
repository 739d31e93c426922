// Layer norm for gfx950, forward and backward.  Bound: HBM; a small call is its launch.
//
// mu = sum(x) / D, r = 1 / sqrt(sum((x - mu)^2) / D + eps), y = (x - mu) r w + b.  A row is held in registers, 16 elements per thread, so it is read
// once and the variance is the sum of squares about the mean itself (no E[x^2] - mu^2, which loses the digits of a row far off centre).
// Backward, with xh = (x - mu) r and g = dy w: dx = r (g - mean(g) - xh mean(g xh)); dw = sum over rows of dy xh, db = sum of dy: every
// workgroup walks rows a grid apart and keeps its share of both sums in registers, 16 columns per thread; a second kernel adds the
// workgroups' sums in order.  No atomics: the same bits every time.
// Rows begin anywhere: 16-byte requests at any element, and the elements of the last, incomplete chunk one by one.
// Measured (a copy reaches 4.9 TB/s here; inputs of this size come partly out of the memory-side cache): 8192 x 4096 in bf16 forward 29.0 us, 4.6 TB/s, backward
// 33.9 us, 5.9 TB/s, and the sums of dw and db 4.7 us; 3000 x 5001 in fp32 forward 26.4 us, 4.5 TB/s, backward 44.1 us; 1 x 4096 in bf16 3.1 us.  In bf16, forward and
// dx + the share of dw and db + their sum: 4096 x 8200 41 us and 57 + 28 + 5 (half of the 1024 threads have nothing to do, and x and dy are read twice), 2048 x 16384 31 and
// 44 + 27 + 5, 2048 x 16400 90 and 111 + 29 + 5 (a lane takes single elements).
#include "atb_device.h"
#include "atb_layers.h"

namespace atb {
namespace {

constexpr int kPerThread = kNormPerThread, kGradThreads = kNormGradThreads, kMaxGradRow = kNormMaxGradRow;
constexpr int kMaxRow = 1024 * kPerThread;     // longer rows are read again for every sum

template <class T> struct Chunk;               // 16 bytes of a row
template <> struct Chunk<__bf16> {
    static constexpr int E = 8;
    typedef bf16x8 vec;
    typedef bf16x8 any __attribute__((aligned(2)));
};
template <> struct Chunk<float> {
    static constexpr int E = 4;
    typedef floatx4 vec;
    typedef floatx4 any __attribute__((aligned(4)));
};

// A chunk of a row of D from element `at` on, as it is; 0 past the end.
template <class T>
ATB_DEV typename Chunk<T>::vec load_chunk(const T *row, int at, int D)
{
    constexpr int E = Chunk<T>::E;
    typename Chunk<T>::vec w = {};
    if (at + E <= D) {
        w = *reinterpret_cast<const typename Chunk<T>::any *>(row + at);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at + e < D) w[e] = row[at + e];
    }
    return w;
}

// Elements at .. at + E - 1 of a row of D; `other` past its end.
template <class T, int E>
ATB_DEV void load(const T *row, int at, int D, float (&v)[E], float other)
{
    constexpr int C = Chunk<T>::E;
    if (at + E <= D) {
#pragma unroll
        for (int c = 0; c < E; c += C) {
            const typename Chunk<T>::vec w = *reinterpret_cast<const typename Chunk<T>::any *>(row + at + c);
#pragma unroll
            for (int e = 0; e < (C < E ? C : E); ++e) v[c + e] = (float)w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at + e < D ? (float)row[at + e] : other;
    }
}
// (half a chunk: parameters in bf16 of rows in fp32)
template <>
ATB_DEV void load<__bf16, 4>(const __bf16 *row, int at, int D, float (&v)[4], float other)
{
    if (at + 4 <= D) {
        const bf16x4 w = *reinterpret_cast<const bf16x4_u *>(row + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)w[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = at + e < D ? (float)row[at + e] : other;
    }
}

template <class T, int E>
ATB_DEV void store(T *row, int at, int D, const float (&v)[E])
{
    static_assert(E == Chunk<T>::E, "one chunk");
    if (at + E <= D) {
        typename Chunk<T>::vec w;
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = (T)v[e];
        *reinterpret_cast<typename Chunk<T>::any *>(row + at) = w;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at + e < D) row[at + e] = (T)v[e];
    }
}

// The parameters of a thread's C chunks of E, 0 past the end.
template <class P, int T, int C, int E>
ATB_DEV void load_params(const P *w, int t, int D, P (&v)[C][E])
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float f[E];
        load<P, E>(w, (c * T + t) * E, D, f, 0.0f);
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] = (P)f[e];
    }
}

ATB_DEV float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Sums over the T threads of a row group.  `scratch`: one float per wave of the workgroup and sum; every thread of the workgroup calls it.
template <int T, int N>
ATB_DEV void row_sums(float (&v)[N], float *scratch)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (T > 64) {
        constexpr int W = T / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[wave * N + i] = v[i];
        __syncthreads();
        const float *mine = scratch + (wave / W) * W * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) s += mine[w * N + i];
            v[i] = s;
        }
    }
}

// Whether workgroups walk rows a grid apart, so that weight and bias are read once (for every row they were twice its own bytes, out of a cache) and the next row is
// on its way while this one is summed: bf16 rows of 256 or 512 threads (walking / not, us, tensors in turn that stay in part in the cache: 8192 x 4096 25.4 / 27.9, 4096 x 8192 27.3 / 28.9).  Shorter rows and the
// longest ones are faster with one row per group and more waves (8192 x 64 9.1 / 7.2, 8192 x 2048 15.2 / 14.2, 4096 x 8200 48.3 / 44.3), and so is fp32, with
// twice the registers for the same elements (3000 x 5001 31.4 / 26.9).
template <class X, int T>
constexpr bool walks() { return sizeof(X) == 2 && T >= 256 && T < 1024; }

// T threads per row, NT / T rows of a workgroup at a time.
template <class X, class P, int T>
__global__ void __launch_bounds__(T < 256 ? 256 : T) norm_kernel(const NormParams p, int rounds)
{
    constexpr int E = Chunk<X>::E, C = kPerThread / E, NT = T < 256 ? 256 : T, R = NT / T;
    constexpr bool WALKS = walks<X, T>();
    typedef typename Chunk<X>::vec Vec;
    __shared__ float scratch[2][NT / 64];
    const int t = threadIdx.x % T, group = threadIdx.x / T, D = (int)p.D;
    const X *x0 = static_cast<const X *>(p.x);
    Vec next[C];
    auto fetch = [&](int64_t row) {
        const X *x = x0 + (row < p.M ? row : 0) * p.ldx;
#pragma unroll
        for (int c = 0; c < C; ++c) next[c] = load_chunk<X>(x, (c * T + t) * E, D);
    };
    fetch((int64_t)blockIdx.x * R + group);
    P w[WALKS ? C : 1][E], b[WALKS ? C : 1][E];
#pragma unroll
    for (int c = 0; c < (WALKS ? C : 1); ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) { w[c][e] = (P)1.0f; b[c][e] = (P)0.0f; }
    if constexpr (WALKS) {
        if (p.weight) load_params<P, T, C, E>(static_cast<const P *>(p.weight), t, D, w);
        if (p.bias) load_params<P, T, C, E>(static_cast<const P *>(p.bias), t, D, b);
    }
    for (int n = 0; n < (WALKS ? rounds : 1); ++n) {                        // the same number for every thread of the workgroup
        const int64_t row = ((int64_t)n * gridDim.x + blockIdx.x) * R + group;
        float v[C][E], sum[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[c][e] = (float)next[c][e];                  // 0 past the end
                sum[0] += v[c][e];
            }
        if (WALKS && n + 1 < rounds) fetch(row + (int64_t)gridDim.x * R);
        row_sums<T, 1>(sum, scratch[0]);
        const float mean = sum[0] / (float)D;
        sum[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[c][e] -= mean;
                if ((c * T + t) * E + e < D) sum[0] += v[c][e] * v[c][e];
            }
        row_sums<T, 1>(sum, scratch[1]);
        const float rstd = 1.0f / sqrtf(sum[0] / (float)D + p.eps);
        if (row >= p.M) continue;                             // (only in the last round)
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        X *y = static_cast<X *>(p.y) + row * p.ldy;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * T + t) * E;
            if (at >= D) break;
            float wf[E], bf[E];
#pragma unroll
            for (int e = 0; e < E; ++e) { wf[e] = (float)w[WALKS ? c : 0][e]; bf[e] = (float)b[WALKS ? c : 0][e]; }
            if constexpr (!WALKS) {
                if (p.weight) load<P, E>(static_cast<const P *>(p.weight), at, D, wf, 0.0f);
                if (p.bias) load<P, E>(static_cast<const P *>(p.bias), at, D, bf, 0.0f);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) v[c][e] = v[c][e] * rstd * wf[e] + bf[e];
            store<X, E>(y, at, D, v[c]);
        }
    }
}

// This thread's share of sums over a row of any length, 1024 threads: f(i, sums) adds element i.  Taken 128 elements at a time, so that a chain has 128 + D / 2^17
// additions and not D / 1024: where rounding errors have one sign (rows and gradients of few values) 16384 of them made a sum wrong by 1.6e-4 of its size.
template <int N, class F>
ATB_DEV void add_long(int D, float (&sums)[N], F f)
{
    constexpr int RUN = 128 * 1024;
#pragma unroll
    for (int n = 0; n < N; ++n) sums[n] = 0.0f;
    for (int from = 0; from < D; from += RUN) {                          // D <= 2^24
        float run[N] = {};
        const int end = min(D, from + RUN);
        for (int i = from + threadIdx.x; i < end; i += 1024) f(i, run);
#pragma unroll
        for (int n = 0; n < N; ++n) sums[n] += run[n];
    }
}

// Rows of any length: read three times (from the second time on out of a cache).
template <class X, class P>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormParams p)
{
    __shared__ float scratch[2][16];
    const int64_t row = blockIdx.x;
    const int D = (int)p.D;
    const X *x = static_cast<const X *>(p.x) + row * p.ldx;
    float sum[1];
    add_long(D, sum, [&](int i, float (&s)[1]) { s[0] += (float)x[i]; });
    row_sums<1024, 1>(sum, scratch[0]);
    const float mean = sum[0] / (float)D;
    add_long(D, sum, [&](int i, float (&s)[1]) {
        const float d = (float)x[i] - mean;
        s[0] += d * d;
    });
    row_sums<1024, 1>(sum, scratch[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / (float)D + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
    X *y = static_cast<X *>(p.y) + row * p.ldy;
    const P *w = static_cast<const P *>(p.weight), *b = static_cast<const P *>(p.bias);
    for (int i = threadIdx.x; i < D; i += 1024)
        y[i] = (X)(((float)x[i] - mean) * rstd * (w ? (float)w[i] : 1.0f) + (b ? (float)b[i] : 0.0f));
}

// Four consecutive of a thread's sums
template <int C, int E>
ATB_DEV floatx4 quarter(const float (&v)[C][E], int q)
{
    return floatx4{v[q * 4 / E][q * 4 % E], v[q * 4 / E][q * 4 % E + 1], v[q * 4 / E][q * 4 % E + 2], v[q * 4 / E][q * 4 % E + 3]};
}

// dx, and (PARAMS) the workgroup's part of dw and db: partial[workgroup][2][D].
template <class X, class P, int T, bool PARAMS>
__global__ void __launch_bounds__(T > kGradThreads ? T : kGradThreads) norm_grad_kernel(const NormParams p, int rounds)
{
    constexpr int E = Chunk<X>::E, C = kPerThread / E, NT = T > kGradThreads ? T : kGradThreads, R = NT / T;
    __shared__ float scratch[2][2 * NT / 64];
    const int t = threadIdx.x % T, group = threadIdx.x / T, D = (int)p.D;
    const X *x0 = static_cast<const X *>(p.x), *dy0 = static_cast<const X *>(p.dy);
    float dw[C][E], db[C][E], w[C][E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int e = 0; e < E; ++e) { dw[c][e] = db[c][e] = 0.0f; w[c][e] = 1.0f; }
        if (p.weight) load<P, E>(static_cast<const P *>(p.weight), (c * T + t) * E, D, w[c], 0.0f);
    }
    // the next row is on its way while this one is summed (8192 x 4096 in 64.4 us without, 38.2 with, as the rest was then)
    typedef typename Chunk<X>::vec Vec;
    Vec next_x[C], next_dy[C];
    float next_mean = 0.0f, next_rstd = 0.0f;
    constexpr bool AHEAD = T <= kGradThreads;                 // (of the longest rows 1024 threads have no registers for it)
    auto fetch = [&](int64_t row) {
        const int64_t at_row = row < p.M ? row : 0;
        next_mean = p.mean[at_row];
        next_rstd = p.rstd[at_row];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            next_x[c] = load_chunk<X>(x0 + at_row * p.ldx, (c * T + t) * E, D);
            next_dy[c] = load_chunk<X>(dy0 + at_row * p.lddy, (c * T + t) * E, D);
        }
    };
    if (AHEAD) fetch((int64_t)blockIdx.x * R + group);
    for (int n = 0; n < rounds; ++n) {                        // the same number for every thread of the workgroup
        const int64_t row = ((int64_t)n * gridDim.x + blockIdx.x) * R + group;
        const bool live = row < p.M;
        if (!AHEAD) fetch(row);
        const float mean = next_mean, rstd = next_rstd;
        Vec vx[C], vdy[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            vx[c] = next_x[c];
            vdy[c] = next_dy[c];
        }
        if (AHEAD && n + 1 < rounds) fetch(row + (int64_t)gridDim.x * R);
        float xh[C][E], g[C][E], s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                xh[c][e] = ((float)vx[c][e] - mean) * rstd;               // (past the end g is 0)
                g[c][e] = (float)vdy[c][e];
                if constexpr (PARAMS) {
                    if (live) {
                        dw[c][e] += g[c][e] * xh[c][e];
                        db[c][e] += g[c][e];
                    }
                }
                g[c][e] *= w[c][e];
                s[0] += g[c][e];
                s[1] += g[c][e] * xh[c][e];
            }
        }
        row_sums<T, 2>(s, scratch[n & 1]);
        if (live && p.dx) {
            const float m0 = s[0] / (float)D, m1 = s[1] / (float)D;
            X *dx = static_cast<X *>(p.dx) + row * p.lddx;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = (c * T + t) * E;
#pragma unroll
                for (int e = 0; e < E; ++e) g[c][e] = rstd * (g[c][e] - m0 - xh[c][e] * m1);
                if (at < D) store<X, E>(dx, at, D, g[c]);
            }
        }
    }
    if constexpr (PARAMS) {
        // the row groups' sums, the upper half of the groups onto the lower one in every step
        extern __shared__ float sums[];                       // [R / 2][2][16 T]
        constexpr int ROOM = 2 * kPerThread * T;
#pragma unroll
        for (int half = R / 2; half >= 1; half /= 2) {
            __syncthreads();
            if (group >= half && group < 2 * half) {
                float *to = sums + (group - half) * ROOM + t * 4;
#pragma unroll
                for (int c = 0; c < kPerThread / 4; ++c) {
                    *reinterpret_cast<floatx4 *>(to + c * T * 4) = quarter(dw, c);
                    *reinterpret_cast<floatx4 *>(to + ROOM / 2 + c * T * 4) = quarter(db, c);
                }
            }
            __syncthreads();
            if (group < half) {
                const float *from = sums + group * ROOM + t * 4;
#pragma unroll
                for (int c = 0; c < kPerThread / 4; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        dw[c * 4 / E][c * 4 % E + e] += from[c * T * 4 + e];
                        db[c * 4 / E][c * 4 % E + e] += from[ROOM / 2 + c * T * 4 + e];
                    }
            }
        }
        if (group > 0) return;
        float *out = p.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
        for (int c = 0; c < kPerThread / 4; ++c) {
            const int at = (c * 4 / E * T + t) * E + c * 4 % E;
            const floatx4 a = quarter(dw, c), b = quarter(db, c);
            const float fa[4] = {a[0], a[1], a[2], a[3]}, fb[4] = {b[0], b[1], b[2], b[3]};
            if (at < D) {
                store<float, 4>(out, at, D, fa);
                store<float, 4>(out + D, at, D, fb);
            }
        }
    }
}

// Rows of any length.
template <class X, class P>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const NormParams p)
{
    __shared__ float scratch[2 * 16];
    const int64_t row = blockIdx.x;
    const int D = (int)p.D;
    const X *x = static_cast<const X *>(p.x) + row * p.ldx, *dy = static_cast<const X *>(p.dy) + row * p.lddy;
    const P *w = static_cast<const P *>(p.weight);
    const float mean = p.mean[row], rstd = p.rstd[row];
    float s[2];
    add_long(D, s, [&](int i, float (&sum)[2]) {
        const float g = (float)dy[i] * (w ? (float)w[i] : 1.0f);
        sum[0] += g;
        sum[1] += g * (((float)x[i] - mean) * rstd);
    });
    row_sums<1024, 2>(s, scratch);
    const float m0 = s[0] / (float)D, m1 = s[1] / (float)D;
    X *dx = static_cast<X *>(p.dx) + row * p.lddx;
    for (int i = threadIdx.x; i < D; i += 1024) {
        const float g = (float)dy[i] * (w ? (float)w[i] : 1.0f), xh = ((float)x[i] - mean) * rstd;
        dx[i] = (X)(rstd * (g - m0 - xh * m1));
    }
}
// ... their dw and db: a thread has a chunk of columns of the rows blockIdx.y, blockIdx.y + gridDim.y, ..
template <class X>
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormParams p)
{
    constexpr int E = Chunk<X>::E;
    const int D = (int)p.D, col = (blockIdx.x * 256 + threadIdx.x) * E;
    if (col >= D) return;
    const X *x = static_cast<const X *>(p.x), *dy = static_cast<const X *>(p.dy);
    float dw[E] = {}, db[E] = {};
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < p.M; row += gridDim.y) {
        const typename Chunk<X>::vec g = load_chunk<X>(dy + row * p.lddy, col, D), v = load_chunk<X>(x + row * p.ldx, col, D);
        const float mean = p.mean[row], rstd = p.rstd[row];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            dw[e] += (float)g[e] * (((float)v[e] - mean) * rstd);
            db[e] += (float)g[e];
        }
    }
    float *out = p.partial + (int64_t)blockIdx.y * 2 * D + col;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (col + e < D) {
            out[e] = dw[e];
            out[D + e] = db[e];
        }
}

// dw, db = the partial sums added in order: 64 columns per workgroup, 16 waves with a run of the partial sums each.
template <class P>
__global__ void __launch_bounds__(1024) norm_params_kernel(const NormParams p, int partials)
{
    __shared__ float sums[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    const int which = blockIdx.y;                             // 0: dw, 1: db
    P *out = static_cast<P *>(which ? p.dbias : p.dweight);
    if (!out) return;                                         // the whole workgroup
    const int run = (partials + 15) / 16, first = wave * run, end = min(first + run, partials);
    float s = 0.0f;
    if (col < p.D) {
        const float *at = p.partial + ((int64_t)first * 2 + which) * p.D + col;
        for (int i = first; i < end; i += 64) {               // 64 at a time: shorter chains
            const int stop = min(end, i + 64);
            float part = 0.0f;
#pragma unroll 8
            for (int n = i; n < stop; ++n, at += 2 * p.D) part += *at;
            s += part;
        }
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < p.D) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += sums[i][lane];
        out[col] = (P)s;
    }
}

// Rows of a launch with a workgroup a row: of up to 1024 threads, and a launch has fewer than 2^32.
constexpr int64_t kMostRows = (int64_t)1 << 21;

// f, called with the rows of p, kMostRows of them at a time
template <class F>
hipError_t by_rows(const NormParams &p, F f)
{
    const int64_t size = p.x_type == ATB_TYPE_F32 ? 4 : 2;
    for (int64_t row = 0; row < p.M; row += kMostRows) {
        NormParams part = p;
        part.M = p.M - row < kMostRows ? p.M - row : kMostRows;
        if (p.x) part.x = static_cast<const char *>(p.x) + row * p.ldx * size;
        if (p.dy) part.dy = static_cast<const char *>(p.dy) + row * p.lddy * size;
        if (p.y) part.y = static_cast<char *>(p.y) + row * p.ldy * size;
        if (p.dx) part.dx = static_cast<char *>(p.dx) + row * p.lddx * size;
        if (p.mean) part.mean = p.mean + row;
        if (p.rstd) part.rstd = p.rstd + row;
        const hipError_t e = f(part);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class X, class P, int T>
hipError_t forward_of(const NormParams &p, hipStream_t stream)
{
    constexpr int NT = T < 256 ? 256 : T, R = NT / T, MOST = 256 * (1024 / NT);        // 16 waves per CU
    const int64_t all = (p.M + R - 1) / R, grid = !walks<X, T>() || all < MOST ? all : MOST;
    hipLaunchKernelGGL((norm_kernel<X, P, T>), dim3((unsigned)grid), dim3(NT), 0, stream, p, (int)((all + grid - 1) / grid));
    return hipGetLastError();
}

template <class X, class P>
hipError_t forward(const NormParams &p, hipStream_t stream)
{
    if (p.D > kMaxRow) {
        hipLaunchKernelGGL((norm_long_kernel<X, P>), dim3((unsigned)p.M), dim3(1024), 0, stream, p);
        return hipGetLastError();
    }
    switch (norm_threads(p.D)) {
        case 64: return forward_of<X, P, 64>(p, stream);
        case 128: return forward_of<X, P, 128>(p, stream);
        case 256: return forward_of<X, P, 256>(p, stream);
        case 512: return forward_of<X, P, 512>(p, stream);
        default: return forward_of<X, P, 1024>(p, stream);
    }
}

// T threads per row: dx, and with PARAMS the partial sums of dw and db as well.
template <class X, class P, int T, bool PARAMS>
hipError_t backward_of(const NormParams &p, int64_t grid, hipStream_t stream)
{
    constexpr int NT = T > kGradThreads ? T : kGradThreads, R = NT / T;
    const int rounds = (int)((p.M + grid * R - 1) / (grid * R));
    const size_t lds = PARAMS && R > 1 ? (size_t)(R / 2) * 2 * kPerThread * T * sizeof(float) : 0;       // 32 KiB
    hipLaunchKernelGGL((norm_grad_kernel<X, P, T, PARAMS>), dim3((unsigned)grid), dim3(NT), lds, stream, p, rounds);
    return hipGetLastError();
}

template <class X, class P, int T>
hipError_t backward_short(const NormParams &p, hipStream_t stream)
{
    if (p.dweight || p.dbias) return backward_of<X, P, T, true>(p, norm_partials(p.M, p.D), stream);
    const int64_t rows = kGradThreads / T, grid = (p.M + rows - 1) / rows;
    return backward_of<X, P, T, false>(p, grid < 2048 ? grid : 2048, stream);
}

// Rows of more than kMaxGradRow elements: with both sums beside the row a thread would need more registers than it has (16 elements in each of
// 1024 threads: 38 spilled), so dw and db are a pass of their own over x and dy.  (Both sums in LDS, up to 128 KiB of it, have not been tried.)
template <class X, class P>
hipError_t backward_long(const NormParams &p, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (p.dx && p.D <= kMaxRow) {
        e = backward_of<X, P, 1024, false>(p, p.M < 2048 ? p.M : 2048, stream);
    } else if (p.dx) {
        e = by_rows(p, [&](const NormParams &part) {
            hipLaunchKernelGGL((norm_grad_long_kernel<X, P>), dim3((unsigned)part.M), dim3(1024), 0, stream, part);
            return hipGetLastError();
        });
    }
    if (e != hipSuccess || !(p.dweight || p.dbias)) return e;
    hipLaunchKernelGGL((norm_columns_kernel<X>), dim3((unsigned)((p.D + 256 * Chunk<X>::E - 1) / (256 * Chunk<X>::E)), (unsigned)norm_partials(p.M, p.D)), dim3(256), 0,
                       stream, p);
    return hipGetLastError();
}

template <class X, class P>
hipError_t backward(const NormParams &p, hipStream_t stream)
{
    const bool params = p.dweight || p.dbias;
    hipError_t e = hipSuccess;
    if (p.M > 0 && (p.dx || params)) {
        if (p.D > kMaxGradRow) e = backward_long<X, P>(p, stream);
        else switch (norm_threads(p.D)) {
            case 64: e = backward_short<X, P, 64>(p, stream); break;
            case 128: e = backward_short<X, P, 128>(p, stream); break;
            case 256: e = backward_short<X, P, 256>(p, stream); break;
            default: e = backward_short<X, P, 512>(p, stream); break;
        }
    }
    if (e != hipSuccess || !params) return e;
    hipLaunchKernelGGL((norm_params_kernel<P>), dim3((unsigned)((p.D + 63) / 64), 2), dim3(1024), 0, stream, p, (int)norm_partials(p.M, p.D));      // no rows: zeros
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormParams &p, hipStream_t stream)
{
    return by_rows(p, [&](const NormParams &part) {
        if (part.x_type == ATB_TYPE_F32) return part.w_type == ATB_TYPE_F32 ? forward<float, float>(part, stream) : forward<float, __bf16>(part, stream);
        return part.w_type == ATB_TYPE_F32 ? forward<__bf16, float>(part, stream) : forward<__bf16, __bf16>(part, stream);
    });
}

hipError_t launch_norm_backward(const NormParams &p, hipStream_t stream)
{
    if (p.x_type == ATB_TYPE_F32) return p.w_type == ATB_TYPE_F32 ? backward<float, float>(p, stream) : backward<float, __bf16>(p, stream);
    return p.w_type == ATB_TYPE_F32 ? backward<__bf16, float>(p, stream) : backward<__bf16, __bf16>(p, stream);
}

}  // namespace atb
