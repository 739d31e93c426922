// A product with its epilogue, y = act(x W^T + b) + residual, and what its gradients need beside products: dz = dy o act'(z) with its column sums, the bias's gradient.
// The product and dx = dz W, dW = dz^T x are tiles (atb_tiles.h), of few rows without a backward pass atb_stream.hip.
//
// For the backward pass act'(z) is kept in fp16: it lies in -0.17 .. 1.13, and 2 bytes are what z in bf16 would take, with eight times the error.  Down to 2^-14, fp16's smallest normal number, it errs by at most 2^-11
// of itself, an eighth of the rounding of dz that follows (dz is an operand of two products, whose matrix instructions take bf16); below by at most 2^-25 absolutely, so that where an activation is flat the slope loses
// digits and then vanishes: SiLU's is 0.2 % off at z = -14, 8 % at -18, 52 % at -20, GELU's 68 % at -6.  What dz loses there is at most 2^-25 |dy|.
// The column sums take dz before it is rounded, in fp32, in runs of rows that are added in order: the same bits every time.
// Bound: as the tiles; dz and its sums HBM.
// Measured: forward M = 2048, K = 4096, N = 14336 214 us, 1126 TFLOP/s (448 tiles, 1.75 rounds of the CUs), MFMAs busy 49 %; M = 8192 with the slope kept 830 to 875 us, 1100 to 1160, 57 %: a tile's end, which
// computes tanh and its derivative and writes 4 bytes an element, is not overlapped with products.  dz 161 us, 4.4 TB/s, the bias's gradient 5.  M = 1500, K = 2056, N = 5001: forward 51 to 57 (240 tiles of
// 128 x 256, one per CU), dz 14, bias 5.4.
#include "atb_block.h"
#include "atb_tiles.h"

namespace atb {

hipError_t launch_tiles_linear(TileParams p, int epilogue, hipStream_t stream)
{
    if (epilogue == kLinearKeep) return launch_tiles<false, false, kLinearKeep>(p, stream);
    return launch_tiles<false, false, kLinear>(p, stream);
}

namespace {

template <class T>
struct Eight {
    typedef T vec __attribute__((ext_vector_type(8)));
    typedef vec any __attribute__((aligned(2)));
};

// Eight columns per thread, a run of rows per workgroup.  Bound: HBM.  The last chunk of a row is moved back to end with it: all are loaded whole, without a branch, at which a wave would wait for its loads (6 x 1654
// took 12.3 us with one); its elements before `first` are another thread's.  (Rows of fewer than eight elements: one by one.)
template <bool SLOPE>
__global__ void __launch_bounds__(256) linear_grad_kernel(const LinearGradParams p, int parts)
{
    const int pitch = (p.N + 7) / 8 * 8, col = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= pitch) return;
    const bool narrow = p.N < 8;
    const int at = narrow ? 0 : min(col, p.N - 8), first = col - at;
    const int64_t from = p.M * blockIdx.y / parts, end = p.M * (blockIdx.y + 1) / parts;
    const __bf16 *dy = reinterpret_cast<const __bf16 *>(p.dy) + at;
    const _Float16 *slope = reinterpret_cast<const _Float16 *>(p.slope) + at;
    float sum[8] = {};
    auto add = [&](int64_t row, const float (&d)[8], int left) {              // of d, the elements first .. left - 1
        if (p.dz) {
            if (first == 0 && left == 8) {
                bf16x8 w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (__bf16)d[e];
                *reinterpret_cast<bf16x8 *>(p.dz + row * pitch + col) = w;
            } else {
                __bf16 *to = reinterpret_cast<__bf16 *>(p.dz) + row * pitch;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e >= first && e < left) to[at + e] = (__bf16)d[e];
                    if (col + e >= p.N) to[col + e] = (__bf16)0.0f;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += d[e];
    };
    if (narrow) {
        for (int64_t row = from; row < end; ++row) {
            float d[8] = {};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < p.N) d[e] = (float)dy[row * p.lddy + e] * (SLOPE ? (float)slope[row * pitch + e] : 1.0f);
            add(row, d, p.N);
        }
    } else {
#pragma unroll 4
        for (int64_t row = from; row < end; ++row) {
            const bf16x8 g = *reinterpret_cast<const Eight<__bf16>::any *>(dy + row * p.lddy);
            float d[8];
            if constexpr (SLOPE) {
                const Eight<_Float16>::vec s = *reinterpret_cast<const Eight<_Float16>::any *>(slope + row * pitch);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = (float)g[e] * (float)s[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = (float)g[e];
            }
            add(row, d, 8);
        }
    }
    if (!p.dbias) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e < first || at + e >= p.N) continue;
        if (parts > 1) p.partial[(int64_t)blockIdx.y * p.N + at + e] = sum[e];
        else if (p.bias_type == ATB_TYPE_F32) static_cast<float *>(p.dbias)[at + e] = sum[e];
        else static_cast<__bf16 *>(p.dbias)[at + e] = (__bf16)sum[e];
    }
}

// The runs' column sums added in order: 64 columns per workgroup, 16 waves with some of the runs each, 64 at a time (shorter chains).
__global__ void __launch_bounds__(1024) linear_bias_kernel(const LinearGradParams p, int parts)
{
    __shared__ float sums[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane;
    const int run = (parts + 15) / 16, first = wave * run, end = min(first + run, parts);
    float s = 0.0f;
    if (col < p.N) {
        const float *at = p.partial + (int64_t)first * p.N + col;
        for (int i = first; i < end; i += 64) {
            const int stop = min(end, i + 64);
            float part = 0.0f;
#pragma unroll 8
            for (int n = i; n < stop; ++n, at += p.N) part += *at;
            s += part;
        }
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < p.N) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += sums[i][lane];
        if (p.bias_type == ATB_TYPE_F32) static_cast<float *>(p.dbias)[col] = s;
        else static_cast<__bf16 *>(p.dbias)[col] = (__bf16)s;
    }
}

}  // namespace

hipError_t launch_linear_grad(const LinearGradParams &p, hipStream_t stream)
{
    const int parts = (int)linear_parts(p.M, p.N);                 // at most 2^14
    if (p.M > 0 && (p.dz || p.dbias)) {
        const dim3 grid((unsigned)((p.N + 2047) / 2048), (unsigned)parts);
        if (p.slope) hipLaunchKernelGGL(linear_grad_kernel<true>, grid, dim3(256), 0, stream, p, parts);
        else hipLaunchKernelGGL(linear_grad_kernel<false>, grid, dim3(256), 0, stream, p, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!p.dbias || parts == 1) return hipSuccess;
    hipLaunchKernelGGL(linear_bias_kernel, dim3((unsigned)((p.N + 63) / 64)), dim3(1024), 0, stream, p, parts);      // no rows: zeros
    return hipGetLastError();
}

}  // namespace atb
