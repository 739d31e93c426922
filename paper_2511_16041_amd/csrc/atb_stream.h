// What the kernels for few rows share (atb_stream.hip: weights in bf16, atb_q4_stream.hip: in 4 bits).
//
// v_mfma_f32_16x16x32_bf16 with x as the first operand: lane l supplies row l % 16 of x and column l % 16 of W^T at 8 k values of group
// l / 16, and holds column l % 16 and rows 4 (l / 16) .. + 3 of the result, so that a column's scale is one value per lane.
#pragma once

#include "atb_activation.h"
#include "atb_layers.h"

namespace atb {

constexpr int kOutside = (int)0x80000000;        // an offset past the end of every descriptor: reads as zero

ATB_DEV floatx4 mfma_rows(const intx4 &x, const intx4 &w, const floatx4 &acc)
{
#if defined(__HIP_DEVICE_COMPILE__)
    union { intx4 i; bf16x8 b; } a, b;
    a.i = x;
    b.i = w;
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, acc, 0, 0, 0);
#else
    return acc;
#endif
}

// LDS by address
template <class T>
ATB_DEV T lds_read(unsigned at)
{
    T r = {};
#if defined(__HIP_DEVICE_COMPILE__)
    r = *(const __attribute__((address_space(3))) T *)at;
#endif
    return r;
}
template <class T>
ATB_DEV void lds_write(unsigned at, T v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    *(__attribute__((address_space(3))) T *)at = v;
#endif
}

// The partial sums of a workgroup's W waves, added in wave order, and the workgroup's part of y: 16 MB rows from m0, 16 COLS columns from n0 on, of which `cols` are
// inside.  GATED: the second half of the NB blocks are the up product.  lds: W MB NB KiB, free on entry.
template <int MB, int NB, int W, bool GATED>
ATB_DEV void finish_rows(const StreamParams &p, const floatx4 (&acc)[MB][NB], float *lds, int m0, int n0, int cols)
{
    constexpr int COLS = GATED ? NB / 2 : NB, PER_WAVE = MB * NB * 256;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) lds[wave * PER_WAVE + ((i * NB + j) * 4 + e) * 64 + lane] = acc[i][j][e];
    __syncthreads();
    // thread -> row, column with neighbouring threads in neighbouring columns
    for (int o = threadIdx.x; o < MB * 16 * COLS * 16; o += W * 64) {
        const int col = o % (COLS * 16), row = o / (COLS * 16);
        const int i = row / 16, j = col / 16, at = ((i * NB + j) * 4 + row % 4) * 64 + (row % 16) / 4 * 16 + col % 16;
        if (m0 + row >= p.M || col >= cols) continue;
        float v = 0.0f, u = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            v += lds[w * PER_WAVE + at];
            if (GATED) u += lds[w * PER_WAVE + at + COLS * 256];
        }
        if (GATED) with_activation(p.act, [&](auto a) { v = activate<decltype(a)::value>(v) * u; });
        const int64_t to = (int64_t)(m0 + row) * p.ldy + n0 + col;
        if (p.y_type == ATB_TYPE_F32) static_cast<float *>(p.y)[to] = v;
        else static_cast<__bf16 *>(p.y)[to] = (__bf16)v;
    }
}

}  // namespace atb
