// 4-bit weights with group scales: quantiser and decoder.  Bound: decoding HBM, 8192 x 8192 to bf16 30 us, 5.8 TB/s (what it has just written is in part in a cache); quantising the VALU, 8192
// x 8192 in bf16 to groups of 32 with zero points 110 to 125 us, 1.4 TB/s: its instructions, 64-bit divisions for a thread's place among them, take 83 % of the cycles.
// w = s (q - z), q and z in 0 .. 15; a group is G neighbouring k of one row with a scale in bf16 and, if kept, a zero point.
#include "atb_device.h"
#include "atb_layers.h"

namespace atb {
namespace {

// A group is 8 (G = 32) to 32 (G = 128) lanes of four k each.  s is rounded to bf16 first and the codes are taken with the rounded one.
template <class X, int G, bool ZEROS>
__global__ void __launch_bounds__(256) q4_quantize_kernel(const X *__restrict__ w, int64_t ldw, uint8_t *__restrict__ packed, uint16_t *__restrict__ scales,
                                                          uint8_t *__restrict__ zeros, int64_t N, int64_t K)
{
    constexpr int LANES = G / 4;
    const int64_t quads = K / 4, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool live = at < N * quads;                        // whole groups: K % G == 0
    const int64_t n = live ? at / quads : 0, k = live ? at % quads * 4 : 0;
    float x[4], hi = 0.0f, lo = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = live ? (float)w[n * ldw + k + e] : 0.0f;
        hi = fmaxf(hi, x[e]);
        lo = fminf(lo, x[e]);
    }
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
        hi = fmaxf(hi, __shfl_xor(hi, d));
        lo = fminf(lo, __shfl_xor(lo, d));
    }
    const float range = hi - lo;                             // may pass fp32's range: then by halves
    const float step = !ZEROS ? fmaxf(hi, -lo) / 7.0f : range <= 3.402823466e38f ? range / 15.0f : (0.5f * hi - 0.5f * lo) / 7.5f;
    union { __bf16 b; uint16_t w; } s;
    s.b = (__bf16)step;
    const float scale = (float)s.b;
    float z = 8.0f;
    if (ZEROS) z = scale > 0.0f ? fminf(fmaxf(rintf(-lo / scale), 0.0f), 15.0f) : 0.0f;
    unsigned code = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float c = scale > 0.0f ? fminf(fmaxf(rintf(x[e] / scale) + z, 0.0f), 15.0f) : z;
        code |= (unsigned)c << (4 * e);
    }
    if (!live) return;
    *reinterpret_cast<uint16_t *>(packed + n * (K / 2) + k / 2) = (uint16_t)code;
    if (k % G == 0) {
        scales[n * (K / G) + k / G] = s.w;
        if (ZEROS) zeros[n * (K / G) + k / G] = (uint8_t)z;
    }
}

// Eight k per thread.
template <class X>
__global__ void __launch_bounds__(256) q4_decode_kernel(const uint8_t *__restrict__ packed, const uint16_t *__restrict__ scales, const uint8_t *__restrict__ zeros,
                                                        X *__restrict__ out, int64_t N, int64_t K, int group)
{
    const int64_t eights = K / 8, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= N * eights) return;
    const int64_t n = at / eights, k = at % eights * 8, g = n * (K / group) + k / group;
    const unsigned code = *reinterpret_cast<const unsigned *>(packed + n * (K / 2) + k / 2);
    const float s = __uint_as_float((unsigned)scales[g] << 16), z = zeros ? (float)zeros[g] : 8.0f;
    X v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (X)(s * ((float)((code >> (4 * e)) & 15u) - z));
#pragma unroll
    for (int e = 0; e < 8; ++e) out[n * K + k + e] = v[e];
}

// f(first row, rows, workgroups of 256 threads), called with N rows of `threads` threads each: as many at a time as a launch, which has fewer than 2^32 threads, can take.
template <class F>
hipError_t by_rows(int64_t N, int64_t threads, F f)
{
    const int64_t most = ((int64_t)1 << 31) / threads;                // K <= 2^22: a row has at most 2^20
    for (int64_t row = 0; row < N; row += most) {
        const int64_t rows = N - row < most ? N - row : most;
        f(row, rows, dim3((unsigned)((rows * threads + 255) / 256)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class X, int G>
hipError_t quantize(const void *w, int64_t ldw, uint8_t *packed, uint16_t *scales, uint8_t *zeros, int64_t N, int64_t K, hipStream_t stream)
{
    return by_rows(N, K / 4, [&](int64_t row, int64_t rows, dim3 grid) {
        const X *from = static_cast<const X *>(w) + row * ldw;
        uint8_t *codes = packed + row * (K / 2);
        uint16_t *s = scales + row * (K / G);
        if (zeros) hipLaunchKernelGGL((q4_quantize_kernel<X, G, true>), grid, dim3(256), 0, stream, from, ldw, codes, s, zeros + row * (K / G), rows, K);
        else hipLaunchKernelGGL((q4_quantize_kernel<X, G, false>), grid, dim3(256), 0, stream, from, ldw, codes, s, zeros, rows, K);
    });
}

template <class X>
hipError_t quantize(const void *w, int64_t ldw, uint8_t *packed, uint16_t *scales, uint8_t *zeros, int64_t N, int64_t K, int group, hipStream_t stream)
{
    if (group == 32) return quantize<X, 32>(w, ldw, packed, scales, zeros, N, K, stream);
    if (group == 64) return quantize<X, 64>(w, ldw, packed, scales, zeros, N, K, stream);
    return quantize<X, 128>(w, ldw, packed, scales, zeros, N, K, stream);
}

template <class X>
hipError_t decode(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, void *out, int64_t N, int64_t K, int group, hipStream_t stream)
{
    return by_rows(N, K / 8, [&](int64_t row, int64_t rows, dim3 grid) {
        hipLaunchKernelGGL((q4_decode_kernel<X>), grid, dim3(256), 0, stream, packed + row * (K / 2), scales + row * (K / group), zeros ? zeros + row * (K / group) : nullptr,
                           static_cast<X *>(out) + row * K, rows, K, group);
    });
}

}  // namespace

hipError_t launch_q4_quantize(const void *w, int w_type, int64_t ldw, uint8_t *packed, uint16_t *scales, uint8_t *zeros,
                              int64_t N, int64_t K, int group, hipStream_t stream)
{
    if (w_type == ATB_TYPE_F32) return quantize<float>(w, ldw, packed, scales, zeros, N, K, group, stream);
    return quantize<__bf16>(w, ldw, packed, scales, zeros, N, K, group, stream);
}

hipError_t launch_q4_decode(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, void *out, int out_type,
                            int64_t N, int64_t K, int group, hipStream_t stream)
{
    if (out_type == ATB_TYPE_F32) return decode<float>(packed, scales, zeros, out, N, K, group, stream);
    return decode<__bf16>(packed, scales, zeros, out, N, K, group, stream);
}

}  // namespace atb
