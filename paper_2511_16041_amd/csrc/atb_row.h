// What the kernels that hold a row in registers share (atb_norm.hip, atb_residual.hip): 16-byte pieces of rows that begin at any element, sums over the threads of a row; sums over a wave (also atb_moe.hip).
#pragma once

#include "atb_device.h"

namespace atb {

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

// v summed over the wave, in every lane.  Among the 16 lanes of a row by swaps in the registers themselves: a shuffle goes through LDS, six of them one after the other take 800 cycles, and two such sums in a
// row of 7000 cycles were a third of the residual norm's backward pass.
template <int control>
ATB_DEV float swapped(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), control, 0xF, 0xF, true)); }
ATB_DEV float lanes_sum(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    v += swapped<0xB1>(v);           // lanes 1 0 3 2 of every four
    v += swapped<0x4E>(v);           // 2 3 0 1
    v += swapped<0x141>(v);          // 7 .. 0 of every eight
    v += swapped<0x140>(v);          // 15 .. 0 of every row
    const int w = __float_as_int(v);
    v = (__int_as_float(__builtin_amdgcn_readlane(w, 0)) + __int_as_float(__builtin_amdgcn_readlane(w, 16))) + (__int_as_float(__builtin_amdgcn_readlane(w, 32)) + __int_as_float(__builtin_amdgcn_readlane(w, 48)));
#endif
    return v;
}

// The greatest over the wave, in every lane; the same way.  v: no NaN
template <int control>
ATB_DEV double swapped(double v)
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), control, 0xF, 0xF, true), hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), control, 0xF, 0xF, true);
    return __hiloint2double(hi, lo);
}
ATB_DEV double of_lane(double v, int from)
{
    const unsigned lo = __builtin_amdgcn_readlane(__double2loint(v), from), hi = __builtin_amdgcn_readlane(__double2hiint(v), from);
    return __hiloint2double((int)hi, (int)lo);
}
ATB_DEV double lanes_max(double v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    v = fmax(v, swapped<0xB1>(v));
    v = fmax(v, swapped<0x4E>(v));
    v = fmax(v, swapped<0x141>(v));
    v = fmax(v, swapped<0x140>(v));
    v = fmax(fmax(of_lane(v, 0), of_lane(v, 16)), fmax(of_lane(v, 32), of_lane(v, 48)));
#endif
    return v;
}

}  // namespace atb
