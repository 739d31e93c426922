// The waves of the kernels for few rows with weights in 4 bits (atb_q4_stream.hip has how they work; also atb_moe_q4.hip).
#pragma once

#include "atb_stream.h"

namespace atb {

constexpr int kQ4PanelK = 256;

ATB_DEV __amdgpu_buffer_rsrc_t rsrc_of(const void *ptr, int64_t bytes) { return uniform_rsrc(static_cast<const char *>(ptr), (int)(bytes < 0x7fffffff ? bytes : 0x7fffffff)); }

// G codes to a scale
template <int G_, int NB_, int W_, bool GATED_, bool ZEROS_>
struct Q4Shape {
    static constexpr int G = G_, NB = NB_, W = W_;
    static constexpr bool GATED = GATED_, ZEROS = ZEROS_;
    static constexpr int COLS = GATED ? NB / 2 : NB;          // blocks of 16 columns of y
    static constexpr int GROUPS = kQ4PanelK / G;                // of a panel
};

// A weight of K inputs from row n on
ATB_DEV StreamWeight q4_columns(const StreamWeight &w, int64_t n, int64_t K, int group)
{
    return {static_cast<const uint8_t *>(w.w) + n * (K / 2), w.scales + n * (K / group), w.zeros ? w.zeros + n * (K / group) : nullptr, 0};
}

// What a workgroup multiplies, as StreamView; w: of its first column
struct Q4View {
    const uint16_t *x;
    int64_t ldx;
    int x_rows, rows;                        // rows: 16 at most
    StreamWeight w[2];
    int cols, K;
};

template <class S>
struct Q4Stream {
    static constexpr int G = S::G, GROUPS = S::GROUPS, NB = S::NB;
    struct Panel {
        intx4 w[NB][2];
        unsigned s[NB][GROUPS / 2];              // two bf16 each, in lanes 0 .. 15
        unsigned z[S::ZEROS ? NB : 1][(GROUPS + 3) / 4];
    };
    const int lane, c, q, wave;
    int K;
    __amdgpu_buffer_rsrc_t xr, wr[2], sr[2], zr[2];
    int w_off[NB], s_off[NB];
    int x_off;
    floatx4 acc[1][NB];

    // (open_rows is the caller's)
    ATB_DEV Q4Stream(const Q4View &v) : lane(threadIdx.x & 63), c(lane & 15), q(lane >> 4), wave(__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)), K(v.K)
    {
#pragma unroll
        for (int g = 0; g < (S::GATED ? 2 : 1); ++g) open_weight(v, g);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int col = min(16 * (j % S::COLS) + c, v.cols - 1);
            w_off[j] = col * (K / 2) + q * 16;
            s_off[j] = lane < 16 ? col * (K / G) : kOutside;
        }
        clear();
    }
    ATB_DEV void clear()
    {
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[0][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    ATB_DEV void open_weight(const Q4View &v, int g)
    {
        const int64_t groups = K / G;
        const StreamWeight &w = v.w[g];
        wr[g] = rsrc_of(w.w, (int64_t)v.cols * (K / 2));
        sr[g] = rsrc_of(w.scales, v.cols * groups * 2);
        if (S::ZEROS) zr[g] = rsrc_of(w.zeros, v.cols * groups);
    }
    // Row i of the workgroup is row row_of(i) of x.  Rows >= M and columns >= N repeat the last one: they only feed sums that are never stored
    template <class F>
    ATB_DEV void open_rows(const Q4View &v, F row_of)
    {
        xr = rsrc_of(v.x, ((int64_t)(v.x_rows - 1) * v.ldx + K) * 2);
        x_off = row_of(min(c, v.rows - 1)) * (int)(v.ldx * 2) + q * 16;
    }

    static ATB_DEV intx4 load16(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0); }

    // Panel `panel`
    ATB_DEV void load(Panel &s, int panel)
    {
        const int k0 = panel * kQ4PanelK;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool live = k0 + 128 * h + 32 * q < K;                     // K % 32 == 0
                s.w[j][h] = load16(wr[S::GATED && j >= S::COLS], live ? w_off[j] + k0 / 2 + 64 * h : kOutside);
            }
        const bool cut = k0 + kQ4PanelK > K;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (cut) load_scales<true>(s, j, k0 / G);
            else load_scales<false>(s, j, k0 / G);
        }
    }

    // The scales and zero points of a panel.  A whole panel's are one request, which lies inside the row; of a cut one they are fetched one by
    // one (a request checks whole dwords against the end, and the last scale may be half of one).  Lanes 16 .. 63 ask for nothing: an offset past the end, which stays there when
    // the groups are added.
    template <bool CUT>
    ATB_DEV void load_scales(Panel &s, int j, int g0)
    {
        const __amdgpu_buffer_rsrc_t r = sr[S::GATED && j >= S::COLS], zs = zr[S::GATED && j >= S::COLS];
        const int at = lane < 16 ? (s_off[j] + g0) * 2 : kOutside, za = s_off[j] + g0;
        if constexpr (CUT) {
            const int groups = K / G - g0;
#pragma unroll
            for (int g = 0; g < GROUPS; g += 2) {
                const unsigned lo = g < groups ? __builtin_amdgcn_raw_buffer_load_b16(r, at + 2 * g, 0, 0) : 0;
                const unsigned hi = g + 1 < groups ? __builtin_amdgcn_raw_buffer_load_b16(r, at + 2 * g + 2, 0, 0) : 0;
                s.s[j][g / 2] = (lo & 0xFFFFu) | (hi << 16);
            }
            if constexpr (S::ZEROS)
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const unsigned b = g < groups ? __builtin_amdgcn_raw_buffer_load_b8(zs, za + g, 0, 0) & 0xFFu : 0;
                    s.z[j][g / 4] = g % 4 == 0 ? b : s.z[j][g / 4] | b << 8 * (g % 4);
                }
        } else {
            if constexpr (GROUPS == 2) {
                s.s[j][0] = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
            } else if constexpr (GROUPS == 4) {
                const intx2 v = __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
                s.s[j][0] = v.x;
                s.s[j][1] = v.y;
            } else {
                const intx4 v = load16(r, at);
#pragma unroll
                for (int e = 0; e < 4; ++e) s.s[j][e] = v[e];
            }
            if constexpr (S::ZEROS) {
                if constexpr (GROUPS == 2) {
                    s.z[j][0] = __builtin_amdgcn_raw_buffer_load_b16(zs, za, 0, 0);
                } else if constexpr (GROUPS == 4) {
                    s.z[j][0] = __builtin_amdgcn_raw_buffer_load_b32(zs, za, 0, 0);
                } else {
                    const intx2 v = __builtin_amdgcn_raw_buffer_load_b64(zs, za, 0, 0);
                    s.z[j][0] = v.x;
                    s.z[j][1] = v.y;
                }
            }
        }
    }
    // Lane l % 16's value in every lane l
    ATB_DEV unsigned of_column(unsigned v) const { return (unsigned)__builtin_amdgcn_ds_bpermute(c * 4, (int)v); }

    static ATB_DEV void swap32(int &a, int &b)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
        const uintx2 r = __builtin_amdgcn_permlane32_swap((unsigned)a, (unsigned)b, false, false);
        a = (int)r.x;
        b = (int)r.y;
#endif
    }
    static ATB_DEV void swap16(int &a, int &b)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
        const uintx2 r = __builtin_amdgcn_permlane16_swap((unsigned)a, (unsigned)b, false, false);
        a = (int)r.x;
        b = (int)r.y;
#endif
    }
    // Dword d of lane group g <-> dword g of lane group d: afterwards dword e of lane group g holds k = 32 e + 8 g .. + 7 of the 128.
    static ATB_DEV intx4 transpose(const intx4 &v)
    {
        int a = v[0], b = v[1], d = v[2], e = v[3];
        swap32(a, d);
        swap32(b, e);
        swap16(a, b);
        swap16(d, e);
        return intx4{a, b, d, e};
    }
    // Eight codes as bf16 16 + q, in the order k = 0 4 1 5 2 6 3 7 ..
    static ATB_DEV intx4 expand(unsigned v)
    {
        constexpr unsigned mask = 0x00780078u, one = 0x41804180u;
        return intx4{(int)((v << 3 & mask) | one), (int)((v >> 1 & mask) | one), (int)((v >> 5 & mask) | one), (int)((v >> 9 & mask) | one)};
    }
    // .. and eight elements of x in the same
    static ATB_DEV intx4 reorder(const intx4 &x)
    {
        intx4 r = {};
#if defined(__HIP_DEVICE_COMPILE__)
        r[0] = (int)__builtin_amdgcn_perm((unsigned)x[2], (unsigned)x[0], 0x05040100u);
        r[1] = (int)__builtin_amdgcn_perm((unsigned)x[2], (unsigned)x[0], 0x07060302u);
        r[2] = (int)__builtin_amdgcn_perm((unsigned)x[3], (unsigned)x[1], 0x05040100u);
        r[3] = (int)__builtin_amdgcn_perm((unsigned)x[3], (unsigned)x[1], 0x07060302u);
#endif
        return r;
    }

    // x of a panel, asked for ahead of the next panel's weights: requests come back in order, and the first MFMA would wait for these too.  With scales and zero points of 8 groups of two columns there are no
    // registers for that: half a panel's is asked for where it is multiplied.
    static constexpr bool ROWS_FIRST = !(GROUPS == 8 && NB > 1);
    struct Rows { intx4 x[ROWS_FIRST ? 8 : 4]; int panel; };
    template <int from, int count>
    ATB_DEV void ask_rows(Rows &r) const
    {
#pragma unroll
        for (int e = from; e < from + count; ++e) {
            const int k = r.panel * kQ4PanelK + 32 * e;                            // K % 32 == 0
            r.x[e % (ROWS_FIRST ? 8 : 4)] = load16(xr, k < K ? x_off + k * 2 : kOutside);
        }
    }
    ATB_DEV void load_rows(Rows &r, int panel) const
    {
        r.panel = panel;
        if constexpr (ROWS_FIRST) {
            ask_rows<0, 8>(r);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    ATB_DEV void multiply(const Panel &s, Rows &r)
    {
        if constexpr (ROWS_FIRST) __builtin_amdgcn_sched_barrier(0);
        constexpr int PER = G / 32, SCHED = S::ZEROS ? 1 : 2;      // MFMAs of a group, and of what is scheduled together (registers)
        const intx4 ones = {0x3F803F80, 0x3F803F80, 0x3F803F80, 0x3F803F80};
        const floatx4 none = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            intx4 codes[NB];
            if constexpr (!ROWS_FIRST) {
                if (h == 0) ask_rows<0, 4>(r);
                else ask_rows<4, 4>(r);
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) codes[j] = transpose(s.w[j][h]);
#pragma unroll
            for (int g = h * GROUPS / 2; g < (h + 1) * GROUPS / 2; ++g) {
                if (g * PER % SCHED == 0) __builtin_amdgcn_sched_barrier(0);
                floatx4 sum[NB], xs = none;
#pragma unroll
                for (int j = 0; j < NB; ++j) sum[j] = none;
#pragma unroll
                for (int e = g * PER; e < (g + 1) * PER; ++e) {
                    const intx4 now = reorder(r.x[e % (ROWS_FIRST ? 8 : 4)]);
                    xs = mfma_rows(now, ones, xs);
#pragma unroll
                    for (int j = 0; j < NB; ++j) sum[j] = mfma_rows(now, expand((unsigned)codes[j][e % 4]), sum[j]);
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const unsigned two = of_column(s.s[j][g / 2]);
                    const float scale = __uint_as_float(g % 2 == 0 ? two << 16 : two & 0xFFFF0000u);
                    float bias = -24.0f;
                    if constexpr (S::ZEROS) bias = -16.0f - (float)((of_column(s.z[j][g / 4]) >> (8 * (g % 4))) & 0xFFu);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[0][j][e] = fmaf(scale, fmaf(bias, xs[e], sum[j][e]), acc[0][j][e]);
                }
            }
        }
    }

    // open: called once the first weights have been asked for; opens the rows
    template <class F>
    ATB_DEV void run(F open)
    {
        const int panels = (K + kQ4PanelK - 1) / kQ4PanelK;
        Panel a, b;
        Rows r;
        int k = wave;
        if (k < panels) load(a, k);
        open();
        while (k < panels) {
            load_rows(r, k);
            if (k + S::W < panels) load(b, k + S::W);
            multiply(a, r);
            k += S::W;
            if (k >= panels) break;
            load_rows(r, k);
            if (k + S::W < panels) load(a, k + S::W);
            multiply(b, r);
            k += S::W;
        }
    }
};

}  // namespace atb
