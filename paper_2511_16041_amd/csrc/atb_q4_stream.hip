// Products of few rows with 4-bit weights and group scales, alone or gated: act(x Wg^T) o (x Wu^T).
// Floor: the bytes of the weights; a small one is its launch.
//
// A workgroup has 16 columns of y times a few and 16 rows, as in atb_stream.hip: W waves take the panels of K in turn, and their sums are added in
// wave order.  A panel is 256 k, one 128-byte line of every row of W.  A lane asks for 16 bytes of its row, 32 codes; the dwords of four lanes are exchanged (a 4 x 4
// transposition in four lane swaps), so that one MFMA's 32 k lie in one group of 32.  The next panel is asked for ahead of the multiplication, and x, out of a cache, in
// it: with x of a panel in registers as well there is room for half as many waves.  Requests come back in order, so the first MFMA of a panel waits for x and
// with it for the next panel, and that is what bounds these kernels rather than decoding: of the cycles VALU instructions take 40 % (16 rows, 8192 -> 8192) to 44 % (the gated
// product below) and MFMAs 7 to 10 %, the rest is waiting.  Scales and zero points are asked for by 16 lanes, one a column, and handed to the others.
//
// w = s (q - z).  A code becomes bf16 without a conversion: 0x4180 | q << 3 is the number 16 + q.  The MFMAs of a group sum (16 + q) x; one more,
// shared by all columns, sums x; then y += s (sum - (16 + z) sum of x), all in fp32.  (With 0x4300 | q, 128 + q, the sum that is subtracted again is
// 30 times the result's size and not 5, and the error against 64 bits 1.8e-6.)
// Measured: one row, 4096 -> 4096 in groups of 128 5.0 us; gated 4096 -> 14336 in groups of 64 with zero points 21.9 us, 3.0 TB/s, and back 13.1; 16 rows,
// 8192 -> 8192 in groups of 32 with zero points 17.6 us, 2.3 TB/s.  Every block of 16 rows is a workgroup that asks for the weights and decodes them again: 32 rows 34.6 us,
// 64 66.4; 64 rows 4096 -> 4096 23.6, 16 7.1.
#include "atb_stream.h"

namespace atb {
namespace {

constexpr int kPanelK = 256;

ATB_DEV __amdgpu_buffer_rsrc_t rsrc_of(const void *ptr, int64_t bytes) { return uniform_rsrc(static_cast<const char *>(ptr), (int)(bytes < 0x7fffffff ? bytes : 0x7fffffff)); }

// G codes to a scale
template <int G_, int NB_, int W_, bool GATED_, bool ZEROS_>
struct Q4Shape {
    static constexpr int G = G_, NB = NB_, W = W_;
    static constexpr bool GATED = GATED_, ZEROS = ZEROS_;
    static constexpr int COLS = GATED ? NB / 2 : NB;          // blocks of 16 columns of y
    static constexpr int GROUPS = kPanelK / G;                // of a panel
};

template <class S>
struct Q4Stream {
    static constexpr int G = S::G, GROUPS = S::GROUPS, NB = S::NB;
    struct Panel {
        intx4 w[NB][2];
        unsigned s[NB][GROUPS / 2];              // two bf16 each, in lanes 0 .. 15
        unsigned z[S::ZEROS ? NB : 1][(GROUPS + 3) / 4];
    };
    const StreamParams &p;
    const int lane, c, q, wave, m0, n0;
    int rows, cols;
    __amdgpu_buffer_rsrc_t xr, wr[2], sr[2], zr[2];
    int w_off[NB], s_off[NB];
    int x_off;
    floatx4 acc[1][NB];

    ATB_DEV Q4Stream(const StreamParams &p_)
        : p(p_), lane(threadIdx.x & 63), c(lane & 15), q(lane >> 4), wave(__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)), m0(blockIdx.y * 16), n0(blockIdx.x * 16 * S::COLS)
    {
        rows = min(p.M - m0, 16);
        cols = min(p.N - n0, 16 * S::COLS);
        const int64_t groups = p.K / G;
#pragma unroll
        for (int g = 0; g < (S::GATED ? 2 : 1); ++g) {
            const StreamWeight &w = p.w[g];
            wr[g] = rsrc_of(static_cast<const uint8_t *>(w.w) + (int64_t)n0 * (p.K / 2), (int64_t)cols * (p.K / 2));
            sr[g] = rsrc_of(w.scales + n0 * groups, cols * groups * 2);
            if (S::ZEROS) zr[g] = rsrc_of(w.zeros + n0 * groups, cols * groups);
        }
        // rows >= M and columns >= N repeat the last one: they only feed sums that are never stored
        xr = rsrc_of(p.x + (int64_t)m0 * p.ldx, ((int64_t)(rows - 1) * p.ldx + p.K) * 2);
        x_off = min(c, rows - 1) * (int)(p.ldx * 2) + q * 16;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int col = min(16 * (j % S::COLS) + c, cols - 1);
            w_off[j] = col * (p.K / 2) + q * 16;
            s_off[j] = lane < 16 ? col * (p.K / G) : kOutside;
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[0][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    static ATB_DEV intx4 load16(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0); }

    // Panel `panel`
    ATB_DEV void load(Panel &s, int panel)
    {
        const int k0 = panel * kPanelK;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool live = k0 + 128 * h + 32 * q < p.K;                     // K % 32 == 0
                s.w[j][h] = load16(wr[S::GATED && j >= S::COLS], live ? w_off[j] + k0 / 2 + 64 * h : kOutside);
            }
        const bool cut = k0 + kPanelK > p.K;
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
            const int groups = p.K / G - g0;
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

    ATB_DEV void multiply(const Panel &s, int panel)
    {
        constexpr int PER = G / 32, SCHED = S::ZEROS ? 1 : 2;      // MFMAs of a group, and of what is scheduled together (registers)
        const intx4 ones = {0x3F803F80, 0x3F803F80, 0x3F803F80, 0x3F803F80};
        const floatx4 none = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            intx4 x[4], codes[NB];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = panel * kPanelK + 32 * (4 * h + e);                  // K % 32 == 0
                x[e] = load16(xr, k < p.K ? x_off + k * 2 : kOutside);
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
                    const intx4 now = reorder(x[e % 4]);
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

    ATB_DEV void run()
    {
        const int panels = (p.K + kPanelK - 1) / kPanelK;
        Panel a, b;
        int k = wave;
        if (k < panels) load(a, k);
        while (k < panels) {
            if (k + S::W < panels) load(b, k + S::W);
            multiply(a, k);
            k += S::W;
            if (k >= panels) break;
            if (k + S::W < panels) load(a, k + S::W);
            multiply(b, k);
            k += S::W;
        }
    }
};

template <class S>
__global__ void __launch_bounds__(S::W * 64, 4) q4_stream_kernel(const StreamParams p)
{
    __shared__ float lds[S::W * S::NB * 256];
    Q4Stream<S> s(p);
    s.run();
    finish_rows<1, S::NB, S::W, S::GATED>(p, s.acc, lds, s.m0, s.n0, s.cols);
}

template <class S>
hipError_t launch_shape(const StreamParams &p, hipStream_t stream)
{
    constexpr int cols = 16 * S::COLS;
    hipLaunchKernelGGL((q4_stream_kernel<S>), dim3((unsigned)((p.N + cols - 1) / cols), (unsigned)((p.M + 15) / 16)), dim3(S::W * 64), 0, stream, p);
    return hipGetLastError();
}

// Waves and columns of a workgroup: 16 columns as long as these are one workgroup per CU at most (N = 4096), 32 beyond; 16 waves where there is at most one workgroup per CU.  (So
// from N = 4097, 129 workgroups, to 8191 a part of the CUs has none; 16 columns in more workgroups have not been measured there.)
// us, 16 columns in 8 / 16 waves, 32 columns in 8 / 16 waves: one row 14336 -> 4096 in groups of 64 16.3 / 13.1, 23.3 / 18.8; 8192 -> 8192 in groups of 128 14.7 / 15.0, 13.4 / 12.8,
// of 32 with 16 rows 25.2 / 25.2, 17.8 / 17.2; 4096 -> 14336 in groups of 64 - / 16.3, 12.6 / 13.6; gated 4096 -> 14336 in 4 / 8 / 16 waves 22.9 / 21.9 / 25.5.
template <int G, bool ZEROS>
hipError_t launch_group(const StreamParams &p, hipStream_t stream)
{
    if (p.gated) return launch_shape<Q4Shape<G, 2, 8, true, ZEROS>>(p, stream);
    if (p.N <= 4096) return launch_shape<Q4Shape<G, 1, 16, false, ZEROS>>(p, stream);
    if (p.N <= 8192) return launch_shape<Q4Shape<G, 2, 16, false, ZEROS>>(p, stream);
    return launch_shape<Q4Shape<G, 2, 8, false, ZEROS>>(p, stream);
}

template <int G>
hipError_t launch_zeros(const StreamParams &p, hipStream_t stream)
{
    return p.w[0].zeros ? launch_group<G, true>(p, stream) : launch_group<G, false>(p, stream);
}

}  // namespace

// A launch has at most 65535 workgroups in y, of 16 rows each.
hipError_t launch_q4_stream(const StreamParams &p, hipStream_t stream)
{
    constexpr int MOST = 65535 * 16;
    for (int row = 0; row < p.M; row += MOST) {
        StreamParams part = p;
        part.M = p.M - row < MOST ? p.M - row : MOST;
        part.x = p.x + row * p.ldx;
        part.y = static_cast<char *>(p.y) + row * p.ldy * (p.y_type == ATB_TYPE_F32 ? 4 : 2);
        const hipError_t e = p.group == 32 ? launch_zeros<32>(part, stream) : p.group == 64 ? launch_zeros<64>(part, stream) : launch_zeros<128>(part, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace atb
