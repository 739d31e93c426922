// Products of few rows, y = x W^T with W in bf16 or in 4 bits with group scales, alone or gated: act(x Wg^T) o (x Wu^T).
// Bound: the bytes of the weights; a small one is its launch.
//
// A workgroup has 16 columns of y times a few (NB blocks of 16 columns of weights; of a gated product half of them are the other weight's) and
// 16 MB rows.  Its waves take the panels of K in turn, load their operands straight into registers in MFMA layout, and the partial sums
// are added once at the end through LDS, in wave order: the same bits every time.  A panel is one 128-byte line of a row of W: 64 k in
// bf16, 256 k in 4 bits, and the next panel is asked for before this one is multiplied.
//
// v_mfma_f32_16x16x32_bf16 with x as the first operand: lane l supplies row l % 16 of x and column l % 16 of W^T at 8 k values of group
// l / 16, and holds column l % 16 and rows 4 (l / 16) .. + 3 of the result, so that a column's scale is one value per lane.
//
// 4 bits: w = s (q - z).  A lane asks for 16 bytes, 32 codes of one row; four lanes' dwords are exchanged (a 4 x 4 transposition in four
// lane swaps) so that one MFMA's 32 k lie in one group of 32.  A code becomes bf16 without a conversion: 0x4300 | q is the number 128 + q.  The
// MFMAs of a group sum (128 + q) x; one more, shared by all columns, sums x; then y += s (sum - (128 + z) sum of x), all in fp32.  The
// sum of 128 x costs up to 5 of fp32's 24 bits against the sum of (q - z) x.
#include <type_traits>

#include "atb_activation.h"
#include "atb_layers.h"

namespace atb {
namespace {

constexpr int kWaves = 8;
constexpr int kOutside = (int)0x80000000;        // an offset past the end of every descriptor: reads as zero

ATB_DEV __amdgpu_buffer_rsrc_t rsrc_of(const void *ptr, int64_t bytes) { return uniform_rsrc(static_cast<const char *>(ptr), (int)(bytes < 0x7fffffff ? bytes : 0x7fffffff)); }

ATB_DEV floatx4 mfma(const intx4 &x, const intx4 &w, const floatx4 &acc)
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

// ---- weights in bf16

template <int MB, int NB>
struct Bf16Panel {
    static constexpr int K = 64;
    intx4 w[NB][2], x[MB][2];
};

// ---- weights in 4 bits, G codes to a scale

template <int MB, int NB, int G, bool ZEROS>
struct Q4Panel {
    static constexpr int K = 256, GROUPS = K / G;
    static constexpr bool X = MB == 1;           // x is asked for with the weights; of more rows it comes, from a cache, when it is needed (registers)
    intx4 w[NB][2], x[X ? MB : 1][X ? 8 : 4];
    unsigned s[NB][GROUPS / 2];                  // two bf16 each
    unsigned z[ZEROS ? NB : 1][(GROUPS + 3) / 4];
};

// FMT: 0 (bf16), or the group size
template <int FMT, int MB, int NB, bool GATED, bool ZEROS>
struct Stream {
    static constexpr int COLS = GATED ? NB / 2 : NB;          // blocks of 16 columns of y
    typedef typename std::conditional<FMT == 0, Bf16Panel<MB, NB>, Q4Panel<MB, NB, FMT ? FMT : 128, ZEROS>>::type Panel;
    static constexpr int GROUPS = FMT ? 256 / (FMT ? FMT : 1) : 2;
    const StreamParams &p;
    int lane, c, q, wave, m0, n0;
    __amdgpu_buffer_rsrc_t xr, wr[2], sr[2], zr[2];
    int x_off[MB], w_off[NB], s_off[NB];
    floatx4 acc[MB][NB];

    ATB_DEV Stream(const StreamParams &p_) : p(p_)
    {
        lane = threadIdx.x & 63;
        c = lane & 15;
        q = lane >> 4;
        wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        m0 = blockIdx.y * 16 * MB;
        n0 = blockIdx.x * 16 * COLS;
        const int rows = min(p.M - m0, 16 * MB), cols = min(p.N - n0, 16 * COLS);
        xr = rsrc_of(p.x + (int64_t)m0 * p.ldx, ((int64_t)(rows - 1) * p.ldx + p.K) * 2);
        // rows >= M and columns >= N repeat the last one: they only feed sums that are never stored
#pragma unroll
        for (int i = 0; i < MB; ++i) x_off[i] = min(16 * i + c, rows - 1) * (int)(p.ldx * 2);
#pragma unroll
        for (int g = 0; g < (GATED ? 2 : 1); ++g) {
            const StreamWeight &w = p.w[g];
            if constexpr (FMT == 0) {
                wr[g] = rsrc_of(static_cast<const uint16_t *>(w.w) + (int64_t)n0 * w.ldw, ((int64_t)(cols - 1) * w.ldw + p.K) * 2);
            } else {
                const int64_t groups = p.K / FMT;
                wr[g] = rsrc_of(static_cast<const uint8_t *>(w.w) + (int64_t)n0 * (p.K / 2), (int64_t)cols * (p.K / 2));
                sr[g] = rsrc_of(w.scales + n0 * groups, cols * groups * 2);
                if (ZEROS) zr[g] = rsrc_of(w.zeros + n0 * groups, cols * groups);
            }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int col = min(16 * (j % COLS) + c, cols - 1);
            if constexpr (FMT == 0) w_off[j] = col * (int)(p.w[GATED && j >= COLS].ldw * 2);
            else {
                w_off[j] = col * (p.K / 2);
                s_off[j] = col * (p.K / FMT);
            }
        }
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    static ATB_DEV intx4 load16(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0); }

    // Panel k; CUT: the last one, which K ends in.
    template <bool CUT>
    ATB_DEV void load(Panel &s, int panel)
    {
        const int k0 = panel * Panel::K;
        if constexpr (FMT == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 16 * q + 8 * h, dead = CUT && k >= p.K ? kOutside : 0;        // K % 8 == 0
#pragma unroll
                for (int j = 0; j < NB; ++j) s.w[j][h] = load16(wr[GATED && j >= COLS], (w_off[j] + k * 2) | dead);
#pragma unroll
                for (int i = 0; i < MB; ++i) s.x[i][h] = load16(xr, (x_off[i] + k * 2) | dead);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 128 * h + 32 * q, dead = CUT && k >= p.K ? kOutside : 0;      // K % 32 == 0
#pragma unroll
                for (int j = 0; j < NB; ++j) s.w[j][h] = load16(wr[GATED && j >= COLS], (w_off[j] + k / 2) | dead);
            }
            const int g0 = k0 / FMT;
#pragma unroll
            for (int j = 0; j < NB; ++j) load_scales<CUT>(s, j, g0);
            if constexpr (Panel::X) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s.x[0][e] = load_x<CUT>(0, k0, e);
            }
        }
    }

    // Row block i of x at the 32 k of MFMA e of a 4-bit panel
    template <bool CUT>
    ATB_DEV intx4 load_x(int i, int k0, int e)
    {
        const int k = k0 + 32 * e + 8 * q, dead = CUT && k >= p.K ? kOutside : 0;
        return load16(xr, (x_off[i] + k * 2) | dead);
    }

    // The scales and zero points of a panel.  A whole panel's are one request, which lies inside the row; of a cut one they are fetched one by
    // one (a request checks whole dwords against the end, and the last scale may be half of one).
    template <bool CUT>
    ATB_DEV void load_scales(Panel &s, int j, int g0)
    {
        if constexpr (FMT != 0) {
            const __amdgpu_buffer_rsrc_t r = sr[GATED && j >= COLS];
            const int at = s_off[j] + g0;
            if constexpr (CUT) {
                const int groups = p.K / FMT - g0;
#pragma unroll
                for (int g = 0; g < GROUPS; g += 2) {
                    const unsigned lo = g < groups ? __builtin_amdgcn_raw_buffer_load_b16(r, (at + g) * 2, 0, 0) : 0;
                    const unsigned hi = g + 1 < groups ? __builtin_amdgcn_raw_buffer_load_b16(r, (at + g + 1) * 2, 0, 0) : 0;
                    s.s[j][g / 2] = (lo & 0xFFFFu) | (hi << 16);
                }
            } else if constexpr (GROUPS == 2) {
                s.s[j][0] = __builtin_amdgcn_raw_buffer_load_b32(r, at * 2, 0, 0);
            } else if constexpr (GROUPS == 4) {
                const intx2 v = __builtin_amdgcn_raw_buffer_load_b64(r, at * 2, 0, 0);
                s.s[j][0] = v.x;
                s.s[j][1] = v.y;
            } else {
                const intx4 v = load16(r, at * 2);
#pragma unroll
                for (int e = 0; e < 4; ++e) s.s[j][e] = v[e];
            }
            if constexpr (ZEROS) {
                const __amdgpu_buffer_rsrc_t zs = zr[GATED && j >= COLS];
                if constexpr (CUT) {
                    const int groups = p.K / FMT - g0;
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const unsigned b = g < groups ? __builtin_amdgcn_raw_buffer_load_b8(zs, at + g, 0, 0) & 0xFFu : 0;
                        s.z[j][g / 4] = g % 4 == 0 ? b : s.z[j][g / 4] | b << 8 * (g % 4);
                    }
                } else if constexpr (GROUPS == 2) {
                    s.z[j][0] = __builtin_amdgcn_raw_buffer_load_b16(zs, at, 0, 0);
                } else if constexpr (GROUPS == 4) {
                    s.z[j][0] = __builtin_amdgcn_raw_buffer_load_b32(zs, at, 0, 0);
                } else {
                    const intx2 v = __builtin_amdgcn_raw_buffer_load_b64(zs, at, 0, 0);
                    s.z[j][0] = v.x;
                    s.z[j][1] = v.y;
                }
            }
        }
    }

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
    static ATB_DEV void transpose(intx4 &v)
    {
        int a = v[0], b = v[1], d = v[2], e = v[3];
        swap32(a, d);
        swap32(b, e);
        swap16(a, b);
        swap16(d, e);
        v = intx4{a, b, d, e};
    }
    // Eight codes as bf16 128 + q, in the order k = 0 4 1 5 2 6 3 7 ..
    static ATB_DEV intx4 expand(unsigned v)
    {
        intx4 r = {};
#pragma unroll
        for (int t = 0; t < 4; ++t) r[t] = (int)(((v >> (4 * t)) & 0x000F000Fu) | 0x43004300u);
        return r;
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

    template <bool CUT>
    ATB_DEV void multiply(Panel &s, int panel)
    {
        if constexpr (FMT == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] = mfma(s.x[i][h], s.w[j][h], acc[i][j]);
        } else {
            constexpr int PER = FMT / 32;                     // MFMAs of a group
            const intx4 ones = {0x3F803F80, 0x3F803F80, 0x3F803F80, 0x3F803F80};
            const floatx4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NB; ++j) transpose(s.w[j][h]);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                floatx4 sum[MB][NB], xs[MB];
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    xs[i] = zero;
#pragma unroll
                    for (int j = 0; j < NB; ++j) sum[i][j] = zero;
                }
#pragma unroll
                for (int e = g * PER; e < (g + 1) * PER; ++e) {
                    intx4 w[NB];
#pragma unroll
                    for (int j = 0; j < NB; ++j) w[j] = expand((unsigned)s.w[j][e / 4][e % 4]);
#pragma unroll
                    for (int i = 0; i < MB; ++i) {
                        const intx4 x = reorder(MB == 1 ? s.x[0][MB == 1 ? e : 0] : load_x<CUT>(i, panel * Panel::K, e));
                        xs[i] = mfma(x, ones, xs[i]);
#pragma unroll
                        for (int j = 0; j < NB; ++j) sum[i][j] = mfma(x, w[j], sum[i][j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const float scale = __uint_as_float(g % 2 == 0 ? s.s[j][g / 2] << 16 : s.s[j][g / 2] & 0xFFFF0000u);
                    float bias = -136.0f;
                    if constexpr (ZEROS) bias = -128.0f - (float)((s.z[j][g / 4] >> (8 * (g % 4))) & 0xFFu);
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(scale, fmaf(bias, xs[i][e], sum[i][j][e]), acc[i][j][e]);
                }
            }
        }
    }

    // This wave's panels: all but a cut one with the next in flight, then the cut one.
    ATB_DEV void run()
    {
        const int whole = p.K / Panel::K, cut = p.K % Panel::K != 0 ? whole : -1;
        Panel a, b;
        int k = wave;
        if (k < whole) load<false>(a, k);
        while (k < whole) {
            if (k + kWaves < whole) load<false>(b, k + kWaves);
            multiply<false>(a, k);
            k += kWaves;
            if (k >= whole) break;
            if (k + kWaves < whole) load<false>(a, k + kWaves);
            multiply<false>(b, k);
            k += kWaves;
        }
        if (cut >= 0 && cut % kWaves == wave) {
            load<true>(a, cut);
            multiply<true>(a, cut);
        }
    }

    // Partial sums of all waves, added in wave order.
    ATB_DEV void finish(float *lds)
    {
        constexpr int PER_WAVE = MB * NB * 256;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) lds[wave * PER_WAVE + ((i * NB + j) * 4 + e) * 64 + lane] = acc[i][j][e];
        __syncthreads();
        // thread -> row, column with neighbouring threads in neighbouring columns
        for (int o = threadIdx.x; o < MB * 16 * COLS * 16; o += kWaves * 64) {
            const int col = o % (COLS * 16), row = o / (COLS * 16);
            const int i = row / 16, j = col / 16, at = ((i * NB + j) * 4 + row % 4) * 64 + (row % 16) / 4 * 16 + col % 16;
            float v = 0.0f, u = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                v += lds[w * PER_WAVE + at];
                if (GATED) u += lds[w * PER_WAVE + at + COLS * 256];
            }
            if (GATED) with_activation(p.act, [&](auto a) { v = activate<decltype(a)::value>(v) * u; });
            if (m0 + row < p.M && n0 + col < p.N) {
                const int64_t to = (int64_t)(m0 + row) * p.ldy + n0 + col;
                if (p.y_type == ATB_TYPE_F32) static_cast<float *>(p.y)[to] = v;
                else static_cast<__bf16 *>(p.y)[to] = (__bf16)v;
            }
        }
    }
};

template <int FMT, int MB, int NB, bool GATED, bool ZEROS>
__global__ void __launch_bounds__(kWaves * 64) stream_kernel(const StreamParams p)
{
    __shared__ float lds[kWaves * MB * NB * 256];
    Stream<FMT, MB, NB, GATED, ZEROS> s(p);
    s.run();
    s.finish(lds);
}

template <int FMT, int MB, int NB, bool GATED, bool ZEROS>
hipError_t launch_shape(const StreamParams &p, hipStream_t stream)
{
    constexpr int cols = 16 * (GATED ? NB / 2 : NB);
    hipLaunchKernelGGL((stream_kernel<FMT, MB, NB, GATED, ZEROS>), dim3((unsigned)((p.N + cols - 1) / cols), (unsigned)((p.M + 16 * MB - 1) / (16 * MB))),
                       dim3(kWaves * 64), 0, stream, p);
    return hipGetLastError();
}

template <int FMT, bool GATED, bool ZEROS>
hipError_t launch_rows(const StreamParams &p, hipStream_t stream)
{
    if (p.M <= 16) return launch_shape<FMT, 1, 2, GATED, ZEROS>(p, stream);
    return launch_shape<FMT, 2, 2, GATED, ZEROS>(p, stream);
}

template <int FMT>
hipError_t launch_format(const StreamParams &p, hipStream_t stream)
{
    if (FMT != 0 && p.w[0].zeros) return p.gated ? launch_rows<FMT, true, FMT != 0>(p, stream) : launch_rows<FMT, false, FMT != 0>(p, stream);
    return p.gated ? launch_rows<FMT, true, false>(p, stream) : launch_rows<FMT, false, false>(p, stream);
}

}  // namespace

hipError_t launch_stream(const StreamParams &p, hipStream_t stream)
{
    if (p.M == 0) return hipSuccess;
    if (p.group == 0) return launch_format<0>(p, stream);
    if (p.group == 32) return launch_format<32>(p, stream);
    if (p.group == 64) return launch_format<64>(p, stream);
    return launch_format<128>(p, stream);
}

}  // namespace atb
