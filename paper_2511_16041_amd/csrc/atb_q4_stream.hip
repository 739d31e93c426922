// Products of few rows with 4-bit weights and group scales, alone or gated: act(x Wg^T) o (x Wu^T).
// Floor: the bytes of the weights; a small one is its launch.
//
// A workgroup has 16 columns of y times a few and 16 rows, as in atb_stream.hip: W waves take the panels of K in turn, and their sums are added in
// wave order.  A panel is 256 k, one 128-byte line of every row of W.  A lane asks for 16 bytes of its row, 32 codes; the dwords of four lanes are exchanged (a 4 x 4
// transposition in four lane swaps), so that one MFMA's 32 k lie in one group of 32.  Before the multiplication x of the panel, out of a cache, is asked for and behind it the next panel:
// requests come back in order, and with x behind the panel the first MFMA would wait for that too (gated 21.9 us, back 13.1 in the products below).  Two columns of 8 groups with zero points a panel have no
// registers for it: there x is asked for in the multiplication, half a panel at a time, and this wait is what bounds those, with VALU instructions in 40 % of the cycles (16 rows, 8192 -> 8192) and MFMAs in 7 %.  Scales and zero points are asked for by 16 lanes, one a column, and handed to the others.
//
// w = s (q - z).  A code becomes bf16 without a conversion: 0x4180 | q << 3 is the number 16 + q.  The MFMAs of a group sum (16 + q) x; one more,
// shared by all columns, sums x; then y += s (sum - (16 + z) sum of x), all in fp32.  (With 0x4300 | q, 128 + q, the sum that is subtracted again is
// 30 times the result's size and not 5, and the error against 64 bits 1.8e-6.)
// Measured: one row, 4096 -> 4096 in groups of 128 5.0 us; gated 4096 -> 14336 in groups of 64 with zero points 20.5 us, 3.2 TB/s, and back 11.5; 16 rows,
// 8192 -> 8192 in groups of 32 with zero points 17.6 us, 2.3 TB/s.  Every block of 16 rows is a workgroup that asks for the weights and decodes them again: 32 rows 34.6 us,
// 64 66.4; 64 rows 4096 -> 4096 23.6, 16 7.1.
#include "atb_q4_rows.h"

namespace atb {
namespace {

template <class S>
__global__ void __launch_bounds__(S::W * 64, 4) q4_stream_kernel(const StreamParams p)
{
    __shared__ float lds[S::W * S::NB * 256];
    const int m0 = blockIdx.y * 16, n0 = blockIdx.x * 16 * S::COLS, rows = min(p.M - m0, 16), cols = min(p.N - n0, 16 * S::COLS);
    const Q4View view = {p.x + (int64_t)m0 * p.ldx, p.ldx, rows, rows, {q4_columns(p.w[0], n0, p.K, S::G), q4_columns(p.w[1], S::GATED ? n0 : 0, p.K, S::G)}, cols, p.K};
    Q4Stream<S> s(view);
    s.run([&] { s.open_rows(view, [](int row) { return row; }); });
    finish_rows<1, S::NB, S::W, S::GATED>(p, s.acc, lds, m0, n0, cols);
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
