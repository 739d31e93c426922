// Products of few rows, y = x W^T with W in bf16, alone or gated: act(x Wg^T) o (x Wu^T).
// Bound: the bytes of the weights; a small one is its launch.
//
// A workgroup has 16 columns of y times a few (NB blocks of 16 rows of weights; of a gated product half of them are the other weight's) and
// 16 MB rows.  Its W waves take the panels of K in turn, and the partial sums are added once at the end through LDS, in wave order: the same
// bits every time, and W does not depend on the rows, so a row's bits do not depend on the others.  A panel is 64 k: one 128-byte line of every row of W.
//
// A wave's panels come straight from memory into two LDS buffers of its own (no barriers: it waits for its own requests), the next one on its way
// while one is multiplied.  A lane of an MFMA needs 16 bytes of one row, its neighbour of the next row; asked for like that, every lane is an
// access of the L1 (63 a request, 86 000 a CU for the block of 16 tokens of 4096, 14336: 36 of its 48 us).  Into LDS eight neighbouring lanes ask for one line.
// Measured, 16 rows, 15 passes over three sets of weights: gated 4096 -> 14336 46.4 us, 5.1 TB/s; plain 14336 -> 4096 26.8 us, 4.4 TB/s.  Among many passes 41.7 and 24.8; one row 39.9
// and 23.6.
#include "atb_stream_rows.h"

namespace atb {
namespace {

template <class S>
__global__ void __launch_bounds__(S::W * 64) stream_kernel(const StreamParams p)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS_BYTES];
    const int m0 = blockIdx.y * 16 * S::MB, n0 = blockIdx.x * 16 * S::COLS, rows = min(p.M - m0, 16 * S::MB), cols = min(p.N - n0, 16 * S::COLS);
    const char *w0 = static_cast<const char *>(p.w[0].w) + n0 * (p.w[0].ldw * 2), *w1 = S::GATED ? static_cast<const char *>(p.w[1].w) + n0 * (p.w[1].ldw * 2) : nullptr;
    const StreamView view = {p.x + (int64_t)m0 * p.ldx, p.ldx, rows, rows, {w0, w1}, {p.w[0].ldw, p.w[1].ldw}, cols, p.K};
    Stream<S> s(view, (unsigned)reinterpret_cast<uintptr_t>(lds), [](int row) { return row; });
    s.run();
    finish_rows<S::MB, S::NB, S::W, S::GATED>(p, s.acc, reinterpret_cast<float *>(lds), m0, n0, cols);
}

template <class S>
hipError_t launch_shape(const StreamParams &p, hipStream_t stream)
{
    constexpr int cols = 16 * S::COLS;
    hipLaunchKernelGGL((stream_kernel<S>), dim3((unsigned)((p.N + cols - 1) / cols), (unsigned)((p.M + 16 * S::MB - 1) / (16 * S::MB))), dim3(S::W * 64), 0, stream, p);
    return hipGetLastError();
}

template <int NB, int W, bool GATED>
hipError_t launch_rows(const StreamParams &p, hipStream_t stream)
{
    if (p.M <= 8) return launch_shape<StreamShape<1, NB, 1, W, GATED>>(p, stream);
    if (p.M <= 16) return launch_shape<StreamShape<1, NB, 2, W, GATED>>(p, stream);
    return launch_shape<StreamShape<2, NB, 4, W, GATED>>(p, stream);
}

}  // namespace

// Waves and columns of a workgroup, us for 16 rows among many passes: gated 4096 -> 14336 in 4 / 8 / 16 waves of 16 + 16 columns 41.7 / 44.1 / 52.5, 14336 -> 4096 in 8 waves of 16 columns
// 24.8 and of 32 (half as many workgroups as CUs) 32.2.
hipError_t launch_stream(const StreamParams &p, hipStream_t stream)
{
    if (p.M == 0) return hipSuccess;
    if (p.group != 0) return launch_q4_stream(p, stream);
    if (p.gated) return launch_rows<2, 4, true>(p, stream);
    if (p.N <= 8192) return launch_rows<1, 8, false>(p, stream);
    return launch_rows<2, 8, false>(p, stream);
}

}  // namespace atb
