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
#include "atb_stream.h"

namespace atb {
namespace {

struct Descriptor {
    const char *ptr;
    int64_t bytes;
    ATB_DEV intx4 words() const
    {
        const uint64_t a = reinterpret_cast<uint64_t>(ptr);
        return intx4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF),
                     __builtin_amdgcn_readfirstlane((int)(bytes < 0x7fffffff ? bytes : 0x7fffffff)), kRsrcFlags};
    }
};

// XQ: requests of 8 rows for x per panel
template <int MB_, int NB_, int XQ_, int W_, bool GATED_>
struct StreamShape {
    static constexpr int MB = MB_, NB = NB_, XQ = XQ_, W = W_;
    static constexpr bool GATED = GATED_;
    static constexpr int COLS = GATED ? NB / 2 : NB;          // blocks of 16 columns of y
    static constexpr int K = 64;                              // of a panel
    static constexpr int REQS = 2 * NB + XQ;                  // of a panel, 1 KiB each
    static constexpr int SLOT = REQS * 1024, LDS_BYTES = W * 2 * SLOT;
    static_assert(LDS_BYTES >= W * MB * NB * 1024, "the partial sums take the ring's place");
};

template <class S>
struct Stream {
    const StreamParams &p;
    const int lane, c, q, wave, m0, n0;
    int cols;
    unsigned ring;                             // LDS: this wave's two buffers
    Descriptor xd, wd[2];
    int x_off[S::XQ], w_off[S::NB][2];
    floatx4 acc[S::MB][S::NB];

    ATB_DEV Stream(const StreamParams &p_, unsigned lds)
        : p(p_), lane(threadIdx.x & 63), c(lane & 15), q(lane >> 4), wave(__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)), m0(blockIdx.y * 16 * S::MB), n0(blockIdx.x * 16 * S::COLS)
    {
        ring = __builtin_amdgcn_readfirstlane(lds + wave * 2 * S::SLOT);
        const int rows = min(p.M - m0, 16 * S::MB);
        cols = min(p.N - n0, 16 * S::COLS);
        xd = {reinterpret_cast<const char *>(p.x + (int64_t)m0 * p.ldx), ((int64_t)(rows - 1) * p.ldx + p.K) * 2};
        // a request: lane l asks for the chunk of 16 bytes that the swizzle keeps at place l of its 8 rows of 128 bytes; rows outside ask for nothing
#pragma unroll
        for (int i = 0; i < S::XQ; ++i) {
            const int row = 8 * i + lane / 8;
            x_off[i] = row < rows ? row * (int)(p.ldx * 2) + chunk() * 16 : kOutside;
        }
#pragma unroll
        for (int g = 0; g < (S::GATED ? 2 : 1); ++g) {
            const int64_t pitch = p.w[g].ldw * 2;
            wd[g] = {static_cast<const char *>(p.w[g].w) + n0 * pitch, (cols - 1) * pitch + p.K * 2};
#pragma unroll
            for (int j = g * S::COLS; j < (S::GATED ? (g + 1) * S::COLS : S::NB); ++j)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int col = 16 * (j - g * S::COLS) + 8 * r + lane / 8;
                    w_off[j][r] = col < cols ? col * (int)pitch + chunk() * 16 : kOutside;
                }
        }
#pragma unroll
        for (int i = 0; i < S::MB; ++i)
#pragma unroll
            for (int j = 0; j < S::NB; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Chunk c of row r lies at c ^ (r % 8) of its 128 bytes.
    ATB_DEV int chunk() const { return (lane & 7) ^ (lane >> 3); }

    // 16 bytes per lane from memory to LDS, by hand: the compiler would wait for it before every read of LDS that follows.  M0, the LDS address, is put back.
    static ATB_DEV void request_one(intx4 words, int off, unsigned to)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        int saved;
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved)
                     : "s"(to), "v"(off), "s"(words) : "memory");
#endif
    }
    // Panel `panel` into buffer `slot`.  What lies past the end of a row is the next row's: its chunks are not asked for (K % 8 == 0).
    ATB_DEV void request(int panel, int slot)
    {
        const bool live = chunk() * 8 < p.K - panel * S::K;
        const unsigned to = ring + slot * S::SLOT;
#pragma unroll
        for (int j = 0; j < S::NB; ++j)
#pragma unroll
            for (int r = 0; r < 2; ++r) request_one(wd[S::GATED && j >= S::COLS].words(), live ? w_off[j][r] + panel * 128 : kOutside, to + (2 * j + r) * 1024);
#pragma unroll
        for (int i = 0; i < S::XQ; ++i) request_one(xd.words(), live ? x_off[i] + panel * 128 : kOutside, to + (2 * S::NB + i) * 1024);
    }
    template <int younger>
    static ATB_DEV void wait() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(younger) : "memory"); }

    // 16 rows of 128 bytes at `at`: this lane's operand of MFMA e (row c, the 8 k of group q)
    ATB_DEV intx4 read(unsigned at, int row, int e) const { return lds_read<intx4>(at + row * 128 + (((4 * e + q) ^ (row & 7)) * 16)); }

    ATB_DEV void multiply(int slot)
    {
        const unsigned at = ring + slot * S::SLOT;
        intx4 w[S::NB][2], x[S::MB][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            // (row blocks whose rows no request brings, of 8 rows or fewer, repeat others: their sums are not stored)
#pragma unroll
            for (int i = 0; i < S::MB; ++i) x[i][e] = read(at + 2 * S::NB * 1024, (16 * i + c) % (8 * S::XQ), e);
#pragma unroll
            for (int j = 0; j < S::NB; ++j) w[j][e] = read(at + j * 2048, c, e);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < S::MB; ++i)
#pragma unroll
                for (int j = 0; j < S::NB; ++j) acc[i][j] = mfma_rows(x[i][e], w[j][e], acc[i][j]);
    }

    ATB_DEV void run()
    {
        const int end = (p.K + S::K - 1) / S::K;
        int k = wave, slot = 0;
        if (k < end) request(k, 0);
        if (k + S::W < end) request(k + S::W, 1);
        for (; k < end; k += S::W, slot ^= 1) {
            if (k + S::W < end) wait<S::REQS>();
            else wait<0>();
            multiply(slot);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the buffer is in registers
            if (k + 2 * S::W < end) request(k + 2 * S::W, slot);
        }
        __syncthreads();
    }
};

template <class S>
__global__ void __launch_bounds__(S::W * 64) stream_kernel(const StreamParams p)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS_BYTES];
    Stream<S> s(p, (unsigned)reinterpret_cast<uintptr_t>(lds));
    s.run();
    finish_rows<S::MB, S::NB, S::W, S::GATED>(p, s.acc, reinterpret_cast<float *>(lds), s.m0, s.n0, s.cols);
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
