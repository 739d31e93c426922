// The waves of the kernels for few rows with weights in bf16 (atb_stream.hip has how they work; also atb_moe.hip).
#pragma once

#include "atb_stream.h"

namespace atb {

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

// What a workgroup multiplies: the rows of x that belong to it and its columns of y, rows of the weights.
struct StreamView {
    const uint16_t *x;                         // x_rows rows of K, of which some are taken
    int64_t ldx;
    int x_rows, rows;                          // rows: how many are taken, 16 MB at most
    const void *w[2];                          // the first column's row; [1]: the up projection of a gated product
    int64_t ldw[2];
    int cols, K;
};

template <class S>
struct Stream {
    const int lane, c, q, wave;
    int K;
    unsigned ring;                             // LDS: this wave's two buffers
    Descriptor xd, wd[2];
    int x_off[S::XQ], w_off[S::NB][2];
    floatx4 acc[S::MB][S::NB];

    // Row i of the workgroup is row row_of(i) of x.
    template <class F>
    ATB_DEV Stream(const StreamView &v, unsigned lds, F row_of) : lane(threadIdx.x & 63), c(lane & 15), q(lane >> 4), wave(__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)), K(v.K)
    {
        ring = __builtin_amdgcn_readfirstlane(lds + wave * 2 * S::SLOT);
        open_rows(v, row_of);
#pragma unroll
        for (int g = 0; g < (S::GATED ? 2 : 1); ++g) {
            open_weight(v, g);
            const int64_t pitch = v.ldw[g] * 2;
#pragma unroll
            for (int j = g * S::COLS; j < (S::GATED ? (g + 1) * S::COLS : S::NB); ++j)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int col = 16 * (j - g * S::COLS) + 8 * r + lane / 8;
                    w_off[j][r] = col < v.cols ? col * (int)pitch + chunk() * 16 : kOutside;
                }
        }
        clear();
    }
    ATB_DEV void clear()
    {
#pragma unroll
        for (int i = 0; i < S::MB; ++i)
#pragma unroll
            for (int j = 0; j < S::NB; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // a request: lane l asks for the chunk of 16 bytes that the swizzle keeps at place l of its 8 rows of 128 bytes; rows outside ask for nothing
    template <class F>
    ATB_DEV void open_rows(const StreamView &v, F row_of)
    {
        xd = {reinterpret_cast<const char *>(v.x), ((int64_t)(v.x_rows - 1) * v.ldx + K) * 2};
#pragma unroll
        for (int i = 0; i < S::XQ; ++i) {
            const int row = 8 * i + lane / 8;
            x_off[i] = row < v.rows ? row_of(row) * (int)(v.ldx * 2) + chunk() * 16 : kOutside;
        }
    }
    ATB_DEV void open_weight(const StreamView &v, int g) { wd[g] = {static_cast<const char *>(v.w[g]), (v.cols - 1) * (v.ldw[g] * 2) + K * 2}; }

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
        const bool live = chunk() * 8 < K - panel * S::K;
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
        const int end = (K + S::K - 1) / S::K;
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

}  // namespace atb
