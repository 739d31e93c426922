// bf16 products in tiles: the kernel behind the gated block and its gradients (atb_ffn.hip, atb_ffn_grad.hip), and behind products with an epilogue and their gradients (atb_linear.hip, atb_linear_pair.hip).
//
// C tile = A tile x B tile with fp32 accumulation in MFMA accumulators, in K-steps of 64.  The tiles of a K-step come straight from memory into
// LDS: three buffers for A and two for B, all of a CU's 160 KiB.  An operand whose reduction index is contiguous lies in LDS as rows of 64 k (128
// bytes) and is read with plain 16-byte reads; one whose other index is contiguous lies there as 64 rows of k and is read through
// the transposing read, so no operand of the backward pass is ever transposed in memory.
//
// Time line of K-step s (the fragments of its first k-slice of 32 are in registers):
//   first half    the MFMAs of k-slice 0; the fragments of k-slice 1 are read under them
//   barrier       every wave has all of tile s in registers, so its buffers are free, and tile s + 1 is complete
//   second half   the MFMAs of k-slice 1; B's tile s + 2 and A's tile s + 3 are asked for, and the fragments of k-slice 0 of tile s + 1 are read
// so no MFMA behind the barrier waits for LDS, and A's tile s + 2 is still on its way at the barrier.
// Where there are fewer tiles than CUs a workgroup takes a share of the reduction (choose_tiles).
//
// Bound: the path by which requests come into a CU (64 KiB a K-step, 30 to 40 GB/s each in the products below; without requests a K-step takes 59 % of its time, without MFMAs
// 94 %), then power.
// Measured, M = 8192, D = 4096, F = 14336: gated 1624 us, 1185 TFLOP/s; down 739, 1302; dh with its epilogue 975, 986; dx 1476, 1304; the gradients of
// the gate and up weights 1540, 1249, of the down weight 898, 1072 (3.5 rounds of tiles).  (From box to box 2 %.)
//
// Rounded to bf16 are, beside the results, the operands of the products that follow: h, dg and du.  Their MFMAs take no other type at this rate; with three terms
// in the place of one an operand in two halves would keep 16 bits.  y and the gradients are 2.4e-3 off in the 2-norm, 1.7e-3 of it the results' rounding.
#pragma once

#include "atb_activation.h"
#include "atb_layers.h"

namespace atb {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

template <int TM_, int TN_, int WM_, int WN_>
struct TileShape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_;       // tile, wave grid
    static constexpr int NT = WM * WN * 64;
    static constexpr int TK = 64;
    static constexpr int MI = TM / WM / 16, NI = TN / WN / 16;         // 16 x 16 blocks of a wave
    static constexpr int A_BYTES = TM * TK * 2, B_BYTES = TN * TK * 2;
    static constexpr int LDS_BYTES = 3 * A_BYTES + 2 * B_BYTES;
    static constexpr int RA = A_BYTES / 16 / NT, RB = B_BYTES / 16 / NT;   // requests per thread and tile
    static_assert(TN / WN == 64, "a wave's columns: 64, of a gated product 32 of each weight");
    static_assert(RA * NT * 16 == A_BYTES && RB * NT * 16 == B_BYTES, "whole requests");
};

// Where a thread's requests for a tile of an operand read.  R: rows (or, with ROWS, columns) of the operand in the tile.  A request covers as
// many rows of LDS in every turn, so request i reads `pitch` bytes behind request i - 1.
// ROWS: 64 rows of k; chunk c (16 bytes) of row k lies at c ^ swizzle(k), so that the rows that a transposing read touches fall into different banks
// (per 32 lanes the rows k0 .. k0 + 3 and k0 + 8 .. k0 + 11 of 16 columns).  Otherwise rows of 64 k; chunk c of row r lies at c ^ (r % 8).
template <int R, int NT, bool ROWS>
struct Requests {
    static constexpr int CPR = ROWS ? R / 8 : 8;          // chunks per LDS row
    static constexpr int STEP = NT / CPR;                 // LDS rows of a request
    static_assert(!ROWS || (R >= 128 && STEP % 16 == 0), "the swizzle repeats after 16 rows of 16 chunks or more");
    static_assert(ROWS || STEP % 8 == 0, "... and after 8");
    int first, pitch;

    static ATB_DEV int swizzle(int row) { return ROWS ? ((row & 3) << 2) | (((row >> 3) & 1) << 1) : row & 7; }
    static ATB_DEV int chunk(int tid) { return (tid % CPR) ^ swizzle(tid / CPR); }

    ATB_DEV void place(int tid, int64_t ld)
    {
        first = (tid / CPR) * (int)(ld * 2) + chunk(tid) * 16;
        pitch = __builtin_amdgcn_readfirstlane(STEP * (int)(ld * 2));
    }
    // (by hand: worked out ahead of the K loop, as the compiler would, it holds a register for the whole kernel)
    template <int i>
    ATB_DEV int added() const
    {
        int r = 0;
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("v_add_u32 %0, %1, %2" : "=v"(r) : "s"(i * pitch), "v"(first));
#endif
        return r;
    }
    // Request i of a tile with k_left of the reduction from its first k on.  What follows the end of a row of K-contiguous elements is the next row's,
    // so the lanes of chunks behind it ask for nothing (K % 8 == 0: a chunk is inside or outside): an offset past the end of every descriptor, which
    // reads as zero.  Rows of k end with the operand.
    template <int i>
    ATB_DEV int offset(int tid, int k_left) const
    {
        int at = first;
        if constexpr (i > 0) at = added<i>();
        if constexpr (ROWS) return at;
        return chunk(tid) * 8 >= k_left ? (int)0x80000000 : at;
    }
};

// A descriptor's four dwords, advanced by whole K-steps.
struct Source {
    const char *ptr;
    int64_t left;          // bytes from ptr to the end of the operand
    ATB_DEV void move(int64_t step, bool more)
    {
        ptr += step;
        left = more ? left - step : 0;
    }
    ATB_DEV intx4 words() const
    {
        const uint64_t a = reinterpret_cast<uint64_t>(ptr);
        const int64_t n = left < 0 ? 0 : left > 0x7fffffff ? 0x7fffffff : left;
        return intx4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF),
                     __builtin_amdgcn_readfirstlane((int)n), kRsrcFlags};
    }
};

template <class S, bool AT, bool BROWS, int EPI>
struct Tile {
    static constexpr bool GATED = is_gated(EPI);
    const TileParams &p;
    const int tid, lane, wave, wm, wn;
    int m0, n0, problem;
    typedef Requests<S::TM, S::NT, AT> ARequests;
    typedef Requests<S::TN, S::NT, BROWS> BRequests;
    ARequests a_off;
    BRequests b_off, b2_off;
    Source a_src, b_src, b2_src;           // b2: the up weight of a gated product
    int64_t a_step, b_step;                // bytes of a K-step
    int a_left, b_left;                    // reduction left to ask for
    int steps;                             // K-steps
    unsigned a_rd, b_rd;                   // LDS addresses: this lane's part of a fragment in the first buffer
    unsigned a_req, b_req;                 // ... this wave's part of a request
    int slot;                              // A's buffer of the tile that is multiplied: its offset
    floatx4 acc[S::MI][S::NI];
    bf16x8 af[2][S::MI], bf[2][S::NI];

    ATB_DEV Tile(const TileParams &p_, char *lds, int m0_, int n0_, int problem_)
        : p(p_), tid(threadIdx.x), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)), wm(wave / S::WN), wn(wave % S::WN),
          m0(m0_), n0(n0_), problem(problem_)
    {
        const unsigned a_lds = (unsigned)reinterpret_cast<uintptr_t>(lds), b_lds = a_lds + 3 * S::A_BYTES;
        a_req = __builtin_amdgcn_readfirstlane(a_lds + wave * 1024);
        b_req = __builtin_amdgcn_readfirstlane(b_lds + wave * 1024);
        a_rd = AT ? rows_address<S::TM>(a_lds, wm * (S::TM / S::WM)) : k_address(a_lds, wm * (S::TM / S::WM));
        b_rd = BROWS ? rows_address<S::TN>(b_lds, wn * 64) : k_address(b_lds, wn * (GATED ? 32 : 64));
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int j = 0; j < S::NI; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Rows of 64 k: lane l reads row l % 16 of a block of 16 and the 8 k of group l / 16 of a k-slice: chunk l / 16 or, of the second, four on.
    ATB_DEV unsigned k_address(unsigned base, int first) const
    {
        const int row = first + (lane & 15);
        return base + row * 128 + (((lane >> 4) ^ (row & 7)) * 16);
    }
    // Rows of k, the transposing read of 16 columns and 8 k: in a group of 16 lanes, lane i addresses columns 4 (i % 4) .. + 3 of row i / 4 and lane j
    // receives column j of the four rows; group g takes rows 8 g .. 8 g + 3 of the k-slice, a second read 4 rows on the others.  (The next 16 columns are
    // two chunks on: the address with 32 added to the bits that the swizzle has been applied to, which are no others' here.)
    template <int R>
    ATB_DEV unsigned rows_address(unsigned base, int first) const
    {
        const int j = lane & 15, row = 8 * (lane >> 4) + (j >> 2), chunk = first / 8 + ((j & 3) >> 1);
        return base + row * (R * 2) + ((chunk ^ Requests<R, S::NT, true>::swizzle(row)) * 16) + (j & 1) * 8;
    }

    // ---- requests

    // Bytes from an operand's element (row, col) to its end; rows of `cols` elements, ld apart.
    // (in whole dwords, as a request checks them: what is odd here has rows that are padded to multiples of 8)
    static ATB_DEV int64_t bytes_left(int64_t rows, int64_t cols, int64_t ld, int64_t row, int64_t col) { return (((rows - 1 - row) * ld + cols - col) * 2 + 3) & ~(int64_t)3; }

    // The operands s: a segment of the reduction, or a problem; K-steps first .. end - 1 of it.
    ATB_DEV void open(int s, int first, int end)
    {
        const int k0 = first * S::TK;
        steps = end - first;
        a_left = b_left = min(p.K, end * S::TK) - k0;
        a_step = AT ? S::TK * 2 * p.lda[s] : S::TK * 2;
        b_step = BROWS ? S::TK * 2 * p.ldb[s] : S::TK * 2;
        Source a, b, up = {};
        if constexpr (AT) a = {reinterpret_cast<const char *>(p.A[s] + k0 * p.lda[s] + m0), bytes_left(p.K, p.M, p.lda[s], k0, m0)};
        else a = {reinterpret_cast<const char *>(p.A[s] + m0 * p.lda[s] + k0), bytes_left(p.M, p.K, p.lda[s], m0, k0)};
        a_off.place(tid, p.lda[s]);
        if constexpr (GATED) {
            // rows 0 .. TN / 2 - 1 of the LDS tile are columns of the gate weight, the others the same columns of the up weight
            b = {reinterpret_cast<const char *>(p.B[0] + n0 * p.ldb[0] + k0), bytes_left(p.N, p.K, p.ldb[0], n0, k0)};
            up = {reinterpret_cast<const char *>(p.B[1] + n0 * p.ldb[1] + k0), bytes_left(p.N, p.K, p.ldb[1], n0, k0)};
            b_off.place(tid, p.ldb[0]);
            b2_off.place(tid, p.ldb[1]);
        } else {
            if constexpr (BROWS) b = {reinterpret_cast<const char *>(p.B[s] + k0 * p.ldb[s] + n0), bytes_left(p.K, p.N, p.ldb[s], k0, n0)};
            else b = {reinterpret_cast<const char *>(p.B[s] + n0 * p.ldb[s] + k0), bytes_left(p.edge, p.K, p.ldb[s], n0, k0)};
            b_off.place(tid, p.ldb[s]);
        }
        a_src = a;
        b_src = b;
        b2_src = up;
    }

    // 16 bytes per lane from memory to LDS.  By hand, so that the compiler does not wait for it before every read of LDS that follows; the wait is
    // the one ahead of the barrier.  M0, the LDS address, is put back: the compiler is not told about it.
    static ATB_DEV void request_one(intx4 words, int off, unsigned to)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        int saved;
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved)
                     : "s"(to), "v"(off), "s"(words) : "memory");
#endif
    }

    // Request r of A's next tile into the buffer at `to`, of B's into its buffer `buf`.  After a tile's last one the stream moves on by a K-step; past the
    // last K-step its descriptor is empty and nothing is asked of memory.
    template <int r>
    ATB_DEV void request_a(int to)
    {
        request_one(a_src.words(), a_off.template offset<r>(tid, a_left), a_req + to + r * S::NT * 16);
        if constexpr (r == S::RA - 1) {
            a_left -= S::TK;
            a_src.move(a_step, a_left > 0);
        }
    }
    template <int r, int buf>
    ATB_DEV void request_b()
    {
        const unsigned to = b_req + buf * S::B_BYTES + r * S::NT * 16;
        if constexpr (GATED && r >= S::RB / 2) request_one(b2_src.words(), b2_off.template offset<r - S::RB / 2>(tid, b_left), to);
        else request_one(b_src.words(), b_off.template offset<r>(tid, b_left), to);
        if constexpr (r == S::RB - 1) {
            b_left -= S::TK;
            b_src.move(b_step, b_left > 0);
            if constexpr (GATED) b2_src.move(b_step, b_left > 0);
        }
    }
    template <int r = 0>
    ATB_DEV void request_all_a(int to)
    {
        if constexpr (r < S::RA) {
            request_a<r>(to);
            request_all_a<r + 1>(to);
        }
    }
    template <int buf, int r = 0>
    ATB_DEV void request_all_b()
    {
        if constexpr (r < S::RB) {
            request_b<r, buf>();
            request_all_b<buf, r + 1>();
        }
    }
    static constexpr int REQS = S::RA + S::RB;

    // ---- LDS -> registers

    template <int R>
    static ATB_DEV bf16x8 read_rows(unsigned at)
    {
        bf16x8 r = {};
#if defined(__HIP_DEVICE_COMPILE__)
        typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
        union { shortx4 s[2]; bf16x8 b; } u;
        u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)at);
        u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at + 4 * R * 2));
        r = u.b;
#endif
        return r;
    }
    static ATB_DEV bf16x8 read_k(unsigned at)
    {
        bf16x8 r = {};
#if defined(__HIP_DEVICE_COMPILE__)
        r = *(const __attribute__((address_space(3))) bf16x8 *)at;
#endif
        return r;
    }
    // Fragment f of k-slice ks of the tile in A's buffer at `from` and B's buffer `buf`, in the order of first use: a0, b0 .. b(NI - 1), a1 .. a(MI - 1)
    template <int ks, int buf, int f>
    ATB_DEV void read_frag(int from)
    {
        if constexpr (f >= 1 && f <= S::NI) {
            constexpr int j = f - 1;
            if constexpr (BROWS) bf[ks][j] = read_rows<S::TN>((b_rd ^ (j * 32)) + buf * S::B_BYTES + ks * 32 * S::TN * 2);
            else bf[ks][j] = read_k((b_rd ^ (ks * 64)) + buf * S::B_BYTES + (GATED && j >= 2 ? S::TN / 2 * 128 + (j - 2) * 2048 : j * 2048));
        } else {
            constexpr int i = f == 0 ? 0 : f - S::NI;
            if constexpr (AT) af[ks][i] = read_rows<S::TM>(((a_rd + from) ^ (i * 32)) + ks * 32 * S::TM * 2);
            else af[ks][i] = read_k(((a_rd + from) ^ (ks * 64)) + i * 2048);
        }
    }
    static constexpr int FRAGS = S::MI + S::NI;
    template <int ks, int buf, int f = 0>
    ATB_DEV void read_all(int from)
    {
        if constexpr (f < FRAGS) {
            read_frag<ks, buf, f>(from);
            read_all<ks, buf, f + 1>(from);
        }
    }

    // ---- half a K-step: MI x NI MFMAs and their side work

    static constexpr int SLOTS = S::MI * S::NI;
    template <int ks, int t>
    ATB_DEV void mfma()
    {
#if defined(__HIP_DEVICE_COMPILE__)
        acc[t / S::NI][t % S::NI] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[ks][t % S::NI], af[ks][t / S::NI], acc[t / S::NI][t % S::NI], 0, 0, 0);
#endif
    }
    template <int buf, int t = 0>
    ATB_DEV void first_half()
    {
        if constexpr (t < SLOTS) {
            mfma<0, t>();
            constexpr int every = SLOTS >= 2 * FRAGS ? 2 : 1;
            if constexpr (t % every == 0 && t / every < FRAGS) read_frag<1, buf, t / every>(slot);
            __builtin_amdgcn_sched_barrier(0);
            first_half<buf, t + 1>();
        }
    }
    template <int buf, int t = 0>
    ATB_DEV void second_half(int next)
    {
        if constexpr (t < SLOTS) {
            mfma<1, t>();
            constexpr int per = (FRAGS + REQS + SLOTS - 1) / SLOTS;
            side_work<buf, t * per, t * per + per>(next);
            __builtin_amdgcn_sched_barrier(0);
            second_half<buf, t + 1>(next);
        }
    }
    // requests, B's first, and reads in turns
    template <int buf, int n, int end>
    ATB_DEV void side_work(int next)
    {
        static_assert(REQS <= FRAGS, "reads are what is left");
        if constexpr (n < end) {
            if constexpr (n < 2 * REQS && n % 2 == 0) {
                if constexpr (n / 2 < S::RB) request_b<n / 2, buf>();
                else request_a<n / 2 - S::RB>(slot);
            } else if constexpr (n < FRAGS + REQS) {
                read_frag<0, buf ^ 1, n < 2 * REQS ? n / 2 : n - REQS>(next);
            }
            side_work<buf, n + 1, end>(next);
        }
    }

    // The `younger` most recent requests of this wave may be on their way; its reads of LDS are done, and so are those of all waves after it.
    template <int younger>
    static ATB_DEV void wait_and_barrier()
    {
        static_assert(younger >= 0 && younger < 64, "vmcnt is a 6-bit counter");
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(younger) : "memory");
    }

    template <int buf>
    ATB_DEV void step()
    {
        first_half<buf>();
        wait_and_barrier<S::RA>();
        const int next = slot == 2 * S::A_BYTES ? 0 : slot + S::A_BYTES;
        second_half<buf>(next);
        slot = next;
    }

    ATB_DEV void multiply_segment()
    {
        request_all_a(0);
        request_all_b<0>();
        request_all_a(S::A_BYTES);
        request_all_b<1>();
        request_all_a(2 * S::A_BYTES);
        wait_and_barrier<2 * S::RA + S::RB>();
        slot = 0;
        read_all<0, 0>(0);
        for (int s = 0; s < steps; s += 2) {
            step<0>();
            if (s + 1 == steps) break;
            step<1>();
        }
        wait_and_barrier<0>();                                 // LDS is free again
    }

    // K-steps first .. end - 1 of the whole reduction.  Segments one after the other: the few requests in flight are awaited in between.
    ATB_DEV void multiply(int first, int end)
    {
        const int all = p.steps;
        for (int s = 0; s < p.segments; ++s) {
            const int from = max(first - s * all, 0), to = min(end - s * all, all);
            if (from >= to) continue;
            open(p.segments > 1 ? s : problem, from, to);
            multiply_segment();
        }
    }
    // x, which the compiler is not to know ahead of this place: it would work out the addresses of the whole tile before the first store
    static ATB_DEV int here(int x)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(x));
#endif
        return x;
    }
    // An element of an accumulator, likewise: of elements, or their bits, the compiler makes values that it carries round the K loop beside the accumulators
    static ATB_DEV float sum(float x)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(x));
#endif
        return x;
    }
    static ATB_DEV unsigned bits(float x) { return __float_as_uint(sum(x)); }

    // ---- epilogue: a lane holds row 16 i + lane % 16 of the wave's part and, of column block j, columns 4 (lane / 16) .. + 3.  One swap of
    // lanes per register makes of two neighbouring column blocks eight consecutive columns per lane.

    static ATB_DEV void swap_halves(unsigned &x, unsigned &y)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        const uintx2 r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
        x = r.x;
        y = r.y;
#endif
    }
    ATB_DEV int piece_col() const { return ((lane >> 4) & 1) * 16 + (lane >> 5) * 8; }

    static ATB_DEV unsigned pack(float a, float b)
    {
        union { bf16x2 v; unsigned w; } u;
        u.v = bf16x2{(__bf16)a, (__bf16)b};
        return u.w;
    }
    // column blocks x, y of a row block -> this lane's eight columns as bf16
    static ATB_DEV intx4 piece(const floatx4 &x, const floatx4 &y)
    {
        unsigned a0 = pack(x[0], x[1]), a1 = pack(x[2], x[3]), b0 = pack(y[0], y[1]), b1 = pack(y[2], y[3]);
        swap_halves(a0, b0);
        swap_halves(a1, b1);
        return intx4{(int)a0, (int)a1, (int)b0, (int)b1};
    }
    // (rows of C begin at multiples of 16 bytes: N, the pitch and the pointer are multiples of 8 elements)
    ATB_DEV void store(uint16_t *c, int64_t ld, int row, int col, intx4 v) const
    {
        if (row < p.M && col < p.N) *reinterpret_cast<intx4 *>(c + (int64_t)row * ld + col) = v;
    }

    // g and u as the backward pass needs them, 24 of their 32 bits (16 of the mantissa): plane 0 has the upper 16 of g, plane 1 those of u, plane 2 the next byte
    // of g and, above it, of u.  In bf16, 16 bits each, their rounding makes as large a part of the error of dx and the weights' gradients as the
    // rounding of dg and du and that of the result (3.1e-3 in the 2-norm instead of 2.4e-3).
    static ATB_DEV unsigned bytes(unsigned hi, unsigned lo, unsigned select)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        return __builtin_amdgcn_perm(hi, lo, select);
#else
        return 0;
#endif
    }
    ATB_DEV void keep(int row, int col, const floatx4 &g0, const floatx4 &g1, const floatx4 &u0, const floatx4 &u1) const
    {
        unsigned w[3][2][2];            // plane, column block, pair of columns
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const floatx4 &g = b ? g1 : g0, &u = b ? u1 : u0;
                const unsigned ga = bits(g[2 * e]), gb = bits(g[2 * e + 1]), ua = bits(u[2 * e]), ub = bits(u[2 * e + 1]);
                w[0][b][e] = bytes(gb, ga, 0x07060302u);
                w[1][b][e] = bytes(ub, ua, 0x07060302u);
                w[2][b][e] = bytes(bytes(ub, gb, 0x0c0c0501u), bytes(ua, ga, 0x0c0c0501u), 0x05040100u);
            }
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            swap_halves(w[n][0][0], w[n][1][0]);
            swap_halves(w[n][0][1], w[n][1][1]);
            store(p.kept + n * ((int64_t)p.M * p.N), p.N, row, col, intx4{(int)w[n][0][0], (int)w[n][0][1], (int)w[n][1][0], (int)w[n][1][1]});
        }
    }
    // The three words of a piece (of the last row or column in place of one outside), and g and u from them
    ATB_DEV void load_kept(int row, int col, intx4 (&w)[3]) const
    {
        const uint16_t *at = p.kept + (int64_t)min(row, p.M - 1) * p.N + min(col, p.N - 8);
#pragma unroll
        for (int n = 0; n < 3; ++n) w[n] = *reinterpret_cast<const intx4 *>(at + n * ((int64_t)p.M * p.N));
    }
    static ATB_DEV void kept(const intx4 (&w)[3], float (&g)[8], float (&u)[8])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned gh = (unsigned)w[0][e], uh = (unsigned)w[1][e], lo = (unsigned)w[2][e];
            g[2 * e] = __uint_as_float(bytes(gh, lo, 0x0504000cu));
            g[2 * e + 1] = __uint_as_float(bytes(gh, lo, 0x0706020cu));
            u[2 * e] = __uint_as_float(bytes(uh, lo, 0x0504010cu));
            u[2 * e + 1] = __uint_as_float(bytes(uh, lo, 0x0706030cu));
        }
    }

    ATB_DEV void finish_plain()
    {
        const int row0 = m0 + wm * (S::TM / S::WM) + (lane & 15), col0 = n0 + wn * 64 + piece_col();
        uint16_t *c = p.C[problem];
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int j = 0; j < S::NI; j += 2) store(c, p.ldc, row0 + 16 * i, col0 + 16 * j, piece(acc[i][j], acc[i][j + 1]));
    }

    ATB_DEV void finish_gated()
    {
        const int row0 = m0 + wm * (S::TM / S::WM) + (lane & 15), col = n0 + wn * 32 + piece_col();
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            const int row = here(row0 + 16 * i);
            if constexpr (EPI == kGatedKeep) keep(row, col, acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
            floatx4 h[2], g[2], u[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    g[j][e] = sum(acc[i][j][e]);
                    u[j][e] = sum(acc[i][j + 2][e]);
                }
            with_activation(p.act, [&](auto a) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[j][e] = activate<decltype(a)::value>(g[j][e]) * u[j][e];
            });
            store(p.C[0], p.ldc, row, col, piece(h[0], h[1]));
            __builtin_amdgcn_sched_barrier(0);             // row block by row block: registers
        }
    }

    // Pieces of eight columns, AHEAD of them on their way (one by one the 16 of a wave took 33 us of latency, a quarter of a tile of K = 4096)
    ATB_DEV void finish_grad()
    {
        constexpr int PIECES = S::MI * S::NI / 2, AHEAD = 6;
        const int row0 = m0 + wm * (S::TM / S::WM) + (lane & 15), col0 = n0 + wn * 64 + piece_col();
        intx4 w[AHEAD][3];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) load_kept(row0 + 16 * (n / (S::NI / 2)), col0 + 32 * (n % (S::NI / 2)), w[n]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < PIECES; ++n) {
            const int i = n / (S::NI / 2), j = 2 * (n % (S::NI / 2));
            const int row = here(row0 + 16 * i), col = col0 + 16 * j;
            float d[8];                                    // dh of this lane's eight columns
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                unsigned x = bits(acc[i][j][e]), y = bits(acc[i][j + 1][e]);
                swap_halves(x, y);
                d[e] = __uint_as_float(x);
                d[4 + e] = __uint_as_float(y);
            }
            float g[8], u[8];
            kept(w[n % AHEAD], g, u);
            bf16x8 dg, du;
            with_activation(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float a, slope;
                    activate_grad<decltype(act)::value>(g[e], a, slope);
                    dg[e] = (__bf16)(d[e] * u[e] * slope);
                    du[e] = (__bf16)(d[e] * a);
                }
            });
            if (row < p.M && col < p.N) {
                const int64_t to = (int64_t)row * p.ldc + col;
                *reinterpret_cast<bf16x8 *>(p.C[0] + to) = dg;
                *reinterpret_cast<bf16x8 *>(p.C[1] + to) = du;
            }
            if (n + AHEAD < PIECES) load_kept(here(row0 + 16 * ((n + AHEAD) / (S::NI / 2))), col0 + 32 * ((n + AHEAD) % (S::NI / 2)), w[n % AHEAD]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // ---- the epilogue of a product: act(sum + bias) + residual, in pieces of eight columns.  The residual's are all asked for ahead of the first store: a wait for a load is one for the stores before it too (6061 x
    // 9088 x 440 with residual and slope, four pieces ahead 159 us, where either alone took 102).  Rows of C and residual begin at any element, and their last piece may be cut; the slope's are padded to multiples of 8.

    // Columns col .. col + 7 of a row of p.edge; 0 past its end
    template <class T>
    ATB_DEV void load_eight(const T *row, int col, float (&v)[8]) const
    {
        typedef T vec __attribute__((ext_vector_type(8)));
        typedef vec any __attribute__((aligned(sizeof(T))));
        if (col + 8 <= p.edge) {
            const vec w = *reinterpret_cast<const any *>(row + col);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)w[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = col + e < p.edge ? (float)row[col + e] : 0.0f;
        }
    }
    typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
    ATB_DEV bf16x8 load_residual(int row, int col) const
    {
        bf16x8 w = {};
        const __bf16 *at = reinterpret_cast<const __bf16 *>(p.residual) + min(row, p.M - 1) * p.ldr;
        if (col + 8 <= p.edge) {
            w = *reinterpret_cast<const bf16x8_any *>(at + col);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < p.edge) w[e] = at[col + e];
        }
        return w;
    }
    template <class T>
    ATB_DEV void store_eight(T *row, int col, const float (&v)[8]) const
    {
        typedef T vec __attribute__((ext_vector_type(8)));
        typedef vec any __attribute__((aligned(2)));
        if (col + 8 <= p.edge) {
            vec w;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = (T)v[e];
            *reinterpret_cast<any *>(row + col) = w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < p.edge) row[col + e] = (T)v[e];
        }
    }

    ATB_DEV void finish_linear()
    {
        constexpr int PIECES = S::MI * S::NI / 2;
        const int row0 = m0 + wm * (S::TM / S::WM) + (lane & 15), col0 = n0 + wn * 64 + piece_col();
        bf16x8 res[PIECES] = {};
        if (p.residual) {
#pragma unroll
            for (int n = 0; n < PIECES; ++n) res[n] = load_residual(here(row0 + 16 * (n / (S::NI / 2))), col0 + 32 * (n % (S::NI / 2)));
        }
        float bias[S::NI / 2][8] = {};
        if (p.bias) {
#pragma unroll
            for (int j = 0; j < S::NI / 2; ++j) {
                if (p.bias_type == ATB_TYPE_F32) load_eight(static_cast<const float *>(p.bias), col0 + 32 * j, bias[j]);
                else load_eight(static_cast<const __bf16 *>(p.bias), col0 + 32 * j, bias[j]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int pitch = (p.edge + 7) & ~7;
#pragma unroll
        for (int n = 0; n < PIECES; ++n) {
            const int i = n / (S::NI / 2), j = n % (S::NI / 2);
            const int row = here(row0 + 16 * i), col = col0 + 32 * j;
            float v[8], slope[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                unsigned x = bits(acc[i][2 * j][e]), y = bits(acc[i][2 * j + 1][e]);
                swap_halves(x, y);
                v[e] = __uint_as_float(x) + bias[j][e];
                v[4 + e] = __uint_as_float(y) + bias[j][4 + e];
            }
            if constexpr (EPI == kLinearKeep) {
                with_activation(p.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) activate_grad<decltype(act)::value>(v[e], v[e], slope[e]);
                });
            } else {
                with_activation_or_none(p.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = activate<decltype(act)::value>(v[e]);
                });
            }
            if (p.residual) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += (float)res[n][e];
            }
            if (row < p.M) {
                store_eight(reinterpret_cast<__bf16 *>(p.C[0]) + (int64_t)row * p.ldc, col, v);
                if constexpr (EPI == kLinearKeep) {
                    typedef _Float16 half8 __attribute__((ext_vector_type(8)));
                    half8 w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = (_Float16)slope[e];
                    if (col < pitch) *reinterpret_cast<half8 *>(p.slope + (int64_t)row * pitch + col) = w;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // A share of the sums, in fp32: plane 0 has the gate's or the (first problem's) sums, plane 1 the up projection's or the second problem's
    ATB_DEV void finish_share(int share)
    {
        const int row0 = m0 + wm * (S::TM / S::WM) + (lane & 15), cols = GATED ? 32 : 64, col0 = n0 + wn * cols + 4 * (lane >> 4);
        const int64_t plane = (int64_t)p.M * p.N;
        float *to = p.shares + (int64_t)share * p.planes * plane + (GATED ? 0 : problem * plane);
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            const int row = row0 + 16 * i;
#pragma unroll
            for (int j = 0; j < S::NI; ++j) {
                const int col = col0 + 16 * (j % (cols / 16));
                if (row < p.M && col < p.N) *reinterpret_cast<floatx4 *>(to + (GATED && j >= 2 ? plane : 0) + (int64_t)row * p.N + col) = acc[i][j];
            }
        }
    }

    ATB_DEV void finish(int share)
    {
        if constexpr (is_share(EPI)) finish_share(share);
        else if constexpr (EPI == kStore) finish_plain();
        else if constexpr (is_linear(EPI)) finish_linear();
        else if constexpr (EPI == kGatedGrad) finish_grad();
        else finish_gated();
    }
};

// Tile and share of workgroup b: workgroups are dealt round-robin to the 8 XCDs, each with an L2 of its own; XCD x takes a contiguous run of the
// tiles of one share after the other, walked in bands of group_m tile rows, so that those resident on it share rows of A and columns of B.
template <class S, bool GATED>
ATB_DEV bool tile_of(const TileParams &p, int b, int &m0, int &n0, int &share)
{
    const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.parts, per_xcd = (total + 7) / 8;
    int t = (b % 8) * per_xcd + b / 8;
    if (b / 8 >= per_xcd || t >= total) return false;
    share = t / tiles;
    t -= share * tiles;
    const int band_size = p.group_m * p.tiles_n, band = t / band_size, in_band = t % band_size;
    const int rows = min(p.group_m, p.tiles_m - band * p.group_m);
    m0 = (band * p.group_m + in_band % rows) * S::TM;
    n0 = (in_band / rows) * (GATED ? S::TN / 2 : S::TN);
    return true;
}

template <class S, bool AT, bool BROWS, int EPI>
__global__ void __launch_bounds__(S::NT, 2) tile_kernel(const TileParams p)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS_BYTES];
    int m0 = 0, n0 = 0, share = 0;
    if (!tile_of<S, is_gated(EPI)>(p, blockIdx.x, m0, n0, share)) return;
    Tile<S, AT, BROWS, EPI> tile(p, lds, m0, n0, blockIdx.y);
    const int all = p.steps * p.segments;
    if constexpr (is_share(EPI)) tile.multiply((int)((int64_t)share * all / p.parts), (int)((int64_t)(share + 1) * all / p.parts));
    else tile.multiply(0, all);
    tile.finish(share);
}

// The shares of a tile's sums, added in order, and the epilogue: four columns per thread.  Bound: the bytes of the shares (two of 2048 x 4096 in 13.7 us, 6.1 TB/s).
template <int EPI>
__global__ void __launch_bounds__(256) join_kernel(const TileParams p)
{
    const int pieces = p.N / 4, at = blockIdx.x * 256 + threadIdx.x;
    if (at >= p.M * pieces) return;
    const int row = at / pieces, col = (at - row * pieces) * 4;
    const int64_t plane = (int64_t)p.M * p.N, place = (int64_t)row * p.N + col;
    constexpr int PLANES = is_gated(EPI) ? 2 : 1;
    const float *from = p.shares + place + blockIdx.y * plane;
    floatx4 sum[PLANES] = {};
#pragma unroll 4
    for (int s = 0; s < p.parts; ++s, from += p.planes * plane)
#pragma unroll
        for (int n = 0; n < PLANES; ++n) sum[n] += *reinterpret_cast<const floatx4 *>(from + n * plane);
    const int64_t to = (int64_t)row * p.ldc + col;
    if constexpr (is_linear(EPI)) {
        const int cols = min(4, p.edge - col);                 // (none or fewer where N is not a multiple of 8)
        float v[4], slope[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = sum[0][e];
            if (p.bias && e < cols) v[e] += p.bias_type == ATB_TYPE_F32 ? static_cast<const float *>(p.bias)[col + e] : (float)static_cast<const __bf16 *>(p.bias)[col + e];
        }
        if constexpr (EPI == kLinearKeep) {
            with_activation(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) activate_grad<decltype(act)::value>(v[e], v[e], slope[e]);
            });
        } else {
            with_activation_or_none(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = activate<decltype(act)::value>(v[e]);
            });
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < cols) {
                if (p.residual) v[e] += (float)reinterpret_cast<const __bf16 *>(p.residual)[row * p.ldr + col + e];
                reinterpret_cast<__bf16 *>(p.C[0])[to + e] = (__bf16)v[e];
                if constexpr (EPI == kLinearKeep) reinterpret_cast<_Float16 *>(p.slope)[(int64_t)row * ((p.edge + 7) & ~7) + col + e] = (_Float16)slope[e];
            }
    } else if constexpr (EPI == kStore) {
        bf16x4 c;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = (__bf16)sum[0][e];
        *reinterpret_cast<bf16x4 *>(p.C[blockIdx.y] + to) = c;
    } else if constexpr (EPI == kGatedGrad) {
        uintx2 w[3];
#pragma unroll
        for (int n = 0; n < 3; ++n) w[n] = *reinterpret_cast<const uintx2 *>(p.kept + n * plane + place);
        bf16x4 dg, du;
        with_activation(p.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned shift = 16 * (e & 1), gh = w[0][e / 2] >> shift, uh = w[1][e / 2] >> shift, lo = w[2][e / 2] >> shift;
                const float g = __uint_as_float(gh << 16 | (lo & 0xff) << 8), u = __uint_as_float(uh << 16 | (lo & 0xff00));
                float a, slope;
                activate_grad<decltype(act)::value>(g, a, slope);
                dg[e] = (__bf16)(sum[0][e] * u * slope);
                du[e] = (__bf16)(sum[0][e] * a);
            }
        });
        *reinterpret_cast<bf16x4 *>(p.C[0] + to) = dg;
        *reinterpret_cast<bf16x4 *>(p.C[1] + to) = du;
    } else {
        bf16x4 h;
        with_activation(p.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = (__bf16)(activate<decltype(act)::value>(sum[0][e]) * sum[PLANES - 1][e]);
        });
        *reinterpret_cast<bf16x4 *>(p.C[0] + to) = h;
        if constexpr (EPI == kGatedKeep) {
            uintx2 w[3] = {};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned shift = 16 * (e & 1), g = __float_as_uint(sum[0][e]), u = __float_as_uint(sum[PLANES - 1][e]);
                w[0][e / 2] |= g >> 16 << shift;
                w[1][e / 2] |= u >> 16 << shift;
                w[2][e / 2] |= ((g >> 8 & 0xff) | (u & 0xff00)) << shift;
            }
#pragma unroll
            for (int n = 0; n < 3; ++n) *reinterpret_cast<uintx2 *>(p.kept + n * plane + place) = w[n];
        }
    }
}

typedef TileShape<256, 256, 2, 4> Tile256;
typedef TileShape<128, 128, 2, 2> Tile128;
typedef TileShape<128, 256, 2, 4> Tile128x256;

template <class S, bool AT, bool BROWS, int EPI>
hipError_t launch_shape(TileParams &p, hipStream_t stream)
{
    p.tiles_m = tile_plan(p.M, p.N, S::TM, is_gated(EPI)).tiles_m;
    p.tiles_n = tile_plan(p.M, p.N, S::TN, is_gated(EPI)).tiles_n;
    p.group_m = 2048 / S::TM;
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n * p.parts;
    if (total > 0xffffff00u / S::NT) return hipErrorInvalidConfiguration;      // 2^32 threads: a result of 2^36 elements or more
    hipLaunchKernelGGL((tile_kernel<S, AT, BROWS, EPI>), dim3((unsigned)((total + 7) / 8 * 8), p.problems), dim3(S::NT), 0, stream, p);
    return hipGetLastError();
}

template <bool AT, bool BROWS, int EPI>
hipError_t launch_tiles(TileParams &p, hipStream_t stream)
{
    const TileChoice how = choose_tiles(p.M, p.N, p.K, p.segments, p.problems, is_gated(EPI), p.shares != nullptr, is_linear(EPI));
    p.steps = (p.K + 63) / 64;
    p.planes = is_gated(EPI) ? 2 : p.problems;
    if (p.edge == 0) p.edge = p.N;
    p.parts = how.parts;
    constexpr int SHARE = is_gated(EPI) ? kGatedShare : kShare;
    if constexpr (is_linear(EPI))
        if (how.wide) return launch_shape<Tile128x256, AT, BROWS, EPI>(p, stream);
    if (p.parts == 1) return how.large ? launch_shape<Tile256, AT, BROWS, EPI>(p, stream) : launch_shape<Tile128, AT, BROWS, EPI>(p, stream);
    hipError_t e;
    if constexpr (is_gated(EPI)) e = launch_shape<Tile128, AT, BROWS, SHARE>(p, stream);           // (their shares are never large tiles)
    else e = how.large ? launch_shape<Tile256, AT, BROWS, SHARE>(p, stream) : launch_shape<Tile128, AT, BROWS, SHARE>(p, stream);
    if (e != hipSuccess) return e;
    const int64_t threads = (int64_t)p.M * (p.N / 4);          // (few tiles: far below 2^31)
    hipLaunchKernelGGL((join_kernel<EPI>), dim3((unsigned)((threads + 255) / 256), p.problems), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace atb
