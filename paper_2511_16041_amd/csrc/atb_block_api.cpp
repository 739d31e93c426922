// C ABI of what a block has around its feed-forward sublayer (see include/atb.h): argument checking and launches.
#include "atb_block.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 23, kMaxPitch = (int64_t)1 << 22;

using atb::hip_status;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool is_type(atb_type t) { return t == ATB_TYPE_BF16 || t == ATB_TYPE_F32; }
bool is_activation(atb_activation a) { return a == ATB_ACT_SILU || a == ATB_ACT_GELU || a == ATB_ACT_GELU_TANH; }
uintptr_t size_of(atb_type t) { return t == ATB_TYPE_F32 ? 4 : 2; }

// A bf16 matrix that the tile kernels read in 16-byte pieces
bool is_matrix(const void *p, int64_t cols, int64_t ld) { return p && aligned(p, 16) && ld >= cols && ld % 8 == 0 && ld < kMaxPitch; }
// ... and one whose rows begin at any element
bool is_rows(const void *p, int64_t cols, int64_t ld, uintptr_t size) { return p && aligned(p, size) && ld >= cols; }

const uint16_t *u16(const void *p) { return static_cast<const uint16_t *>(p); }
uint16_t *u16(void *p) { return static_cast<uint16_t *>(p); }

// ------------------------------------------------------------------ a product with its epilogue

bool linear_lengths(int64_t M, int64_t N, int64_t K)
{
    return M >= 0 && M <= kMaxRows && N >= 1 && N <= kMaxPitch - 8 && K >= 8 && K % 8 == 0 && K <= kMaxPitch - 8;
}
bool linear_activation(atb_activation act) { return act == ATB_ACT_NONE || is_activation(act); }

bool is_linear(const atb_linear *l)
{
    if (!l || !linear_lengths(l->M, l->N, l->K) || !linear_activation(l->act) || !is_type(l->bias_type) || !aligned(l->bias, size_of(l->bias_type))) return false;
    return aligned(l->workspace, 16) && is_matrix(l->w, l->K, l->ldw) && (l->M == 0 || is_matrix(l->x, l->K, l->ldx));
}

// dy itself is what the products of the backward pass read
bool direct(int64_t N, atb_activation act) { return act == ATB_ACT_NONE && N % 8 == 0; }

// The parts of the backward pass's workspace, in bytes: dz, the column sums, the shares of the products (not at the same time as the sums, but dz is with both)
struct LinearRoom { int64_t dz, partial, shares; };
LinearRoom linear_room(int64_t M, int64_t N, int64_t K, atb_activation act)
{
    LinearRoom r;
    r.dz = direct(N, act) ? 0 : atb::round_up(M * atb::round_up(N, 8) * 2, 256);
    r.partial = atb::round_up(atb::linear_parts(M, N) * N * (int64_t)sizeof(float), 256);
    r.shares = (int64_t)sizeof(float) * std::max(atb::tile_shares(M, K, N, 1, 1, false), atb::tile_shares(N, K, M, 1, 1, false));
    return r;
}

atb::TileParams tiles(void *shares, int64_t M, int64_t N, int64_t K)
{
    atb::TileParams p = {};
    p.shares = static_cast<float *>(shares);
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.segments = p.problems = 1;
    return p;
}

}  // namespace

extern "C" size_t atb_linear_workspace(int64_t M, int64_t N, int64_t K, int keeps)
{
    if (!linear_lengths(M, N, K) || (atb::ffn_streams(M) && !keeps)) return 0;
    return sizeof(float) * (size_t)atb::tile_shares(M, atb::round_up(N, 8), K, 1, 1, false);
}

extern "C" atb_status atb_linear_forward(const atb_linear *l, const void *residual, int64_t ldr, void *slope, void *y, int64_t ldy, void *hip_stream)
{
    if (!is_linear(l) || (slope && l->act == ATB_ACT_NONE)) return ATB_ERR_INVALID_ARG;
    if (l->M == 0) return ATB_OK;
    if (!is_rows(y, l->N, ldy, 2) || (residual && !is_rows(residual, l->N, ldr, 2)) || !aligned(slope, 2)) return ATB_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (atb::ffn_streams(l->M) && !slope) {
        atb::StreamParams s = {};
        s.w[0] = {l->w, nullptr, nullptr, l->ldw};
        s.x = u16(l->x); s.ldx = l->ldx;
        s.y = y; s.ldy = ldy;
        s.M = (int)l->M; s.N = (int)l->N; s.K = (int)l->K;
        s.act = l->act;
        s.y_type = ATB_TYPE_BF16;
        s.linear = 1;
        s.bias = l->bias;
        s.bias_type = l->bias_type;
        s.residual = u16(residual);
        s.ldr = ldr;
        return hip_status(atb::launch_stream(s, stream));
    }
    atb::TileParams p = tiles(l->workspace, l->M, atb::round_up(l->N, 8), l->K);
    p.A[0] = u16(l->x); p.lda[0] = l->ldx;
    p.B[0] = u16(l->w); p.ldb[0] = l->ldw;
    p.C[0] = u16(y);
    p.ldc = ldy;
    p.act = l->act;
    p.edge = (int)l->N;
    p.bias = l->bias;
    p.bias_type = l->bias_type;
    p.residual = u16(residual);
    p.ldr = ldr;
    p.slope = u16(slope);
    return hip_status(atb::launch_tiles_linear(p, slope ? atb::kLinearKeep : atb::kLinear, stream));
}

extern "C" size_t atb_linear_backward_workspace(int64_t M, int64_t N, int64_t K, atb_activation act)
{
    if (!linear_lengths(M, N, K) || !linear_activation(act)) return 0;
    const LinearRoom r = linear_room(M, N, K, act);
    return (size_t)(r.dz + std::max(r.partial, r.shares));
}

extern "C" atb_status atb_linear_backward(const atb_linear *l, const void *slope, const void *dy, int64_t lddy, void *dx, int64_t lddx, void *dw, void *dbias, void *hip_stream)
{
    if (!is_linear(l) || !aligned(dw, 16) || !aligned(dbias, size_of(l->bias_type))) return ATB_ERR_INVALID_ARG;
    const int64_t M = l->M, N = l->N, K = l->K;
    const bool as_it_is = direct(N, l->act);
    const LinearRoom room = linear_room(M, N, K, l->act);
    if (M > 0) {
        if (!(as_it_is ? is_matrix(dy, N, lddy) : is_rows(dy, N, lddy, 2)) || (dx && !is_matrix(dx, K, lddx))) return ATB_ERR_INVALID_ARG;
        if ((l->act == ATB_ACT_NONE) != !slope || !aligned(slope, 2)) return ATB_ERR_INVALID_ARG;
        if (!l->workspace && (room.dz || room.partial || room.shares)) return ATB_ERR_INVALID_ARG;
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char *work = static_cast<char *>(l->workspace);
    void *shares = work ? work + room.dz : nullptr;
    const bool products = M > 0 && (dx || dw);
    atb::LinearGradParams g = {};
    g.dy = u16(dy); g.lddy = lddy;
    g.slope = u16(slope);
    g.dz = products && !as_it_is ? u16(static_cast<void *>(work)) : nullptr;
    g.partial = dbias ? static_cast<float *>(shares) : nullptr;
    g.dbias = dbias;
    g.bias_type = l->bias_type;
    g.M = M;
    g.N = (int)N;
    atb_status st = hip_status(atb::launch_linear_grad(g, stream));
    const uint16_t *dz = as_it_is ? u16(dy) : u16(static_cast<const void *>(work));
    const int64_t lddz = M == 0 ? atb::round_up(N, 8) : as_it_is ? lddy : atb::round_up(N, 8);       // (no tokens: no K-steps, and nothing of the operands is read)
    if (st == ATB_OK && M > 0 && dx) {
        atb::TileParams p = tiles(shares, M, K, N);
        p.A[0] = dz; p.lda[0] = lddz;
        p.B[0] = u16(l->w); p.ldb[0] = l->ldw;
        p.C[0] = u16(dx);
        p.ldc = lddx;
        st = hip_status(atb::launch_tiles_dx(p, atb::kStore, stream));
    }
    if (st == ATB_OK && dw) {
        atb::TileParams p = tiles(shares, N, K, M);
        p.A[0] = dz; p.lda[0] = lddz;
        p.B[0] = u16(l->x); p.ldb[0] = M > 0 ? l->ldx : K;
        p.C[0] = u16(dw);
        p.ldc = K;
        st = hip_status(atb::launch_tiles_dw(p, stream));
    }
    return st;
}
