// C ABI of the feed-forward sublayer's operators (see include/atb.h): argument checking and launches.
#include "atb_layers.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 23, kMaxPitch = (int64_t)1 << 22, kMaxRowsApart = (int64_t)1 << 26, kMaxNorm = (int64_t)1 << 24;

using atb::hip_status;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool is_type(atb_type t) { return t == ATB_TYPE_BF16 || t == ATB_TYPE_F32; }
bool is_activation(atb_activation a) { return a == ATB_ACT_SILU || a == ATB_ACT_GELU || a == ATB_ACT_GELU_TANH; }
uintptr_t size_of(atb_type t) { return t == ATB_TYPE_F32 ? 4 : 2; }

// A bf16 matrix that the tile kernels read or write in 16-byte pieces
bool is_matrix(const void *p, int64_t cols, int64_t ld) { return p && aligned(p, 16) && ld >= cols && ld % 8 == 0 && ld < kMaxPitch; }

bool ffn_lengths(int64_t M, int64_t D, int64_t F)
{
    return M >= 0 && M <= kMaxRows && D >= 8 && D % 8 == 0 && D <= kMaxPitch - 8 && F >= 8 && F % 8 == 0 && F <= kMaxPitch - 8;
}

bool ffn_sizes(const atb_ffn *f)
{
    if (!f || !ffn_lengths(f->M, f->D, f->F) || !aligned(f->workspace, 16)) return false;
    return is_activation(f->act) && is_matrix(f->w_gate, f->D, f->ld_gate) && is_matrix(f->w_up, f->D, f->ld_up) && is_matrix(f->w_down, f->F, f->ld_down) &&
           (f->M == 0 || is_matrix(f->x, f->D, f->ldx));
}

bool is_q4(const atb_q4 *w)
{
    if (!w || w->N < 1 || w->N > kMaxNorm || (w->group != 32 && w->group != 64 && w->group != 128) || w->K < w->group || w->K % w->group != 0 || w->K > kMaxPitch) return false;
    return w->packed && aligned(w->packed, 16) && w->scales && aligned(w->scales, 2);
}

const uint16_t *u16(const void *p) { return static_cast<const uint16_t *>(p); }
uint16_t *u16(void *p) { return static_cast<uint16_t *>(p); }

atb::TileParams tiles(const atb_ffn *f, int64_t M, int64_t N, int64_t K)
{
    atb::TileParams p = {};
    p.shares = static_cast<float *>(f->workspace);
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.segments = p.problems = 1;
    return p;
}
void operand_a(atb::TileParams &p, int i, const void *a, int64_t ld) { p.A[i] = u16(a); p.lda[i] = ld; }
void operand_b(atb::TileParams &p, int i, const void *b, int64_t ld) { p.B[i] = u16(b); p.ldb[i] = ld; }

}  // namespace

// ------------------------------------------------------------------ layer norm

extern "C" atb_status atb_layer_norm(const void *x, int64_t ldx, const void *weight, const void *bias, double eps, void *y, int64_t ldy,
                                     float *mean, float *rstd, int64_t M, int64_t D, atb_type type, atb_type param_type, void *stream)
{
    if (M < 0 || M > kMaxRows || D < 1 || D > kMaxNorm || !is_type(type) || !is_type(param_type) || !(eps >= 0.0)) return ATB_ERR_INVALID_ARG;
    if (M == 0) return ATB_OK;
    if (!x || !y || ldx < D || ldy < D || !aligned(x, size_of(type)) || !aligned(y, size_of(type))) return ATB_ERR_INVALID_ARG;
    if (!aligned(weight, size_of(param_type)) || !aligned(bias, size_of(param_type)) || !aligned(mean, 4) || !aligned(rstd, 4)) return ATB_ERR_INVALID_ARG;
    atb::NormParams p = {};
    p.x = x; p.ldx = ldx;
    p.y = y; p.ldy = ldy;
    p.weight = weight;
    p.bias = bias;
    p.mean = mean;
    p.rstd = rstd;
    p.M = M;
    p.D = D;
    p.eps = (float)eps;
    p.x_type = type;
    p.w_type = param_type;
    return hip_status(atb::launch_norm(p, static_cast<hipStream_t>(stream)));
}

extern "C" size_t atb_layer_norm_workspace(int64_t M, int64_t D)
{
    if (M < 0 || M > kMaxRows || D < 1 || D > kMaxNorm) return 0;
    return (size_t)(atb::norm_partials(M, D) * 2 * D) * sizeof(float);
}

extern "C" atb_status atb_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, const float *mean, const float *rstd,
                                              const void *weight, void *dx, int64_t lddx, void *dweight, void *dbias, void *workspace,
                                              int64_t M, int64_t D, atb_type type, atb_type param_type, void *stream)
{
    if (M < 0 || M > kMaxRows || D < 1 || D > kMaxNorm || !is_type(type) || !is_type(param_type)) return ATB_ERR_INVALID_ARG;
    if (!aligned(weight, size_of(param_type)) || !aligned(dweight, size_of(param_type)) || !aligned(dbias, size_of(param_type))) return ATB_ERR_INVALID_ARG;
    if (M > 0) {
        if (!dy || !x || !mean || !rstd || lddy < D || ldx < D || !aligned(dy, size_of(type)) || !aligned(x, size_of(type)) || !aligned(mean, 4) || !aligned(rstd, 4)) return ATB_ERR_INVALID_ARG;
        if (dx && (lddx < D || !aligned(dx, size_of(type)))) return ATB_ERR_INVALID_ARG;
        if ((dweight || dbias) && (!workspace || !aligned(workspace, 16))) return ATB_ERR_INVALID_ARG;
    }
    atb::NormParams p = {};
    p.dy = dy; p.lddy = lddy;
    p.x = x; p.ldx = ldx;
    p.dx = dx; p.lddx = lddx;
    p.mean = const_cast<float *>(mean);
    p.rstd = const_cast<float *>(rstd);
    p.weight = weight;
    p.dweight = dweight;
    p.dbias = dbias;
    p.partial = static_cast<float *>(workspace);
    p.M = M;
    p.D = D;
    p.x_type = type;
    p.w_type = param_type;
    return hip_status(atb::launch_norm_backward(p, static_cast<hipStream_t>(stream)));
}

// ------------------------------------------------------------------ the gated block in bf16

extern "C" size_t atb_ffn_kept_bytes(int64_t M, int64_t F)
{
    if (M < 0 || M > kMaxRows || F < 8 || F % 8 != 0 || F > kMaxPitch - 8) return 0;
    return (size_t)(6 * M * F);
}

extern "C" size_t atb_ffn_workspace(int64_t M, int64_t D, int64_t F, int keeps)
{
    if (!ffn_lengths(M, D, F) || (atb::ffn_streams(M) && !keeps)) return 0;
    return sizeof(float) * (size_t)std::max(atb::tile_shares(M, F, D, 1, 1, true), atb::tile_shares(M, D, F, 1, 1, false));
}

extern "C" size_t atb_ffn_backward_workspace(int64_t M, int64_t D, int64_t F)
{
    if (!ffn_lengths(M, D, F)) return 0;
    return sizeof(float) * (size_t)std::max({atb::tile_shares(M, F, D, 1, 1, false), atb::tile_shares(M, D, F, 2, 1, false),       // dh, dx
                                             atb::tile_shares(F, D, M, 1, 2, false), atb::tile_shares(D, F, M, 1, 1, false)});     // the weights'
}

extern "C" atb_status atb_ffn_forward(const atb_ffn *f, void *h, void *kept, void *y, int64_t ldy, void *hip_stream)
{
    if (!ffn_sizes(f)) return ATB_ERR_INVALID_ARG;
    if (f->M == 0) return ATB_OK;
    if (!is_matrix(h, f->F, f->F) || !is_matrix(y, f->D, ldy) || !aligned(kept, 16)) return ATB_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (atb::ffn_streams(f->M) && !kept) {
        atb::StreamParams s = {};
        s.w[0] = {f->w_gate, nullptr, nullptr, f->ld_gate};
        s.w[1] = {f->w_up, nullptr, nullptr, f->ld_up};
        s.x = u16(f->x); s.ldx = f->ldx;
        s.y = h; s.ldy = f->F;
        s.M = (int)f->M; s.N = (int)f->F; s.K = (int)f->D;
        s.gated = 1;
        s.act = f->act;
        s.y_type = ATB_TYPE_BF16;
        const atb_status st = hip_status(atb::launch_stream(s, stream));
        if (st != ATB_OK) return st;
        atb::StreamParams d = {};
        d.w[0] = {f->w_down, nullptr, nullptr, f->ld_down};
        d.x = u16(h); d.ldx = f->F;
        d.y = y; d.ldy = ldy;
        d.M = (int)f->M; d.N = (int)f->D; d.K = (int)f->F;
        d.y_type = ATB_TYPE_BF16;
        return hip_status(atb::launch_stream(d, stream));
    }
    atb::TileParams p = tiles(f, f->M, f->F, f->D);
    operand_a(p, 0, f->x, f->ldx);
    operand_b(p, 0, f->w_gate, f->ld_gate);
    operand_b(p, 1, f->w_up, f->ld_up);
    p.C[0] = u16(h);
    p.ldc = f->F;
    p.kept = u16(kept);
    p.act = f->act;
    const atb_status st = hip_status(atb::launch_tiles_forward(p, kept ? atb::kGatedKeep : atb::kGated, stream));
    if (st != ATB_OK) return st;
    atb::TileParams d = tiles(f, f->M, f->D, f->F);
    operand_a(d, 0, h, f->F);
    operand_b(d, 0, f->w_down, f->ld_down);
    d.C[0] = u16(y);
    d.ldc = ldy;
    return hip_status(atb::launch_tiles_forward(d, atb::kStore, stream));
}

extern "C" atb_status atb_ffn_backward(const atb_ffn *f, const void *h, const void *kept, const void *dy, int64_t lddy,
                                       void *dgate, void *dup, void *dx, int64_t lddx, void *dw_gate, void *dw_up, void *dw_down, void *hip_stream)
{
    if (!ffn_sizes(f) || !dw_gate != !dw_up) return ATB_ERR_INVALID_ARG;
    if (!aligned(dw_gate, 16) || !aligned(dw_up, 16) || !aligned(dw_down, 16)) return ATB_ERR_INVALID_ARG;
    if (f->M > 0) {
        if (!is_matrix(h, f->F, f->F) || !kept || !aligned(kept, 16) || !is_matrix(dy, f->D, lddy)) return ATB_ERR_INVALID_ARG;
        if (!is_matrix(dgate, f->F, f->F) || !is_matrix(dup, f->F, f->F) || (dx && !is_matrix(dx, f->D, lddx))) return ATB_ERR_INVALID_ARG;
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    atb_status st = ATB_OK;
    if (f->M > 0 && (dx || dw_gate)) {
        atb::TileParams p = tiles(f, f->M, f->F, f->D);                 // dh = dy Wd
        operand_a(p, 0, dy, lddy);
        operand_b(p, 0, f->w_down, f->ld_down);
        p.C[0] = u16(dgate);
        p.C[1] = u16(dup);
        p.ldc = f->F;
        p.kept = const_cast<uint16_t *>(u16(kept));
        p.act = f->act;
        st = hip_status(atb::launch_tiles_dx(p, atb::kGatedGrad, stream));
    }
    if (st == ATB_OK && f->M > 0 && dx) {
        atb::TileParams p = tiles(f, f->M, f->D, f->F);
        operand_a(p, 0, dgate, f->F);
        operand_a(p, 1, dup, f->F);
        operand_b(p, 0, f->w_gate, f->ld_gate);
        operand_b(p, 1, f->w_up, f->ld_up);
        p.segments = 2;
        p.C[0] = u16(dx);
        p.ldc = lddx;
        st = hip_status(atb::launch_tiles_dx(p, atb::kStore, stream));
    }
    // (no tokens: no K-steps, and nothing of the operands is read)
    const int64_t ldx = f->M > 0 ? f->ldx : f->D, ld_dy = f->M > 0 ? lddy : f->D;
    if (st == ATB_OK && dw_gate) {
        atb::TileParams p = tiles(f, f->F, f->D, f->M);
        operand_a(p, 0, dgate, f->F);
        operand_a(p, 1, dup, f->F);
        operand_b(p, 0, f->x, ldx);
        operand_b(p, 1, f->x, ldx);
        p.problems = 2;
        p.C[0] = u16(dw_gate);
        p.C[1] = u16(dw_up);
        p.ldc = f->D;
        st = hip_status(atb::launch_tiles_dw(p, stream));
    }
    if (st == ATB_OK && dw_down) {
        atb::TileParams p = tiles(f, f->D, f->F, f->M);
        operand_a(p, 0, dy, ld_dy);
        operand_b(p, 0, h, f->F);
        p.C[0] = u16(dw_down);
        p.ldc = f->F;
        st = hip_status(atb::launch_tiles_dw(p, stream));
    }
    return st;
}

// ------------------------------------------------------------------ 4-bit weights

extern "C" atb_status atb_q4_quantize(const void *W, int64_t ldw, atb_type type, void *packed, void *scales, void *zeros,
                                      int64_t N, int64_t K, int group, void *stream)
{
    const atb_q4 w = {packed, scales, zeros, N, K, group};
    if (!is_q4(&w) || !W || ldw < K || !is_type(type) || !aligned(W, size_of(type))) return ATB_ERR_INVALID_ARG;
    return hip_status(atb::launch_q4_quantize(W, type, ldw, static_cast<uint8_t *>(packed), u16(scales), static_cast<uint8_t *>(zeros), N, K, group, static_cast<hipStream_t>(stream)));
}

extern "C" atb_status atb_q4_decode(const atb_q4 *w, void *out, atb_type out_type, void *stream)
{
    if (!is_q4(w) || !out || !is_type(out_type) || !aligned(out, size_of(out_type))) return ATB_ERR_INVALID_ARG;
    return hip_status(atb::launch_q4_decode(static_cast<const uint8_t *>(w->packed), u16(w->scales), static_cast<const uint8_t *>(w->zeros), out, out_type, w->N, w->K, w->group,
                                            static_cast<hipStream_t>(stream)));
}

namespace {

bool q4_operands(const atb_q4 *w, const void *x, int64_t ldx, const void *y, int64_t ldy, atb_type y_type, int64_t M)
{
    // 16 rows of x are within 2^31 bytes
    return x && aligned(x, 16) && ldx >= w->K && ldx % 8 == 0 && ldx <= kMaxRowsApart && y && aligned(y, size_of(y_type)) && ldy >= w->N && M <= kMaxRows;
}

atb::StreamParams q4_params(const atb_q4 *w, const void *x, int64_t ldx, void *y, int64_t ldy, atb_type y_type, int64_t M)
{
    atb::StreamParams s = {};
    s.w[0] = {w->packed, u16(w->scales), static_cast<const uint8_t *>(w->zeros), 0};
    s.x = u16(x); s.ldx = ldx;
    s.y = y; s.ldy = ldy;
    s.M = (int)M; s.N = (int)w->N; s.K = (int)w->K;
    s.group = w->group;
    s.y_type = y_type;
    return s;
}

}  // namespace

extern "C" atb_status atb_q4_matvec(const atb_q4 *w, const void *x, int64_t ldx, void *y, int64_t ldy, atb_type y_type, int64_t M, void *stream)
{
    if (!is_q4(w) || !is_type(y_type) || M < 0) return ATB_ERR_INVALID_ARG;
    if (M == 0) return ATB_OK;
    if (!q4_operands(w, x, ldx, y, ldy, y_type, M)) return ATB_ERR_INVALID_ARG;
    return hip_status(atb::launch_stream(q4_params(w, x, ldx, y, ldy, y_type, M), static_cast<hipStream_t>(stream)));
}

extern "C" atb_status atb_q4_gated(const atb_q4 *w_gate, const atb_q4 *w_up, atb_activation act, const void *x, int64_t ldx, void *h, int64_t ldh,
                                   int64_t M, void *stream)
{
    if (!is_q4(w_gate) || !is_q4(w_up) || !is_activation(act) || M < 0) return ATB_ERR_INVALID_ARG;
    if (w_gate->N != w_up->N || w_gate->K != w_up->K || w_gate->group != w_up->group || !w_gate->zeros != !w_up->zeros) return ATB_ERR_INVALID_ARG;
    if (M == 0) return ATB_OK;
    if (!q4_operands(w_gate, x, ldx, h, ldh, ATB_TYPE_BF16, M)) return ATB_ERR_INVALID_ARG;
    atb::StreamParams s = q4_params(w_gate, x, ldx, h, ldh, ATB_TYPE_BF16, M);
    s.w[1] = {w_up->packed, u16(w_up->scales), static_cast<const uint8_t *>(w_up->zeros), 0};
    s.gated = 1;
    s.act = act;
    return hip_status(atb::launch_stream(s, static_cast<hipStream_t>(stream)));
}
