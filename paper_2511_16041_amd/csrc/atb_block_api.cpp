// C ABI of what a block has around its feed-forward sublayer (see include/atb.h): argument checking and launches.
#include "atb_block.h"

#include <cmath>
#include <limits>

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 23, kMaxPitch = (int64_t)1 << 22, kMaxNorm = (int64_t)1 << 24;

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

extern "C" size_t atb_linear_workspace(int64_t M, int64_t N, int64_t K)
{
    if (!linear_lengths(M, N, K) || atb::ffn_streams(M)) return 0;
    return sizeof(float) * (size_t)atb::tile_shares(M, atb::round_up(N, 8), K, 1, 1, false, true);
}

extern "C" atb_status atb_linear_forward(const atb_linear *l, const void *residual, int64_t ldr, void *slope, void *y, int64_t ldy, void *hip_stream)
{
    if (!is_linear(l) || (slope && l->act == ATB_ACT_NONE)) return ATB_ERR_INVALID_ARG;
    if (l->M == 0) return ATB_OK;
    if (!is_rows(y, l->N, ldy, 2) || (residual && !is_rows(residual, l->N, ldr, 2)) || !aligned(slope, 16)) return ATB_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (atb::ffn_streams(l->M)) {
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
        s.slope = u16(slope);
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
        if ((l->act == ATB_ACT_NONE) != !slope || !aligned(slope, 16)) return ATB_ERR_INVALID_ARG;
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
    atb::TileParams px = tiles(shares, M, K, N), pw = tiles(shares, N, K, M);
    px.A[0] = pw.A[0] = dz; px.lda[0] = pw.lda[0] = lddz;
    px.B[0] = u16(l->w); px.ldb[0] = l->ldw;
    px.C[0] = u16(dx);
    px.ldc = lddx;
    pw.B[0] = u16(l->x); pw.ldb[0] = M > 0 ? l->ldx : K;
    pw.C[0] = u16(dw);
    pw.ldc = K;
    const int together = M > 0 && dx && dw ? atb::linear_pair(M, N, K) : 0;
    if (st == ATB_OK && together) return hip_status(atb::launch_tiles_pair(px, pw, together, stream));
    if (st == ATB_OK && M > 0 && dx) st = hip_status(atb::launch_tiles_dx(px, atb::kStore, stream));
    if (st == ATB_OK && dw) st = hip_status(atb::launch_tiles_dw(pw, stream));
    return st;
}

// ------------------------------------------------------------------ norms on both sides of a residual sum

namespace {

bool residual_lengths(int64_t M, int64_t D, int64_t groups)
{
    return M >= 0 && M <= kMaxRows && D >= 1 && D <= kMaxNorm && groups >= 1 && groups <= 65535 && M % groups == 0;
}
bool is_norm(const atb_norm &n, atb_type type)
{
    if (n.kind == ATB_NORM_NONE) return true;
    // (the kernels take eps in fp32: one that becomes 0 there would make NaN of a row of zeros)
    if (!(n.eps >= 0.0) || n.eps > std::numeric_limits<float>::max() || (n.eps > 0.0 && (float)n.eps == 0.0f)) return false;
    return (n.kind == ATB_NORM_RMS || n.kind == ATB_NORM_LAYER) && aligned(n.weight, size_of(type)) && aligned(n.bias, size_of(type));
}
bool is_residual(const atb_residual_norm *p)
{
    if (!p || !residual_lengths(p->M, p->D, p->groups) || !is_type(p->stream_type) || !is_type(p->block_type) || !is_type(p->param_type)) return false;
    if (p->block_type == ATB_TYPE_F32 && p->stream_type != ATB_TYPE_F32) return false;
    if (!is_norm(p->post, p->param_type) || !is_norm(p->pre, p->param_type) || !aligned(p->gate, size_of(p->param_type)) || (!p->gate && p->groups != 1)) return false;
    if (!(std::abs(p->scale) <= std::numeric_limits<float>::max())) return false;          // (the kernels take it in fp32)
    return p->M == 0 || (is_rows(p->x, p->D, p->ldx, size_of(p->stream_type)) && is_rows(p->z, p->D, p->ldz, size_of(p->block_type)));
}
atb::NormSpec spec(const atb_norm &n)
{
    if (n.kind == ATB_NORM_NONE) return {ATB_NORM_NONE, nullptr, nullptr, 0.0f};
    return {n.kind, n.weight, n.bias, (float)n.eps};
}
atb::ResidualParams residual(const atb_residual_norm *p)
{
    atb::ResidualParams r = {};
    r.x = p->x; r.ldx = p->ldx;
    r.z = p->z; r.ldz = p->ldz;
    r.post = spec(p->post);
    r.pre = spec(p->pre);
    r.gate = p->gate;
    r.groups = p->groups;
    r.scale = (float)p->scale;
    r.M = p->M;
    r.D = (int)p->D;
    r.x_type = p->stream_type;
    r.z_type = p->block_type;
    r.w_type = p->param_type;
    return r;
}

}  // namespace

extern "C" atb_status atb_residual_norm_forward(const atb_residual_norm *p, void *r, int64_t ldr, void *h, int64_t ldh, float *stats, void *hip_stream)
{
    if (!is_residual(p) || !aligned(stats, 4)) return ATB_ERR_INVALID_ARG;
    if (p->M == 0) return ATB_OK;
    if (!is_rows(r, p->D, ldr, size_of(p->stream_type))) return ATB_ERR_INVALID_ARG;
    if (p->pre.kind == ATB_NORM_NONE ? h != nullptr : !is_rows(h, p->D, ldh, size_of(p->block_type))) return ATB_ERR_INVALID_ARG;
    atb::ResidualParams q = residual(p);
    q.r = r; q.ldr = ldr;
    q.h = h; q.ldh = ldh;
    q.stats = stats;
    return hip_status(atb::launch_residual(q, static_cast<hipStream_t>(hip_stream)));
}

extern "C" size_t atb_residual_norm_workspace(int64_t M, int64_t D, int64_t groups)
{
    return residual_lengths(M, D, groups) ? sizeof(float) * (size_t)atb::residual_room(M, D, groups).total : 0;
}

extern "C" atb_status atb_residual_norm_backward(const atb_residual_norm *p, const float *stats, const void *dr, int64_t lddr, const void *dh, int64_t lddh,
                                                 const atb_residual_norm_grads *grads, void *workspace, void *hip_stream)
{
    if (!is_residual(p) || !grads) return ATB_ERR_INVALID_ARG;
    const uintptr_t es = size_of(p->stream_type), eb = size_of(p->block_type), ep = size_of(p->param_type);
    const atb_residual_norm_grads &g = *grads;
    for (const void *d : {g.dgate, g.dpost_weight, g.dpost_bias, g.dpre_weight, g.dpre_bias})
        if (!aligned(d, ep)) return ATB_ERR_INVALID_ARG;
    // a gradient of what there is not
    if (((g.dpost_weight || g.dpost_bias) && p->post.kind == ATB_NORM_NONE) || ((g.dpre_weight || g.dpre_bias) && p->pre.kind == ATB_NORM_NONE) || (g.dgate && !p->gate)) return ATB_ERR_INVALID_ARG;
    const bool asked = g.dgate || g.dpost_weight || g.dpost_bias || g.dpre_weight || g.dpre_bias;
    if (asked && atb::residual_room(p->M, p->D, p->groups).total > 0 && (!workspace || !aligned(workspace, 16))) return ATB_ERR_INVALID_ARG;
    if (p->M > 0) {
        if (!stats || !aligned(stats, 4) || (dr && !is_rows(dr, p->D, lddr, es))) return ATB_ERR_INVALID_ARG;
        if (p->pre.kind == ATB_NORM_NONE ? dh != nullptr : !is_rows(dh, p->D, lddh, eb)) return ATB_ERR_INVALID_ARG;
        if ((g.dx && !is_rows(g.dx, p->D, g.lddx, es)) || (g.dz && !is_rows(g.dz, p->D, g.lddz, eb))) return ATB_ERR_INVALID_ARG;
    }
    atb::ResidualParams q = residual(p);
    q.stats = const_cast<float *>(stats);
    q.dr = dr; q.lddr = lddr;
    q.dh = dh; q.lddh = lddh;
    q.dx = g.dx; q.lddx = g.lddx;
    q.dz = g.dz; q.lddz = g.lddz;
    q.dgate = g.dgate;
    q.dpost_weight = g.dpost_weight;
    q.dpost_bias = g.dpost_bias;
    q.dpre_weight = g.dpre_weight;
    q.dpre_bias = g.dpre_bias;
    q.workspace = static_cast<float *>(workspace);
    return hip_status(atb::launch_residual_backward(q, static_cast<hipStream_t>(hip_stream)));
}

// ------------------------------------------------------------------ a mixture of experts for few tokens

namespace {

bool moe_counts(int64_t M, int experts, int top_k)
{
    return M >= 0 && M <= atb::kMoeTokens && experts >= 1 && experts <= atb::kMoeExperts && top_k >= 1 && top_k <= atb::kMoeTopK && top_k <= experts;
}
bool moe_group(int group) { return group == 0 || group == 32 || group == 64 || group == 128; }
bool moe_length(int64_t n, int group) { return n >= 8 && n < kMaxPitch && n % (group ? group : 8) == 0; }
bool is_moe_weight(const atb_moe_weight &w, int group, bool zeros)
{
    if (!w.w || !aligned(w.w, 16)) return false;
    return group == 0 || (w.scales && aligned(w.scales, 2) && !w.zeros == !zeros);
}
atb::StreamWeight moe_weight(const atb_moe_weight &w, int group)
{
    if (group == 0) return {w.w, nullptr, nullptr, 0};
    return {w.w, u16(w.scales), static_cast<const uint8_t *>(w.zeros), 0};
}

}  // namespace

extern "C" size_t atb_moe_workspace(int64_t M, int64_t D, int64_t F, int experts, int top_k, int group)
{
    if (!moe_counts(M, experts, top_k) || !moe_group(group) || !moe_length(D, group) || !moe_length(F, group)) return 0;
    return (size_t)atb::moe_room(M, D, F, experts, top_k, group).total;
}

extern "C" atb_status atb_moe_forward(const atb_moe *m, void *y, int64_t ldy, int32_t *chosen, float *p, void *hip_stream)
{
    if (!m || !moe_counts(m->M, m->experts, m->top_k) || !is_activation(m->act)) return ATB_ERR_INVALID_ARG;
    if (!moe_group(m->group) || !moe_length(m->D, m->group) || !moe_length(m->F, m->group)) return ATB_ERR_INVALID_ARG;
    const bool zeros = m->w_gate.zeros != nullptr;
    if (!is_moe_weight(m->w_gate, m->group, zeros) || !is_moe_weight(m->w_up, m->group, zeros) || !is_moe_weight(m->w_down, m->group, zeros)) return ATB_ERR_INVALID_ARG;
    if (!is_matrix(m->router, m->D, m->ld_router) || !aligned(chosen, 4) || !aligned(p, 4)) return ATB_ERR_INVALID_ARG;
    if (m->M == 0) return ATB_OK;
    if (!is_matrix(m->x, m->D, m->ldx) || !is_rows(y, m->D, ldy, 2) || !m->workspace || !aligned(m->workspace, 16)) return ATB_ERR_INVALID_ARG;
    const atb::MoeRoom room = atb::moe_room(m->M, m->D, m->F, m->experts, m->top_k, m->group);
    char *work = static_cast<char *>(m->workspace);
    atb::MoeParams q = {};
    q.x = u16(m->x); q.ldx = m->ldx;
    q.router = u16(m->router); q.ld_router = m->ld_router;
    q.gate = moe_weight(m->w_gate, m->group);
    q.up = moe_weight(m->w_up, m->group);
    q.down = moe_weight(m->w_down, m->group);
    q.y = u16(y); q.ldy = ldy;
    q.experts = chosen;
    q.weights = p;
    q.M = (int)m->M; q.D = (int)m->D; q.F = (int)m->F; q.E = m->experts; q.k = m->top_k;
    q.group = m->group;
    q.act = m->act;
    q.renormalize = m->renormalize;
    q.few = atb::moe_is_few(m->M, m->experts, m->top_k, m->F);
    q.logits = reinterpret_cast<double *>(work);
    q.plan = reinterpret_cast<atb::MoePlan *>(work + room.logits);
    q.h = reinterpret_cast<uint16_t *>(work + room.logits + room.plan);
    q.shares = atb::moe_shares(m->M, m->D, m->F, m->experts, m->top_k, m->group);
    q.partial = reinterpret_cast<float *>(work + room.logits + room.plan + room.h);
    return hip_status(atb::launch_moe(q, static_cast<hipStream_t>(hip_stream)));
}
