// Host program of the sanitizer build: the argument handling of a block's operators (atb_block_api.cpp) and the rules that choose tiles, shares and sizes of workspaces (atb_block.h, atb_layers.h), with the
// launches replaced by ones that check what they are given; in every other call they fail, as without a GPU.
#include "atb.h"
#include "atb_block.h"

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#define CHECK(x) do { if (!(x)) { std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

namespace {

char *g_work = nullptr;          // the workspace of the call and its bytes
size_t g_bytes = 0;
int g_launches = 0;
hipError_t g_result = hipSuccess;

// [at, at + bytes) lies in the workspace
bool inside(const void *at, uint64_t bytes)
{
    const uintptr_t from = reinterpret_cast<uintptr_t>(at), base = reinterpret_cast<uintptr_t>(g_work);
    return from >= base && bytes <= g_bytes && from - base <= g_bytes - bytes && (from & 15) == 0;
}

hipError_t tiles(const atb::TileParams &p, bool linear)
{
    ++g_launches;
    CHECK(p.M >= 1 && p.N >= 1 && p.N % 8 == 0 && p.K >= 0 && p.segments == 1 && p.problems == 1);
    CHECK(linear ? p.edge >= 1 && p.N - p.edge >= 0 && p.N - p.edge < 8 : p.edge == 0);
    const atb::TileChoice how = atb::choose_tiles(p.M, p.N, p.K, 1, 1, false, p.shares != nullptr, linear);
    CHECK(how.parts >= 1 && (how.parts == 1 || p.shares) && !(how.wide && how.parts > 1) && !(how.wide && !linear));
    if (how.parts > 1) {
        CHECK(inside(p.shares, (uint64_t)how.parts * (uint64_t)p.M * (uint64_t)p.N * 4));
        CHECK((int64_t)p.M * (p.N / 4) < (int64_t)1 << 31);                       // the join's index
        CHECK((int64_t)((p.K + 63) / 64) >= how.parts);                           // no empty share
    }
    return g_result;
}

}  // namespace

namespace atb {
hipError_t launch_tiles_linear(TileParams p, int epilogue, hipStream_t) { CHECK(is_linear(epilogue) && (epilogue == kLinearKeep) == (p.slope != nullptr)); return tiles(p, true); }
hipError_t launch_tiles_dx(TileParams p, int epilogue, hipStream_t) { CHECK(epilogue == kStore); return tiles(p, false); }
hipError_t launch_tiles_dw(TileParams p, hipStream_t) { return tiles(p, false); }
hipError_t launch_tiles_pair(TileParams dx, TileParams dw, int tile, hipStream_t)
{
    ++g_launches;
    for (const TileParams &p : {dx, dw}) CHECK(p.M >= 1 && p.N % 8 == 0 && p.K >= 1 && p.edge == 0 && p.segments == 1 && p.problems == 1);
    CHECK((tile == 128 || tile == 256) && dx.M == dw.K && dx.K == dw.M && dx.N == dw.N);
    return g_result;
}
hipError_t launch_stream(const StreamParams &p, hipStream_t) { ++g_launches; CHECK(p.M >= 1 && p.M <= 32 && p.N >= 1 && p.K >= 8 && p.linear); return g_result; }
hipError_t launch_linear_grad(const LinearGradParams &p, hipStream_t)
{
    ++g_launches;
    const int64_t parts = linear_parts(p.M, p.N);
    CHECK(p.M == 0 ? parts == 0 : parts >= 1 && parts <= 65535 && (p.M + parts - 1) / parts <= 512);
    if (p.dz) CHECK(inside(p.dz, (uint64_t)p.M * (uint64_t)round_up(p.N, 8) * 2));
    if (p.dbias && p.M > 0) CHECK(inside(p.partial, (uint64_t)parts * (uint64_t)p.N * 4));
    if (p.dz && p.dbias) CHECK((char *)p.partial >= (char *)p.dz + (uint64_t)p.M * (uint64_t)round_up(p.N, 8) * 2);
    return g_result;
}
hipError_t launch_residual(const ResidualParams &p, hipStream_t) { ++g_launches; CHECK(p.M >= 1 && p.D >= 1 && p.groups >= 1 && p.M % p.groups == 0); return g_result; }
hipError_t launch_residual_backward(const ResidualParams &p, hipStream_t)
{
    ++g_launches;
    const ResidualRoom r = residual_room(p.M, p.D, p.groups);
    if (p.dgate || p.dpost_weight || p.dpost_bias || p.dpre_weight || p.dpre_bias) {
        if (r.total > 0) CHECK(inside(p.workspace, (uint64_t)r.total * 4));
        CHECK(r.sums >= p.groups * r.parts * 4 * p.D && (p.groups == 1 || r.totals >= p.groups * 4 * p.D) && (!residual_is_long(p.D) || r.rows >= 2 * p.M) && r.total == r.sums + r.totals + r.rows);
        if (p.M > 0) {
            const int64_t at_once = residual_is_long(p.D) ? 1 : kResidualThreads / residual_threads(p.D), rows = p.M / p.groups;
            CHECK(r.parts >= 1 && (rows + at_once * r.parts - 1) / (at_once * r.parts) <= 512);
        }
    }
    return g_result;
}
hipError_t launch_moe(const MoeParams &p, hipStream_t)
{
    ++g_launches;
    CHECK(p.M >= 1 && p.M <= kMoeTokens && p.E >= p.k && p.k >= 1 && p.k <= kMoeTopK && p.E <= kMoeExperts && p.shares >= 1 && p.shares <= 512);
    CHECK(inside(p.logits, (uint64_t)p.M * p.E * 8) && inside(p.plan, sizeof(MoePlan)) && inside(p.h, (uint64_t)p.M * p.k * p.F * 2));
    CHECK((char *)p.plan >= (char *)(p.logits + p.M * p.E) && (char *)p.h >= (char *)(p.plan + 1));
    if (p.shares > 1) CHECK(inside(p.partial, (uint64_t)p.shares * p.M * p.D * 4) && (char *)p.partial >= (char *)p.h + (uint64_t)p.M * p.k * p.F * 2);
    for (int rows : {16, 32}) CHECK(moe_segments(p.M, p.E, p.k, rows) <= kMoeSegments);
    return g_result;
}
}  // namespace atb

int main()
{
    alignas(256) static char room[256];
    char *a = room;
    g_work = reinterpret_cast<char *>((uintptr_t)1 << 50);                        // never touched
    const int64_t lengths[] = {INT64_MIN, -1, 0, 1, 2, 7, 8, 9, 24, 32, 33, 64, 100, 129, 257, 1000, 2600, 4096, 5001, 8192, 8193, 14336, 16384, 16385, 65536, (int64_t)1 << 20, ((int64_t)1 << 22) - 8, (int64_t)1 << 22,
                               (int64_t)1 << 23, ((int64_t)1 << 23) + 1, (int64_t)1 << 24, ((int64_t)1 << 24) + 1, (int64_t)1 << 40, INT64_MAX};
    int accepted = 0, refused = 0;
    auto count = [&](atb_status st) {
        g_result = g_result == hipSuccess ? hipErrorNoDevice : hipSuccess;
        (st == ATB_ERR_INVALID_ARG ? refused : accepted)++;
        CHECK(st == ATB_OK || st == ATB_ERR_INVALID_ARG || st == ATB_ERR_HIP);
    };

    for (int64_t M : lengths)
        for (int64_t N : lengths)
            for (int64_t K : lengths)
                for (atb_activation act : {ATB_ACT_GELU, ATB_ACT_NONE}) {
                    const size_t forward = atb_linear_workspace(M, N, K), backward = atb_linear_backward_workspace(M, N, K, act);
                    CHECK(forward <= (size_t)64 << 20 && forward % 16 == 0 && backward % 16 == 0);
                    for (int with = 0; with < 2; ++with) {
                        atb_linear l = {a, a, K, K, a, M, N, K, act, ATB_TYPE_F32, with ? g_work : nullptr};
                        g_bytes = with ? forward : 0;
                        count(atb_linear_forward(&l, a, N, act == ATB_ACT_NONE ? nullptr : a, a, N, nullptr));
                        count(atb_linear_forward(&l, nullptr, 0, nullptr, a, N, nullptr));
                        g_bytes = with ? backward : 0;
                        count(atb_linear_backward(&l, act == ATB_ACT_NONE ? nullptr : a, a, N, a, K, a, a, nullptr));
                        count(atb_linear_backward(&l, act == ATB_ACT_NONE ? nullptr : a, a, N, nullptr, K, a, nullptr, nullptr));
                        count(atb_linear_backward(&l, act == ATB_ACT_NONE ? nullptr : a, a, N, nullptr, K, nullptr, a, nullptr));
                    }
                }

    const atb_norm norms[] = {{nullptr, nullptr, 0.0, ATB_NORM_NONE}, {a, nullptr, 1e-5, ATB_NORM_RMS}, {a, a, 0.0, ATB_NORM_LAYER}, {a, a, -1.0, ATB_NORM_RMS}};
    for (int64_t M : lengths)
        for (int64_t D : lengths)
            for (int64_t groups : {INT64_MIN, (int64_t)0, (int64_t)1, (int64_t)2, (int64_t)8, (int64_t)4096, (int64_t)65535, (int64_t)65536, INT64_MAX}) {
                g_bytes = atb_residual_norm_workspace(M, D, groups);
                CHECK(g_bytes % 16 == 0);
                for (const atb_norm &post : norms)
                    for (const atb_norm &pre : norms) {
                        const atb_residual_norm p = {a, a, D, D, post, pre, a, groups, 0.5, M, D, ATB_TYPE_F32, ATB_TYPE_BF16, ATB_TYPE_BF16};
                        void *h = pre.kind == ATB_NORM_NONE ? nullptr : a;
                        count(atb_residual_norm_forward(&p, a, D, h, D, (float *)a, nullptr));
                        const atb_residual_norm_grads all = {a, a, D, D, a, post.kind ? a : nullptr, post.kind ? a : nullptr, h, h}, none = {a, a, D, D, nullptr, nullptr, nullptr, nullptr, nullptr};
                        count(atb_residual_norm_backward(&p, (float *)a, a, D, h, D, &all, g_work, nullptr));
                        count(atb_residual_norm_backward(&p, (float *)a, nullptr, 0, h, D, &none, nullptr, nullptr));
                    }
            }

    for (int64_t M : {INT64_MIN, (int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)17, (int64_t)64, (int64_t)65, INT64_MAX})
        for (int64_t D : lengths)
            for (int64_t F : lengths)
                for (int E : {INT32_MIN, 0, 1, 2, 60, 256, 257, INT32_MAX})
                    for (int k : {INT32_MIN, 0, 1, 2, 16, 17, INT32_MAX})
                        for (int group : {0, 32, 128, 48}) {
                            const atb_moe_weight w = {a, group ? a : nullptr, nullptr};
                            const atb_moe m = {a, a, D, D, w, w, w, M, D, F, E, k, group, ATB_ACT_SILU, 1, g_work};
                            g_bytes = atb_moe_workspace(M, D, F, E, k, group);
                            count(atb_moe_forward(&m, a, D, (int32_t *)a, (float *)a, nullptr));
                        }
    count(atb_linear_forward(nullptr, a, 8, a, a, 8, nullptr));
    count(atb_linear_backward(nullptr, a, a, 8, a, 8, a, a, nullptr));
    count(atb_residual_norm_forward(nullptr, a, 8, a, 8, nullptr, nullptr));
    count(atb_moe_forward(nullptr, a, 8, nullptr, nullptr, nullptr));
    CHECK(accepted > 1000 && refused > 1000 && g_launches > 1000);
    std::printf("sanitize_block: ok, %d calls accepted, %d refused, %d launches\n", accepted, refused, g_launches);
    return 0;
}
