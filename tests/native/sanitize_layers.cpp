// Host program of the sanitizer build: the argument handling of the feed-forward sublayer's operators (atb_layers_api.cpp) and the rules that choose
// tiles and sizes of workspaces (atb_layers.h), with the launches replaced by ones that check what they are given; in every other call they fail, as without a GPU.
#include "atb.h"
#include "atb_layers.h"

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#define CHECK(x) do { if (!(x)) { std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

namespace {

size_t g_workspace = 0;          // bytes of the buffer behind TileParams::shares and NormParams::partial
int g_launches = 0;
hipError_t g_result = hipSuccess;

hipError_t tiles(const atb::TileParams &p, bool gated)
{
    ++g_launches;
    CHECK(p.M >= 1 && p.N >= 1 && p.K >= 0 && p.segments >= 1 && p.problems >= 1);
    const atb::TileChoice how = atb::choose_tiles(p.M, p.N, p.K, p.segments, p.problems, gated, p.shares != nullptr);
    CHECK(how.parts >= 1 && (how.parts == 1 || p.shares));
    CHECK(!(gated && how.large && how.parts > 1));
    if (how.parts > 1) {
        CHECK((uint64_t)how.parts * (gated ? 2 : p.problems) * (uint64_t)p.M * (uint64_t)p.N * 4 <= g_workspace);
        CHECK((int64_t)p.M * (p.N / 4) < (int64_t)1 << 31);                       // the join's index
        CHECK((int64_t)((p.K + 63) / 64) * p.segments >= how.parts);              // no empty share
    }
    return g_result;
}

}  // namespace

namespace atb {
hipError_t launch_norm(const NormParams &p, hipStream_t) { ++g_launches; CHECK(p.M >= 1 && p.D >= 1); return g_result; }
hipError_t launch_norm_backward(const NormParams &p, hipStream_t)
{
    ++g_launches;
    if (p.dweight || p.dbias) CHECK((uint64_t)norm_partials(p.M, p.D) * 2 * (uint64_t)p.D * 4 <= g_workspace);
    return g_result;
}
hipError_t launch_tiles_forward(TileParams p, int epilogue, hipStream_t) { return tiles(p, is_gated(epilogue)); }
hipError_t launch_tiles_dx(TileParams p, int, hipStream_t) { return tiles(p, false); }
hipError_t launch_tiles_dw(TileParams p, hipStream_t) { return tiles(p, false); }
hipError_t launch_stream(const StreamParams &p, hipStream_t) { ++g_launches; CHECK(p.M >= 1 && p.N >= 1 && p.K >= 1); return g_result; }
hipError_t launch_q4_quantize(const void *, int, int64_t, uint8_t *, uint16_t *, uint8_t *, int64_t, int64_t, int, hipStream_t) { ++g_launches; return g_result; }
hipError_t launch_q4_decode(const uint8_t *, const uint16_t *, const uint8_t *, void *, int, int64_t, int64_t, int, hipStream_t) { ++g_launches; return g_result; }
}  // namespace atb

int main()
{
    alignas(256) static char room[256];
    char *a = room;
    const int64_t lengths[] = {INT64_MIN, -1, 0, 1, 7, 8, 24, 33, 64, 100, 128, 129, 257, 1000, 2600, 4096, 8192, 14336, 65535, 65536, (int64_t)1 << 20, ((int64_t)1 << 22) - 8, (int64_t)1 << 22,
                               (int64_t)1 << 23, ((int64_t)1 << 23) + 1, (int64_t)1 << 24, ((int64_t)1 << 24) + 1, (int64_t)1 << 40, INT64_MAX};
    int accepted = 0, refused = 0;
    auto count = [&](atb_status st) {
        g_result = g_result == hipSuccess ? hipErrorNoDevice : hipSuccess;
        (st == ATB_ERR_INVALID_ARG ? refused : accepted)++; CHECK(st == ATB_OK || st == ATB_ERR_INVALID_ARG || st == ATB_ERR_HIP);
    };

    for (int64_t M : lengths)
        for (int64_t D : lengths) {
            g_workspace = atb_layer_norm_workspace(M, D);
            const bool valid = M >= 0 && M <= ((int64_t)1 << 23) && D >= 1 && D <= ((int64_t)1 << 24);
            CHECK(valid ? (g_workspace > 0) == (M > 0) : g_workspace == 0);
            if (valid && M > 0) {
                const int64_t partials = atb::norm_partials(M, D), rows = D > atb::kNormMaxGradRow ? 1 : atb::kNormGradThreads / atb::norm_threads(D);
                CHECK(partials >= 1 && partials <= 65535 && g_workspace == (uint64_t)partials * 2 * (uint64_t)D * 4);
                CHECK((M + rows * partials - 1) / (rows * partials) <= 512);
            }
            for (int type = -1; type <= 2; ++type) {
                count(atb_layer_norm(a, D, a, a, 1e-5, a, D, (float *)a, (float *)a, M, D, (atb_type)type, ATB_TYPE_F32, nullptr));
                count(atb_layer_norm_backward(a, D, a, D, (float *)a, (float *)a, a, a, D, a, a, a, M, D, (atb_type)type, ATB_TYPE_BF16, nullptr));
            }
        }

    for (int64_t M : lengths)
        for (int64_t D : lengths)
            for (int64_t F : lengths) {
                const size_t forward = atb_ffn_workspace(M, D, F, 0), keeps = atb_ffn_workspace(M, D, F, 1), backward = atb_ffn_backward_workspace(M, D, F);
                CHECK(forward <= keeps && keeps <= (size_t)64 << 20 && backward <= (size_t)64 << 20);
                const size_t kept = atb_ffn_kept_bytes(M, F);
                CHECK(kept == 0 || kept == 6 * (uint64_t)M * (uint64_t)F);
                for (int with = 0; with < 4; ++with) {
                    const atb_ffn f = {a, a, a, a, D, D, D, F, M, D, F, ATB_ACT_GELU, with & 1 ? a : nullptr};
                    g_result = with & 2 ? hipErrorNoDevice : hipSuccess;
                    g_workspace = with & 1 ? forward : 0;
                    count(atb_ffn_forward(&f, a, nullptr, a, D, nullptr));
                    g_workspace = with & 1 ? keeps : 0;
                    count(atb_ffn_forward(&f, a, a, a, D, nullptr));
                    g_workspace = with & 1 ? backward : 0;
                    count(atb_ffn_backward(&f, a, a, a, D, a, a, a, D, a, a, a, nullptr));
                    count(atb_ffn_backward(&f, a, a, a, D, a, a, nullptr, D, a, a, nullptr, nullptr));
                    count(atb_ffn_backward(&f, a, a, a, D, a, a, nullptr, D, nullptr, nullptr, a, nullptr));
                }
            }

    for (int64_t N : lengths)
        for (int64_t K : lengths)
            for (int group : {-32, 0, 16, 32, 64, 128, 256, INT32_MAX})
                for (int64_t M : {INT64_MIN, (int64_t)0, (int64_t)1, (int64_t)17, (int64_t)1 << 23, INT64_MAX}) {
                    const atb_q4 w = {a, a, nullptr, N, K, group};
                    count(atb_q4_matvec(&w, a, K, a, N, ATB_TYPE_F32, M, nullptr));
                    count(atb_q4_gated(&w, &w, ATB_ACT_SILU, a, K, a, N, M, nullptr));
                    if (M == 1) {
                        count(atb_q4_quantize(a, K, ATB_TYPE_BF16, a, a, a, N, K, group, nullptr));
                        count(atb_q4_decode(&w, a, ATB_TYPE_F32, nullptr));
                    }
                }
    count(atb_ffn_forward(nullptr, a, a, a, 8, nullptr));
    count(atb_q4_matvec(nullptr, a, 64, a, 4, ATB_TYPE_F32, 1, nullptr));
    count(atb_q4_decode(nullptr, a, ATB_TYPE_F32, nullptr));
    CHECK(accepted > 1000 && refused > 1000 && g_launches > 1000);
    std::printf("sanitize_layers: ok, %d calls accepted, %d refused, %d launches\n", accepted, refused, g_launches);
    return 0;
}
