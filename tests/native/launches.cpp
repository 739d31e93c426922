// The kernel launches of libatb's feed-forward operators, recorded on the host: this program defines the runtime's launch calls itself, so that
// no GPU is needed and nothing runs.  launches <operator> <sizes ..> makes one call with made-up addresses and prints its status, then a
// line per launch: workgroups and threads in x and y, and the rows that it takes, from the addresses in its arguments.
#include "atb.h"
#include "atb_layers.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

namespace {

std::string g_operator;
const int64_t kX = (int64_t)1 << 40, kY = (int64_t)1 << 42, kZ = (int64_t)1 << 44, kW = (int64_t)1 << 45, kMean = (int64_t)1 << 46, kRstd = (int64_t)3 << 46;

void *at(int64_t address) { return reinterpret_cast<void *>(address); }
long long off(const void *p, int64_t base) { return (long long)(reinterpret_cast<int64_t>(p) - base); }
template <class T> T argument(void **args, int i) { return *static_cast<T *>(args[i]); }

}  // namespace

static struct { dim3 grid, block; size_t lds; hipStream_t stream; } g_configuration;

extern "C" hipError_t hipGetLastError(void) { return hipSuccess; }
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    g_configuration = {grid, block, lds, stream};
    return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = g_configuration.grid;
    *block = g_configuration.block;
    *lds = g_configuration.lds;
    *stream = g_configuration.stream;
    return hipSuccess;
}
extern "C" hipError_t hipLaunchKernel(const void *, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    std::printf("launch %u %u %u %u", grid.x, grid.y, block.x, block.y);
    if (g_operator == "norm") {
        const auto &p = *static_cast<const atb::NormParams *>(args[0]);
        std::printf(" rows %lld x %lld y %lld mean %lld rstd %lld", (long long)p.M, off(p.x, kX), off(p.y, kY), off(p.mean, kMean), off(p.rstd, kRstd));
    } else if (g_operator == "norm_backward") {
        const auto &p = *static_cast<const atb::NormParams *>(args[0]);
        std::printf(" rows %lld x %lld dy %lld dx %lld mean %lld rstd %lld", (long long)p.M, off(p.x, kX), off(p.dy, kY), off(p.dx, kZ), off(p.mean, kMean), off(p.rstd, kRstd));
    } else if (g_operator == "q4" || g_operator == "q4_gated") {
        const auto &p = *static_cast<const atb::StreamParams *>(args[0]);
        std::printf(" rows %lld x %lld y %lld", (long long)p.M, off(p.x, kX), off(p.y, kY));
    } else if (g_operator == "ffn" || g_operator == "ffn_backward") {
        const auto &p = *static_cast<const atb::TileParams *>(args[0]);
        std::printf(" m %d n %d k %d parts %d planes %d", p.M, p.N, p.K * p.segments, p.parts, p.planes);
    } else if (g_operator == "q4_quantize") {      // w, ldw, packed, scales, zeros, N, K
        std::printf(" rows %lld w %lld packed %lld scales %lld zeros %lld", (long long)argument<int64_t>(args, 5), off(argument<void *>(args, 0), kX), off(argument<void *>(args, 2), kY),
                    off(argument<void *>(args, 3), kZ), off(argument<void *>(args, 4), kW));
    } else if (g_operator == "q4_decode") {        // packed, scales, zeros, out, N, K, group
        std::printf(" rows %lld packed %lld scales %lld zeros %lld out %lld", (long long)argument<int64_t>(args, 4), off(argument<void *>(args, 0), kY), off(argument<void *>(args, 1), kZ),
                    off(argument<void *>(args, 2), kW), off(argument<void *>(args, 3), kX));
    }
    std::printf("\n");
    return hipSuccess;
}

int main(int argc, char **argv)
{
    if (argc < 2) return 2;
    g_operator = argv[1];
    int64_t v[8] = {};
    for (int i = 2; i < argc && i < 10; ++i) v[i - 2] = std::atoll(argv[i]);
    int st = -1;
    if (g_operator == "norm")                  // M, D, type, pitch of x, pitch of y
        st = atb_layer_norm(at(kX), v[3], at(kW), at(kW), 1e-5, at(kY), v[4], static_cast<float *>(at(kMean)), static_cast<float *>(at(kRstd)), v[0], v[1], (atb_type)v[2], (atb_type)v[2], nullptr);
    else if (g_operator == "norm_backward")    // M, D, type, pitch of x, pitch of dy, pitch of dx, whether the parameters' gradients are asked for
        st = atb_layer_norm_backward(at(kY), v[4], at(kX), v[3], static_cast<float *>(at(kMean)), static_cast<float *>(at(kRstd)), at(kW), at(kZ), v[5], v[6] ? at(kW) : nullptr,
                                     v[6] ? at(kW) : nullptr, v[6] ? at(kW) : nullptr, v[0], v[1], (atb_type)v[2], (atb_type)v[2], nullptr);
    else if (g_operator == "q4") {             // M, N, K, group, type of y, pitch of x, pitch of y
        const atb_q4 w = {at(kW), at(kW), at(kW), v[1], v[2], (int)v[3]};
        st = atb_q4_matvec(&w, at(kX), v[5], at(kY), v[6], (atb_type)v[4], v[0], nullptr);
    } else if (g_operator == "q4_gated") {     // M, N, K, group, pitch of x, pitch of h
        const atb_q4 w = {at(kW), at(kW), nullptr, v[1], v[2], (int)v[3]};
        st = atb_q4_gated(&w, &w, ATB_ACT_SILU, at(kX), v[4], at(kY), v[5], v[0], nullptr);
    }
    else if (g_operator == "q4_quantize")      // N, K, group, type, pitch
        st = atb_q4_quantize(at(kX), v[4], (atb_type)v[3], at(kY), at(kZ), at(kW), v[0], v[1], (int)v[2], nullptr);
    else if (g_operator == "q4_decode") {      // N, K, group, type
        const atb_q4 w = {at(kY), at(kZ), at(kW), v[0], v[1], (int)v[2]};
        st = atb_q4_decode(&w, at(kX), (atb_type)v[3], nullptr);
    }
    else if (g_operator == "ffn" || g_operator == "ffn_backward") {      // M, D, F, whether there is a workspace, whether the forward pass keeps what the backward pass needs
        const atb_ffn f = {at(kX), at(kW), at(kW), at(kW), v[1], v[1], v[1], v[2], v[0], v[1], v[2], ATB_ACT_SILU, v[3] ? at(kZ) : nullptr};
        if (g_operator == "ffn") st = atb_ffn_forward(&f, at(kY), v[4] ? at(kMean) : nullptr, at(kY), v[1], nullptr);
        else st = atb_ffn_backward(&f, at(kY), at(kMean), at(kY), v[1], at(kW), at(kW), at(kX), v[1], at(kW), at(kW), at(kW), nullptr);
    }
    std::printf("status %d\n", st);
    return 0;
}
