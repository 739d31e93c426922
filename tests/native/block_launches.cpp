// The kernel launches of a block's operators (atb_block_api.cpp), recorded on the host: this program defines the runtime's launch calls itself, so that no GPU is needed and nothing runs.
// block_launches <operator> <sizes ..> makes one call with made-up addresses and prints a line per launch, its workgroups and threads in x and y, and then the call's status.
#include "atb.h"

#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <string>

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
extern "C" hipError_t hipLaunchKernel(const void *, dim3 grid, dim3 block, void **, size_t, hipStream_t)
{
    std::printf("launch %u %u %u %u\n", grid.x, grid.y, block.x, block.y);
    return hipSuccess;
}

int main(int argc, char **argv)
{
    if (argc < 2) return 2;
    const std::string op = argv[1];
    int64_t v[8] = {};
    for (int i = 2; i < argc && i < 10; ++i) v[i - 2] = std::atoll(argv[i]);
    auto at = [](int64_t n) { return reinterpret_cast<void *>(n << 40); };
    int st = -1;
    if (op == "linear" || op == "linear_backward") {          // M, N, K, activation, whether there is a workspace, and residual and slope or the gradients asked for
        const atb_linear l = {at(1), at(2), v[2], v[2], at(3), v[0], v[1], v[2], (atb_activation)v[3], ATB_TYPE_BF16, v[4] ? at(4) : nullptr};
        void *slope = v[5] && v[3] != ATB_ACT_NONE ? at(5) : nullptr;
        if (op == "linear") st = atb_linear_forward(&l, v[5] ? at(6) : nullptr, v[1], slope, at(7), v[1], nullptr);
        else st = atb_linear_backward(&l, slope, at(6), v[1], v[6] & 1 ? at(7) : nullptr, v[2], v[6] & 2 ? at(8) : nullptr, v[6] & 4 ? at(9) : nullptr, nullptr);
    } else if (op == "residual" || op == "residual_backward") {      // M, D, groups, kinds of the norms, type of the stream, whether the parameters' gradients are asked for
        const atb_norm post = {v[3] ? at(1) : nullptr, v[3] == ATB_NORM_LAYER ? at(2) : nullptr, 1e-5, (atb_norm_kind)v[3]}, pre = {v[4] ? at(3) : nullptr, v[4] == ATB_NORM_LAYER ? at(4) : nullptr, 1e-5, (atb_norm_kind)v[4]};
        const atb_residual_norm p = {at(5), at(6), v[1], v[1], post, pre, at(7), v[2], 1.0, v[0], v[1], (atb_type)v[5], (atb_type)v[5], ATB_TYPE_BF16};
        void *h = v[4] ? at(8) : nullptr;
        if (op == "residual") st = atb_residual_norm_forward(&p, at(9), v[1], h, v[1], static_cast<float *>(at(10)), nullptr);
        else {
            auto asked = [&](bool there, int n) { return v[6] && there ? at(n) : nullptr; };
            const atb_residual_norm_grads g = {at(11), at(12), v[1], v[1], asked(true, 13), asked(v[3] != 0, 14), asked(v[3] == ATB_NORM_LAYER, 15), asked(v[4] != 0, 16), asked(v[4] == ATB_NORM_LAYER, 17)};
            st = atb_residual_norm_backward(&p, static_cast<float *>(at(10)), at(9), v[1], h, v[1], &g, at(18), nullptr);
        }
    } else if (op == "moe") {                                 // M, D, F, experts, top_k, group
        const atb_moe_weight w = {at(1), v[5] ? at(2) : nullptr, nullptr};
        const atb_moe m = {at(3), at(4), v[1], v[1], w, w, w, v[0], v[1], v[2], (int)v[3], (int)v[4], (int)v[5], ATB_ACT_SILU, 1, at(5)};
        st = atb_moe_forward(&m, at(6), v[1], static_cast<int32_t *>(at(7)), static_cast<float *>(at(8)), nullptr);
    }
    std::printf("status %d\n", st);
    return 0;
}
