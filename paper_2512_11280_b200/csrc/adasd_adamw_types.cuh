// AdamW over many tensors: what the entry point hands to the launcher (adasd_adamw.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/adasd.h"

namespace adasd {

constexpr int kAdBlock = ADASD_ADAMW_BLOCK;      // elements of a warp, and of a scale
constexpr int kAdThreads = 256;
constexpr int kAdRound = kAdThreads / 32 * kAdBlock;     // a CTA's warps, a block each

struct AdTensor {
    void* param;
    const void* grad;
    void* exp_avg;
    void* exp_avg_sq;
    float* avg_scale;
    float* sq_scale;
    void* param_copy;
    long long n;
    float weight_decay;
    int32_t first_item;                          // of the launch
    int32_t index;                               // in the call
    uint8_t kind, aligned;                       // 1: fp32 parameters, 2: fp32 gradients
};
// The tensors of a launch travel as its argument: nothing of them is kept on the device, and a graph holds its own copy.
template <int N>
struct AdTable {
    int32_t n, items, rounds;                    // an item: so many rounds of a CTA
    AdTensor t[N];
};
struct AdCoef {
    float rate, root;                            // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float lr, grad_scale;
    uint32_t step;
};
struct AdParams {
    AdCoef coef;
    float b1, b1c, b2, b2c, eps;                 // (b1c, b2c: 1 - b, rounded once)
    double lr, log_b1, log_b2;
    int32_t step;
    uint32_t seed;
    int32_t stochastic;
    const float* lr_dev;                         // nullable: these stand in for the host's values
    const float* grad_scale_dev;
    const int32_t* step_dev;
    uint32_t* status;
};

int launch_adamw(const AdParams& p, const adasd_adamw_tensor* tensors, int n, int sm_count, cudaStream_t stream);

}  // namespace adasd
