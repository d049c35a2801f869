// Scoring and training from hidden states: what the entry points hand to the launchers (adasd_head.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/adasd.h"

namespace adasd {

constexpr int kHeadMaxV = 1 << 30;                   // (columns are counted in 32 bits, tiles beyond the last included)

enum HeadOp : int32_t {
    HEAD_LOGPROB,        // log-probs, entropies
    HEAD_GIVEN,          // gradients of a loss with given dL/dl, dL/dH
    HEAD_CE              // cross entropy, with or without gradients
};

struct HeadCall {
    int32_t op, n_rows, V, D;
    const void* hidden;
    long long h_stride;
    const void* weight;
    long long w_stride;
    const int32_t* tok;
    float temperature;
    uint32_t* status;
    void* scratch;
    float* logp;                                   // outputs [n_rows], nullable
    float* H;
    float* lse;
    const float* lse_in;                           // HEAD_GIVEN; H_in, g_H nullable
    const float* H_in;
    const float* g_logp;
    const float* g_H;
    const float* row_weight;                       // HEAD_CE; nullable
    float smoothing, z_loss, scale;
    float* row_loss;
    float* loss;                                   // nullable [1]
    void* grad_h;                                  // nullable
    long long gh_stride;
    void* grad_w;                                  // nullable
    long long gw_stride;
    int32_t sm_count;
    bool gradient() const { return grad_h || grad_w; }
};

// Bytes of scratch that a call of n_rows rows needs, and that serve calls of any number up to n_rows.
size_t head_scratch_need(int n_rows, int V, int D, bool gradient, int sm_count);
size_t head_scratch_bytes(int n_rows, int V, int D, bool gradient, int sm_count);
// The launches of a call.  Returns ADASD_OK or a code of the header.
int launch_head(const HeadCall& c, cudaStream_t stream);

}  // namespace adasd
