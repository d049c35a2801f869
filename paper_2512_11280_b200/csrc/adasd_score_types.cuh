// Scoring and losses of given tokens: what the entry points hand to the launchers (adasd_score.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/adasd.h"

namespace adasd {

enum ScoreOp : int32_t {
    SCORE_LOGPROB,       // log-probs, entropies
    SCORE_GIVEN,         // gradient of a loss with given dL/dl, dL/dH
    SCORE_POLICY,        // clipped policy loss
    SCORE_PREF           // statistics of the rows of a preference loss
};

// What the preference loss keeps of a row between its launches (the caller's scratch).
struct __align__(16) PrefRow {
    float m, S;          // largest logit, sum 2^((z - m) log2 e / T)
    float dz;            // z[x] - m; from pref_pair_kernel on: the row's dL/dl
    int32_t kind;        // -1: in no sequence, 0: left out (gradient of zeros), 1: counted
};

struct ScoreParams {
    const void* z;
    long long row_stride;
    const int32_t* tok;
    void* grad;                                    // nullable
    long long g_stride;
    int32_t n_rows, V, op;
    int32_t cs, per_cta, pieces;                   // CTAs per row; 16-byte units of a CTA (or a warp), in pieces
    float c1;                                      // log2 e / temperature
    double inv_temp;
    uint32_t* status;
    float* logp;                                   // [n_rows] outputs, nullable
    float* H;
    float* lse;
    const float* g_logp;                           // SCORE_GIVEN; g_H nullable
    const float* g_H;
    const float* adv;                              // SCORE_POLICY
    const float* old_logp;                         // nullable
    const float* ref_logp;                         // nullable
    const float* weight;                           // nullable
    float clip_low, clip_high, kl_coef, ent_coef, scale;
    float* row_loss;
    float* kl;                                     // nullable
    const int32_t* seq_start;                      // SCORE_PREF
    PrefRow* pref;
    int32_t n_seqs;
};

struct PrefParams {
    const void* z;
    long long row_stride;
    const int32_t* tok;
    void* grad;                                    // nullable
    long long g_stride;
    int32_t n_rows, V, n_pairs;
    int32_t segs, per_cta;                         // CTAs per row; 16-byte units of a CTA
    float temperature, c1;
    const int32_t* seq_start;                      // [2 n_pairs + 1]
    const float* ref_logp;                         // nullable [2 n_pairs]
    const float* pair_weight;                      // nullable [n_pairs]
    int32_t rule, average;
    float beta, margin, label_smoothing, scale;
    PrefRow* pref;                                 // [n_rows]
    float* seq_logp;                               // [2 n_pairs]
    float* pair_loss;                              // [n_pairs]
    float* loss;                                   // nullable
};

// All return ADASD_OK or a code of the header.  entropy: the call needs H or its gradient.
int launch_score(const ScoreParams& p, int dtype, bool entropy, int sm_count, cudaStream_t stream);
int launch_pref_pairs(const PrefParams& p, cudaStream_t stream);     // (the total too)
int launch_pref_grad(PrefParams p, int dtype, cudaStream_t stream);
int launch_total(const float* terms, int n, float* out, cudaStream_t stream);

}  // namespace adasd
