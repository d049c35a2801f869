// Launches of the AdamW step (adasd_adamw.cuh).
#include "adasd_adamw.cuh"
#include "adasd_launch.cuh"

#include <algorithm>
#include <cstring>

namespace adasd {
namespace {

constexpr int kAdFew = 24, kAdMany = 384;        // tensors of a launch: 2 and 32 KB of arguments

inline bool at(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The tensors with states in 8 bits (EIGHT) or in 32.
template <int N, bool EIGHT>
int launch_all(const AdParams& p, const adasd_adamw_tensor* in, int n, int sm_count, cudaStream_t stream) {
    AdTable<N> table;
    table.n = table.items = 0;
    // Rounds of an item: up to 8, as long as there are 16 items for every SM.
    long long all = 0;
    for (int k = 0; k < n; ++k)
        if ((in[k].state_bits == 8) == EIGHT) all += (in[k].n + kAdRound - 1) / kAdRound;
    if (all == 0) return ADASD_OK;
    table.rounds = (int)std::max<long long>(1, std::min<long long>(8, all / (16LL * sm_count)));
    const long long item = (long long)table.rounds * kAdRound;
    auto launch = [&] {
        if constexpr (EIGHT) return launch_pdl(adamw8_kernel<N>, table.items, kAdThreads, 0, 0, stream, p, table);
        else return launch_pdl(adamw_kernel<N>, table.items, kAdThreads, 0, 0, stream, p, table);
    };
    for (int k = 0; k < n; ++k) {
        const adasd_adamw_tensor& s = in[k];
        const long long items = (s.n + item - 1) / item;
        if ((s.state_bits == 8) != EIGHT || items == 0) continue;
        if (table.n == N || table.items + items > 0x7FFFFFFFLL) {        // (a tensor by itself has up to 2^40 elements, 2^29 items)
            if (const int rc = launch()) return rc;
            table.n = table.items = 0;
        }
        AdTensor& t = table.t[table.n++];
        t.param = s.param;
        t.grad = s.grad;
        t.exp_avg = s.exp_avg;
        t.exp_avg_sq = s.exp_avg_sq;
        t.avg_scale = s.avg_scale;
        t.sq_scale = s.sq_scale;
        t.param_copy = s.param_copy;
        t.n = s.n;
        t.weight_decay = s.weight_decay;
        t.first_item = table.items;
        t.index = k;
        t.kind = (uint8_t)((s.param_dtype == ADASD_FP32 ? 1 : 0) | (s.grad_dtype == ADASD_FP32 ? 2 : 0));
        const uintptr_t states = EIGHT ? 8 : 16;
        t.aligned = at(s.param, 16) && at(s.grad, 16) && at(s.param_copy, 16) && at(s.exp_avg, states) && at(s.exp_avg_sq, states);
        table.items += (int32_t)items;
    }
    return launch();
}
template <int N>
int launch_all(const AdParams& p, const adasd_adamw_tensor* tensors, int n, int sm_count, cudaStream_t stream) {
    if (const int rc = launch_all<N, true>(p, tensors, n, sm_count, stream)) return rc;
    return launch_all<N, false>(p, tensors, n, sm_count, stream);
}

}  // namespace

int launch_adamw(const AdParams& p, const adasd_adamw_tensor* tensors, int n, int sm_count, cudaStream_t stream) {
    return n <= kAdFew ? launch_all<kAdFew>(p, tensors, n, sm_count, stream) : launch_all<kAdMany>(p, tensors, n, sm_count, stream);
}

}  // namespace adasd
