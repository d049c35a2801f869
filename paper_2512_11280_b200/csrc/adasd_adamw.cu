// Launches of the AdamW step (adasd_adamw.cuh).
#include "adasd_adamw.cuh"
#include "adasd_launch.cuh"

#include <algorithm>
#include <cstring>

namespace adasd {
namespace {

constexpr int kAdFew = 24, kAdMany = 384;        // tensors of a launch: 2 and 32 KB of arguments

template <int N>
int launch_table(const AdParams& p, const AdTable<N>& table, int sm_count, cudaStream_t stream) {
    return launch_pdl(adamw_kernel<N>, table.items, kAdThreads, 0, 0, stream, p, table);
}

inline bool at(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <int N>
int launch_all(const AdParams& p, const adasd_adamw_tensor* in, int n, int sm_count, cudaStream_t stream) {
    AdTable<N> table;
    table.n = table.items = 0;
    for (int k = 0; k < n; ++k) {
        const adasd_adamw_tensor& s = in[k];
        // tensors larger than a launch's items can count are cut: 2^30 items are 2^41 elements, more than the device holds
        const long long items = (s.n + kAdItem - 1) / kAdItem;
        if (items > (1 << 30)) return ADASD_ERR_SHAPE;
        if (table.n == N || (long long)table.items + items > 0x7FFFFFFFLL) {
            if (const int rc = launch_table(p, table, sm_count, stream)) return rc;
            table.n = table.items = 0;
        }
        if (items == 0) continue;
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
        t.kind = (uint8_t)((s.param_dtype == ADASD_FP32 ? 1 : 0) | (s.grad_dtype == ADASD_FP32 ? 2 : 0) | (s.state_bits == 8 ? 4 : 0));
        const uintptr_t states = s.state_bits == 8 ? 8 : 16;
        t.aligned = at(s.param, 16) && at(s.grad, 16) && at(s.param_copy, 16) && at(s.exp_avg, states) && at(s.exp_avg_sq, states);
        table.items += (int32_t)items;
    }
    return table.items > 0 ? launch_table(p, table, sm_count, stream) : ADASD_OK;
}

}  // namespace

int launch_adamw(const AdParams& p, const adasd_adamw_tensor* tensors, int n, int sm_count, cudaStream_t stream) {
    return n <= kAdFew ? launch_all<kAdFew>(p, tensors, n, sm_count, stream) : launch_all<kAdMany>(p, tensors, n, sm_count, stream);
}

}  // namespace adasd
