// Launches of the scoring and loss kernels (adasd_score.cuh).
#include "adasd_launch.cuh"
#include "adasd_score.cuh"

#include <algorithm>

namespace adasd {
namespace {

inline bool aligned_rows(const void* base, long long stride, int dtype) {
    return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && (stride * (dtype == ADASD_BF16 ? 2 : 4)) % 16 == 0;
}
// Units of a row, at most.
inline int row_units(int V, int dtype, bool aligned) {
    const int N = dtype == ADASD_BF16 ? 8 : 4;
    return (int)(((long long)V + (aligned ? N - 1 : 2 * N - 2)) / N);
}

template <typename T, bool ALIGNED, int NW, int UPT, bool HOLD, bool GRAD, bool ENT>
int launch(const ScoreParams& p, cudaStream_t stream) {
    return launch_pdl(score_kernel<T, ALIGNED, NW, UPT, HOLD, GRAD, ENT>, p.n_rows * p.cs, NW * 32, 0, p.cs, stream, p);
}
template <typename T, bool ALIGNED, int NW, int UPT, bool HOLD>
int launch(const ScoreParams& p, bool ent, cudaStream_t stream) {
    if (p.grad) return ent ? launch<T, ALIGNED, NW, UPT, HOLD, true, true>(p, stream) : launch<T, ALIGNED, NW, UPT, HOLD, true, false>(p, stream);
    return ent ? launch<T, ALIGNED, NW, UPT, HOLD, false, true>(p, stream) : launch<T, ALIGNED, NW, UPT, HOLD, false, false>(p, stream);
}

constexpr int kScNW = 8, kScUnits = kScNW * 32;      // CTAs of 8 warps; units of a CTA and unit a thread

template <typename T, bool ALIGNED>
int launch(ScoreParams p, bool ent, int NU, int sms, cudaStream_t stream) {
    if (NU <= 2 * 32 * 4) {
        p.cs = 1;
        p.per_cta = NU;
        return launch<T, ALIGNED, 2, 4, true>(p, ent, stream);
    }
    int cs = std::min(kScMaxCluster, (NU + kScUnits * 16 - 1) / (kScUnits * 16));
    while (cs < kScMaxCluster && (long long)p.n_rows * cs < 2LL * sms && NU > cs * kScUnits) cs = std::min(2 * cs, kScMaxCluster);
    p.cs = cs;
    p.per_cta = (NU + cs - 1) / cs;
    if (p.per_cta <= kScUnits * 4) return launch<T, ALIGNED, kScNW, 4, true>(p, ent, stream);
    if (p.per_cta <= kScUnits * 8) return launch<T, ALIGNED, kScNW, 8, true>(p, ent, stream);
    if (p.per_cta <= kScUnits * 16) return launch<T, ALIGNED, kScNW, 16, true>(p, ent, stream);
    return launch<T, ALIGNED, kScNW, 16, false>(p, ent, stream);
}

}  // namespace

int launch_score(ScoreParams p, int dtype, bool entropy, int sm_count, cudaStream_t stream) {
    const bool al = aligned_rows(p.z, p.row_stride, dtype) && (!p.grad || aligned_rows(p.grad, p.g_stride, dtype));
    const int NU = row_units(p.V, dtype, al);
    if (dtype == ADASD_BF16)
        return al ? launch<__nv_bfloat16, true>(p, entropy, NU, sm_count, stream) : launch<__nv_bfloat16, false>(p, entropy, NU, sm_count, stream);
    return al ? launch<float, true>(p, entropy, NU, sm_count, stream) : launch<float, false>(p, entropy, NU, sm_count, stream);
}

int launch_pref_pairs(const PrefParams& p, cudaStream_t stream) {
    return launch_pdl(pref_pair_kernel, p.n_pairs, kPairThreads, 0, 0, stream, p);
}

int launch_pref_grad(PrefParams p, int dtype, cudaStream_t stream) {
    const bool al = aligned_rows(p.z, p.row_stride, dtype) && aligned_rows(p.grad, p.g_stride, dtype);
    const int NU = row_units(p.V, dtype, al);
    p.segs = (NU + kPgThreads * kPgUnits - 1) / (kPgThreads * kPgUnits);
    p.per_cta = (NU + p.segs - 1) / p.segs;
    if ((long long)p.n_rows * p.segs > 0x7FFFFFFFLL) return ADASD_ERR_SHAPE;
    const int grid = p.n_rows * p.segs;
    if (dtype == ADASD_BF16)
        return al ? launch_pdl(pref_grad_kernel<__nv_bfloat16, true>, grid, kPgThreads, 0, 0, stream, p)
                  : launch_pdl(pref_grad_kernel<__nv_bfloat16, false>, grid, kPgThreads, 0, 0, stream, p);
    return al ? launch_pdl(pref_grad_kernel<float, true>, grid, kPgThreads, 0, 0, stream, p)
              : launch_pdl(pref_grad_kernel<float, false>, grid, kPgThreads, 0, 0, stream, p);
}

int launch_total(const float* terms, int n, float* out, cudaStream_t stream) {
    return launch_pdl(total_kernel, 1, kTotThreads, 0, 0, stream, terms, n, out);
}

}  // namespace adasd
