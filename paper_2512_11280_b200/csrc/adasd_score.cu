// Launches of the scoring and loss kernels (adasd_score.cuh).
#include "adasd_launch.cuh"
#include "adasd_score_deep.cuh"
#include "adasd_score_forward.cuh"

#include <algorithm>
#include <atomic>

namespace adasd {
namespace {

inline int unit_elements(int dtype) { return dtype == ADASD_BF16 ? 8 : 4; }
// How rows of logits, and of a gradient (null: none), lie relative to 16-byte boundaries.
inline Layout layout_of(const void* z, long long stride, const void* g, long long g_stride, int V, int dtype) {
    const int N = unit_elements(dtype);
    const uintptr_t a = reinterpret_cast<uintptr_t>(z) & 15u, b = g ? reinterpret_cast<uintptr_t>(g) & 15u : a;
    if (g && (a != b || (stride - g_stride) % N != 0)) return ROWS_ANY;
    return a == 0 && stride % N == 0 && V % N == 0 ? ROWS_WHOLE : ROWS_SAME;
}
// Units of a row, at most.
inline int row_units(int V, int dtype, Layout layout) {
    const int N = unit_elements(dtype);
    return (int)(((long long)V + (layout == ROWS_WHOLE ? 0 : 2 * N - 2)) / N);
}

template <typename K>
int resident_clusters(K kern, int threads, int smem, int cs) {
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)cs, 1, 1);
    lc.blockDim = dim3((unsigned)threads, 1, 1);
    lc.dynamicSmemBytes = (size_t)smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cs;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &lc) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return n;
}
// Clusters of a persistent kernel that are resident at once, asked for once per device and cluster size (0: not usable).
struct Resident {
    std::atomic<int> known[64][kScMaxCluster + 1];           // (0: not asked yet)
    template <typename K>
    int operator()(K kern, int threads, int smem, int cs) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
        int n = known[dev][cs].load(std::memory_order_acquire);
        if (n == 0) {
            n = resident_clusters(kern, threads, smem, cs);
            known[dev][cs].store(n > 0 ? n : -1, std::memory_order_release);
        }
        return std::max(n, 0);
    }
};
// A launch of a persistent kernel, a row a cluster at a time; kNotTaken unless there are more rows than clusters.  (score_kernel /
// score_deep_kernel from there on: 100 rows of 128256 bf16 18.9 / 16.5 us, 200 of 50256 18.2 / 15.1; 80 rows 15.8 / 15.3.)
constexpr int kNotTaken = 1;
template <typename K>
int launch_rows(Resident& resident, K kern, ScoreParams p, int threads, int smem, int cs, int per, cudaStream_t stream) {
    const long long ncl = resident(kern, threads, smem, cs);
    if (ncl == 0 || p.n_rows <= ncl) return kNotTaken;
    p.cs = cs;
    p.per_cta = per;
    return launch_pdl(kern, (int)ncl * cs, threads, smem, cs, stream, p);
}
// CTAs of a row: as many as make the last of the resident clusters' rounds end first, a CTA more costing a row 3 % more (an estimate:
// the exchange and shorter stretches; not measured by itself).
template <typename T, int L, int NW, bool ENT>
int launch_forward(ScoreParams p, int NU, int most, cudaStream_t stream) {
    static Resident r;
    const auto kern = score_forward_kernel<T, L, NW, ENT>;
    constexpr int smem = NW * kSfRingB;
    int best = 0, best_n = 0;
    double least = 0.0;
    for (int cs = 1; cs <= most; ++cs) {
        const int n = r(kern, NW * 32, smem, cs);
        if (n == 0) continue;
        const double t = (double)((p.n_rows + n - 1) / n) / cs * (1.0 + 0.03 * (cs - 1));
        if (best == 0 || t < least) {
            least = t;
            best = cs;
            best_n = n;
        }
    }
    if (best == 0) return kNotTaken;
    const int its = ((NU + 31) / 32 + NW * best - 1) / (NW * best);
    p.pieces = (its + kSfGroup - 1) / kSfGroup;
    p.per_cta = its * 32;
    p.cs = best;
    return launch_pdl(kern, std::min(best_n, p.n_rows) * best, NW * 32, smem, best, stream, p);
}
template <typename T, int L, int NW, bool ENT>
int launch_stream(const ScoreParams& p, int cs, int per, cudaStream_t stream) {
    static Resident r;
    return launch_rows(r, score_stream_kernel<T, L, NW, ENT>, p, NW * 32, NW * kSsStage, cs, per, stream);
}
template <typename T, int L, bool ENT>
int launch_deep(const ScoreParams& p, int cs, int per, cudaStream_t stream) {
    static Resident r;
    return launch_rows(r, score_deep_kernel<T, L, ENT>, p, kSdThreads, kSdSmem, cs, per, stream);
}
// Many rows.
// Without a gradient: score_forward_kernel, as soon as clusters of eight would fill the SMs twice.
// With one: score_deep_kernel, whose pipeline needs rows of 2048 units, where its stretches are about as full as
// score_stream_kernel's.  Deep / stream, us for 2000 rows: bf16 V=12000 30.5 / 24.3, 16384 36.1 / 35.1, 20000 40.9 / 45.0, 64000
// (80 and 98 % full) 103 / 100, 32000 (60 and 98 %) 61.6 / 55.0; 128256 (96 and 98 %, 2065 rows) 183 / 219; fp32 V=8200
// 28.6 / 33.1, 16000 47.9 / 53.5, 64000 183 / 191.  (One rule for both types, made for bf16: fp32 rows of 16000, which score_deep_kernel
// would do in less, go to the other.)
template <typename T, int L, bool ENT>
int launch_many(const ScoreParams& p, int NU, int sms, cudaStream_t stream) {
    if (!p.grad && (long long)p.n_rows * kScMaxCluster <= 2LL * sms) return kNotTaken;
    const int its = (NU + 31) / 32;
    if (p.grad && NU >= 2048) {
        constexpr int kStreamUnits = 8 * 32 * kSsUPT;        // of a CTA of score_stream_kernel
        const int cs = (NU + kSdUnits - 1) / kSdUnits, cs2 = (NU + kStreamUnits - 1) / kStreamUnits;
        if (cs <= kScMaxCluster && (cs2 > kScMaxCluster || 1.2 * cs2 * kStreamUnits >= 1.0 * cs * kSdUnits))
            if (const int rc = launch_deep<T, L, ENT>(p, cs, (its + cs - 1) / cs * 32, stream); rc != kNotTaken) return rc;
    }
    const int warps = (NU + kSsUPT * 32 - 1) / (kSsUPT * 32);
    auto launch = [&](auto nw, int cs) -> int {
        constexpr int NW = decltype(nw)::value;
        if (p.grad) return cs <= kScMaxCluster ? launch_stream<T, L, NW, ENT>(p, cs, (NU + NW * cs - 1) / (NW * cs), stream) : kNotTaken;
        return launch_forward<T, L, NW, ENT>(p, NU, NW == 8 ? kScMaxCluster : 1, stream);
    };
    if (warps == 1) return launch(std::integral_constant<int, 1>{}, 1);
    if (warps == 2) return launch(std::integral_constant<int, 2>{}, 1);
    if (warps <= 4) return launch(std::integral_constant<int, 4>{}, 1);
    return launch(std::integral_constant<int, 8>{}, (warps + 7) / 8);
}

constexpr int kScNW = 8, kScUnits = kScNW * 32;      // score_kernel: CTAs of 8 warps; units of a CTA and unit a thread

template <typename T, int L, bool GRAD, bool ENT>
int launch_few(ScoreParams p, int NU, int sms, cudaStream_t stream) {
    auto go = [&](auto kern, int threads) { return launch_pdl(kern, p.n_rows * p.cs, threads, 0, p.cs, stream, p); };
    if (NU <= 2 * 32 * 4) {
        p.cs = 1;
        p.per_cta = NU;
        return go(score_kernel<T, L, 2, 4, true, GRAD, ENT>, 64);
    }
    int cs = std::min(kScMaxCluster, (NU + kScUnits * 16 - 1) / (kScUnits * 16));
    while (cs < kScMaxCluster && (long long)p.n_rows * cs < 2LL * sms && NU > cs * kScUnits) cs = std::min(2 * cs, kScMaxCluster);
    p.cs = cs;
    p.per_cta = (NU + cs - 1) / cs;
    if (p.per_cta <= kScUnits * 4) return go(score_kernel<T, L, kScNW, 4, true, GRAD, ENT>, kScNW * 32);
    if (p.per_cta <= kScUnits * 8) return go(score_kernel<T, L, kScNW, 8, true, GRAD, ENT>, kScNW * 32);
    if (p.per_cta <= kScUnits * 16) return go(score_kernel<T, L, kScNW, 16, true, GRAD, ENT>, kScNW * 32);
    return go(score_kernel<T, L, kScNW, 16, false, GRAD, ENT>, kScNW * 32);
}
template <typename T, int L, bool ENT>
int launch(const ScoreParams& p, int NU, int sms, cudaStream_t stream) {
    if constexpr (L != ROWS_ANY)
        if (const int rc = launch_many<T, L, ENT>(p, NU, sms, stream); rc != kNotTaken) return rc;
    if (p.grad) return launch_few<T, L, true, ENT>(p, NU, sms, stream);
    if constexpr (L != ROWS_ANY) return launch_few<T, L, false, ENT>(p, NU, sms, stream);
    return ADASD_ERR_SHAPE;                          // (without a gradient no row lies across granules)
}
template <typename T, bool ENT>
int launch(const ScoreParams& p, int layout, int NU, int sms, cudaStream_t stream) {
    if (layout == ROWS_WHOLE) return launch<T, ROWS_WHOLE, ENT>(p, NU, sms, stream);
    if (layout == ROWS_SAME) return launch<T, ROWS_SAME, ENT>(p, NU, sms, stream);
    return launch<T, ROWS_ANY, ENT>(p, NU, sms, stream);
}
template <typename T>
int launch_grad(const PrefParams& p, int layout, int grid, cudaStream_t stream) {
    if (layout == ROWS_WHOLE) return launch_pdl(pref_grad_kernel<T, ROWS_WHOLE>, grid, kPgThreads, 0, 0, stream, p);
    if (layout == ROWS_SAME) return launch_pdl(pref_grad_kernel<T, ROWS_SAME>, grid, kPgThreads, 0, 0, stream, p);
    return launch_pdl(pref_grad_kernel<T, ROWS_ANY>, grid, kPgThreads, 0, 0, stream, p);
}

}  // namespace

int launch_score(const ScoreParams& p, int dtype, bool entropy, int sm_count, cudaStream_t stream) {
    const Layout layout = layout_of(p.z, p.row_stride, p.grad, p.g_stride, p.V, dtype);
    const int NU = row_units(p.V, dtype, layout);
    if (dtype == ADASD_BF16)
        return entropy ? launch<__nv_bfloat16, true>(p, layout, NU, sm_count, stream) : launch<__nv_bfloat16, false>(p, layout, NU, sm_count, stream);
    return entropy ? launch<float, true>(p, layout, NU, sm_count, stream) : launch<float, false>(p, layout, NU, sm_count, stream);
}

int launch_pref_pairs(const PrefParams& p, cudaStream_t stream) {
    if (p.loss && p.n_pairs <= kPairSum) {
        const int cs = std::min(8, p.n_pairs);
        return launch_pdl(pref_pair_kernel, cs, kPairThreads, 0, cs, stream, p, 1);
    }
    if (const int rc = launch_pdl(pref_pair_kernel, p.n_pairs, kPairThreads, 0, 1, stream, p, 0)) return rc;
    return p.loss ? launch_total(p.pair_loss, p.n_pairs, p.loss, stream) : ADASD_OK;
}

int launch_pref_grad(PrefParams p, int dtype, cudaStream_t stream) {
    const Layout layout = layout_of(p.z, p.row_stride, p.grad, p.g_stride, p.V, dtype);
    const int NU = row_units(p.V, dtype, layout);
    p.segs = (NU + kPgThreads * kPgUnits - 1) / (kPgThreads * kPgUnits);
    p.per_cta = (NU + p.segs - 1) / p.segs;
    if ((long long)p.n_rows * p.segs > 0x7FFFFFFFLL) return ADASD_ERR_SHAPE;
    return dtype == ADASD_BF16 ? launch_grad<__nv_bfloat16>(p, layout, p.n_rows * p.segs, stream) : launch_grad<float>(p, layout, p.n_rows * p.segs, stream);
}

int launch_total(const float* terms, int n, float* out, cudaStream_t stream) {
    return launch_pdl(total_kernel, 1, kTotThreads, 0, 0, stream, terms, n, out);
}

}  // namespace adasd
