// Launches of the scoring and loss kernels (adasd_score.cuh).
#include "adasd_launch.cuh"
#include "adasd_score_deep.cuh"

#include <algorithm>
#include <atomic>

namespace adasd {
namespace {

inline int unit_elements(int dtype) { return dtype == ADASD_BF16 ? 8 : 4; }
// Rows that start on 16-byte boundaries and end on one.
inline bool whole_rows(const void* base, long long stride, int V, int dtype) {
    const int N = unit_elements(dtype);
    return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && stride % N == 0 && V % N == 0;
}
// Units of a row, at most.
inline int row_units(int V, int dtype, bool whole) {
    const int N = unit_elements(dtype);
    return (int)(((long long)V + (whole ? 0 : 2 * N - 2)) / N);
}

template <typename T, bool WHOLE, int NW, int UPT, bool HOLD, bool GRAD, bool ENT>
int launch(const ScoreParams& p, cudaStream_t stream) {
    return launch_pdl(score_kernel<T, WHOLE, NW, UPT, HOLD, GRAD, ENT>, p.n_rows * p.cs, NW * 32, 0, p.cs, stream, p);
}
template <typename T, bool WHOLE, int NW, int UPT, bool HOLD>
int launch(const ScoreParams& p, bool ent, cudaStream_t stream) {
    if (p.grad) return ent ? launch<T, WHOLE, NW, UPT, HOLD, true, true>(p, stream) : launch<T, WHOLE, NW, UPT, HOLD, true, false>(p, stream);
    return ent ? launch<T, WHOLE, NW, UPT, HOLD, false, true>(p, stream) : launch<T, WHOLE, NW, UPT, HOLD, false, false>(p, stream);
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
    if (cudaOccupancyMaxActiveClusters(&n, kern, &lc) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return n;
}
// Clusters of a kernel that are resident at once, asked for once per device, kernel and cluster size.
template <typename T, bool WHOLE, int NW, bool GRAD, bool ENT>
int stream_clusters(int cs) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices][kScMaxCluster + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return 0;
    int n = known[dev][cs].load(std::memory_order_acquire);
    if (n == 0) {
        const auto kern = score_stream_kernel<T, WHOLE, NW, GRAD, ENT>;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, NW * kSsStage) != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        n = resident_clusters(kern, NW * 32, NW * kSsStage, cs);
        known[dev][cs].store(n, std::memory_order_release);
    }
    return n;
}
// ADASD_ERR_SHAPE: not a launch for score_stream_kernel (rows too long, or too few of them).
template <typename T, bool WHOLE, int NW, bool GRAD, bool ENT>
int launch_stream_t(ScoreParams p, int cs, int per_warp, cudaStream_t stream) {
    const int ncl = stream_clusters<T, WHOLE, NW, GRAD, ENT>(cs);
    if (p.n_rows <= ncl || ncl == 0) return ADASD_ERR_SHAPE;
    p.cs = cs;
    p.per_cta = per_warp;
    return launch_pdl(score_stream_kernel<T, WHOLE, NW, GRAD, ENT>, ncl * cs, NW * 32, NW * kSsStage, cs, stream, p);
}
template <typename T, bool WHOLE, int NW>
int launch_stream_n(const ScoreParams& p, bool ent, int cs, int per_warp, cudaStream_t stream) {
    if (p.grad) return ent ? launch_stream_t<T, WHOLE, NW, true, true>(p, cs, per_warp, stream) : launch_stream_t<T, WHOLE, NW, true, false>(p, cs, per_warp, stream);
    return ent ? launch_stream_t<T, WHOLE, NW, false, true>(p, cs, per_warp, stream) : launch_stream_t<T, WHOLE, NW, false, false>(p, cs, per_warp, stream);
}
template <typename T, bool WHOLE, bool ENT>
int launch_deep_t(ScoreParams p, int cs, int per_warp, cudaStream_t stream) {
    static std::atomic<int> known[64][kScMaxCluster + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ADASD_ERR_SHAPE;
    int ncl = known[dev][cs].load(std::memory_order_acquire);
    const auto kern = score_deep_kernel<T, WHOLE, ENT>;
    if (ncl == 0) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSdSmem) != cudaSuccess) {
            cudaGetLastError();
            return ADASD_ERR_SHAPE;
        }
        ncl = resident_clusters(kern, kSdThreads, kSdSmem, cs);
        known[dev][cs].store(ncl, std::memory_order_release);
    }
    if (p.n_rows <= 2 * ncl || ncl == 0) return ADASD_ERR_SHAPE;
    p.cs = cs;
    p.per_cta = per_warp;
    return launch_pdl(kern, ncl * cs, kSdThreads, kSdSmem, cs, stream, p);
}
template <typename T, bool WHOLE>
int launch_deep(const ScoreParams& p, bool ent, int NU, cudaStream_t stream) {
    const int its = (NU + 31) / 32, cs = (NU + kSdUnits - 1) / kSdUnits, per = (its + cs - 1) / cs * 32;
    if (!p.grad || cs > kScMaxCluster || NU < 2048) return ADASD_ERR_SHAPE;
    return ent ? launch_deep_t<T, WHOLE, true>(p, cs, per, stream) : launch_deep_t<T, WHOLE, false>(p, cs, per, stream);
}
template <typename T, bool WHOLE>
int launch_stream(const ScoreParams& p, bool ent, int NU, cudaStream_t stream) {
    constexpr int W = kSsUPT * 32;
    const int warps = (NU + W - 1) / W;
    if (warps == 1) return launch_stream_n<T, WHOLE, 1>(p, ent, 1, NU, stream);
    if (warps == 2) return launch_stream_n<T, WHOLE, 2>(p, ent, 1, (NU + 1) / 2, stream);
    if (warps <= 4) return launch_stream_n<T, WHOLE, 4>(p, ent, 1, (NU + 3) / 4, stream);
    const int cs = (warps + 7) / 8;
    if (cs > kScMaxCluster) return ADASD_ERR_SHAPE;
    return launch_stream_n<T, WHOLE, 8>(p, ent, cs, (NU + 8 * cs - 1) / (8 * cs), stream);
}

constexpr int kScNW = 8, kScUnits = kScNW * 32;      // CTAs of 8 warps; units of a CTA and unit a thread

template <typename T, bool WHOLE>
int launch(ScoreParams p, bool ent, int NU, int sms, cudaStream_t stream) {
    if (const int rc = launch_deep<T, WHOLE>(p, ent, NU, stream); rc != ADASD_ERR_SHAPE) return rc;
    if (const int rc = launch_stream<T, WHOLE>(p, ent, NU, stream); rc != ADASD_ERR_SHAPE) return rc;
    if (NU <= 2 * 32 * 4) {
        p.cs = 1;
        p.per_cta = NU;
        return launch<T, WHOLE, 2, 4, true>(p, ent, stream);
    }
    int cs = std::min(kScMaxCluster, (NU + kScUnits * 16 - 1) / (kScUnits * 16));
    while (cs < kScMaxCluster && (long long)p.n_rows * cs < 2LL * sms && NU > cs * kScUnits) cs = std::min(2 * cs, kScMaxCluster);
    p.cs = cs;
    p.per_cta = (NU + cs - 1) / cs;
    if (p.per_cta <= kScUnits * 4) return launch<T, WHOLE, kScNW, 4, true>(p, ent, stream);
    if (p.per_cta <= kScUnits * 8) return launch<T, WHOLE, kScNW, 8, true>(p, ent, stream);
    if (p.per_cta <= kScUnits * 16) return launch<T, WHOLE, kScNW, 16, true>(p, ent, stream);
    return launch<T, WHOLE, kScNW, 16, false>(p, ent, stream);
}

}  // namespace

int launch_score(ScoreParams p, int dtype, bool entropy, int sm_count, cudaStream_t stream) {
    const bool whole = whole_rows(p.z, p.row_stride, p.V, dtype) && (!p.grad || whole_rows(p.grad, p.g_stride, p.V, dtype));
    const int NU = row_units(p.V, dtype, whole);
    if (dtype == ADASD_BF16)
        return whole ? launch<__nv_bfloat16, true>(p, entropy, NU, sm_count, stream) : launch<__nv_bfloat16, false>(p, entropy, NU, sm_count, stream);
    return whole ? launch<float, true>(p, entropy, NU, sm_count, stream) : launch<float, false>(p, entropy, NU, sm_count, stream);
}

int launch_pref_pairs(const PrefParams& p, cudaStream_t stream) {
    return launch_pdl(pref_pair_kernel, p.n_pairs, kPairThreads, 0, 0, stream, p);
}

int launch_pref_grad(PrefParams p, int dtype, cudaStream_t stream) {
    const bool whole = whole_rows(p.z, p.row_stride, p.V, dtype) && whole_rows(p.grad, p.g_stride, p.V, dtype);
    const int NU = row_units(p.V, dtype, whole);
    p.segs = (NU + kPgThreads * kPgUnits - 1) / (kPgThreads * kPgUnits);
    p.per_cta = (NU + p.segs - 1) / p.segs;
    if ((long long)p.n_rows * p.segs > 0x7FFFFFFFLL) return ADASD_ERR_SHAPE;
    const int grid = p.n_rows * p.segs;
    if (dtype == ADASD_BF16)
        return whole ? launch_pdl(pref_grad_kernel<__nv_bfloat16, true>, grid, kPgThreads, 0, 0, stream, p)
                  : launch_pdl(pref_grad_kernel<__nv_bfloat16, false>, grid, kPgThreads, 0, 0, stream, p);
    return whole ? launch_pdl(pref_grad_kernel<float, true>, grid, kPgThreads, 0, 0, stream, p)
              : launch_pdl(pref_grad_kernel<float, false>, grid, kPgThreads, 0, 0, stream, p);
}

int launch_total(const float* terms, int n, float* out, cudaStream_t stream) {
    return launch_pdl(total_kernel, 1, kTotThreads, 0, 0, stream, terms, n, out);
}

}  // namespace adasd
