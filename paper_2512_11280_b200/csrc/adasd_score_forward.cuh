// Log-probs, entropies and losses without a gradient on many rows (same outputs as score_kernel): a cluster takes row after row, and
// no warp waits for another's sums.  A warp owns a stretch of units of every row, in two halves that each have a stage: a half is
// taken into registers when it has landed, the same half of the next row is asked for, and the half is summed.  A warp keeps
// its partials of 32 rows; then all warps of the cluster fold them, a few rows each, and report them a row a lane.
#pragma once

#include "adasd_score_stream.cuh"

namespace adasd {

constexpr int kSfUPT = 8;                                    // units a lane holds
constexpr int kSfStage = kSfUPT * 32 * 16;                   // half a stretch
constexpr int kSfWarpUnits = 2 * kSfUPT * 32;

template <typename T, int L, int NW, bool ENT>
__global__ void __launch_bounds__(NW * 32, 24 / NW) score_forward_kernel(const __grid_constant__ ScoreParams p) {
    using U = Unit<T>;
    constexpr int UPT = kSfUPT;
    const float floor_v = U::N == 8 ? ADASD_FLOOR_BF : kFloor;
    extern __shared__ __align__(128) unsigned char dyn_smem[];
    __shared__ unsigned long long full_s[NW][2];
    // 32 rows of partials, twice: those of one set of rows are folded by others while the next set's are formed
    __shared__ float4 keep[2][NW][32];
    __shared__ int rows_s[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CS = p.cs, ncl = (int)(gridDim.x / (unsigned)CS), cl = (int)(blockIdx.x / (unsigned)CS);
    const int rank = (int)(blockIdx.x - (unsigned)cl * (unsigned)CS);
    unsigned char* const stages = dyn_smem + warp * 2 * kSfStage;
    cg::cluster_group cluster = cg::this_cluster();
    if (lane == 0) {
        mbar_init(reinterpret_cast<uint64_t*>(&full_s[warp][0]), 1);
        mbar_init(reinterpret_cast<uint64_t*>(&full_s[warp][1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (CS > 1) cluster.sync();
    else __syncthreads();
    pdl_wait();
    pdl_trigger();

    const int ua = (rank * NW + warp) * p.per_cta, half = (p.per_cta + 63) / 64 * 32;        // (per_cta: units of a WARP here)
    auto units = [&](int row) {
        const T* const z = reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride;
        return RowUnits<T, L>(z, z, p.V);
    };
    // units [first, end) of half h of a row's stretch
    auto first_of = [&](const RowUnits<T, L>& ru, int h) { return min(ua + h * half, ru.NU); };
    auto end_of = [&](const RowUnits<T, L>& ru, int h) { return min(ua + (h ? p.per_cta : min(half, p.per_cta)), ru.NU); };

    RowWindow win;
    auto open = [&](int wi) {
        win.wi = wi;
        const long long r = (long long)cl + (long long)(wi + lane) * ncl;
        int kind = -2;
        if (r < p.n_rows) {
            win.row = (int)r;
            win.x = __ldcg(p.tok + r);
            kind = row_kind(p, (int)r, win.x);
            if (rank == 0 && warp == 0 && kind != 1) row_report_out(p, (int)r, kind);
        }
        win.todo = __ballot_sync(0xFFFFFFFFu, kind == 1);
    };
    int nrow = -1, nx = 0;                                   // the next row (-1: none left)
    auto next = [&]() {
        while (!win.todo) {
            nrow = -1;
            if ((long long)cl + (long long)(win.wi + 32) * ncl >= p.n_rows) return;
            open(win.wi + 32);
        }
        const int j = __ffs(win.todo) - 1;
        win.todo &= win.todo - 1;
        nrow = __shfl_sync(0xFFFFFFFFu, win.row, j);
        nx = __shfl_sync(0xFFFFFFFFu, win.x, j);
    };
    bool alive = true;                                       // (no more copies once a wait has run out; those under way are waited for)
    unsigned asked = 0u;                                     // stages a copy is under way to
    auto ask = [&](int h) {                                  // half h of the next row
        asked &= ~(1u << h);
        if (nrow < 0 || !alive) return;
        asked |= 1u << h;
        if (lane == 0) {
            const RowUnits<T, L> ru = units(nrow);
            const int g0 = first_of(ru, h), g1 = end_of(ru, h);
            const uint32_t bytes = (uint32_t)max(g1 - g0, 0) * 16u;
            uint64_t* const bar = reinterpret_cast<uint64_t*>(&full_s[warp][h]);
            mbar_expect_tx(bar, bytes);
            if (bytes) bulk_g2s(stages + h * kSfStage, ru.src + g0, bytes, bar);
        }
    };
    open(0);
    next();
    ask(0);
    ask(1);

    const float c1 = p.c1;
    const float2 L2 = pair2(c1);
    int done = 0;
    while (nrow >= 0) {
        const int row = nrow, x = nx;
        const RowUnits<T, L> ru = units(row);
        float m = -INFINITY, S = 0.f, Ts = 0.f, zx = -INFINITY;
        uint32_t bad = 0u;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            if (asked >> h & 1u) {
                const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(reinterpret_cast<uint64_t*>(&full_s[warp][h]), (uint32_t)done & 1u));
                if (!ok && lane == 0) atomicOr(p.status, ADASD_STATUS_TIMEOUT);
                alive = alive && ok;
            }
            if (!alive) bad = 1u;
            const int u0 = first_of(ru, h), un = end_of(ru, h), nk = max(0, (un - u0 + 31) >> 5);
            const RowStage<T, L> rs(stages + h * kSfStage, ru, u0, un);
            rs.clean(0);
            uint4 w[UPT];
            typename U::Max mx = U::max0();
#pragma unroll
            for (int k = 0; k < UPT; ++k) {
                const int u = u0 + k * 32 + lane;
                w[k] = u < un ? rs.held(u) : U::none4();
            }
#pragma unroll
            for (int k = 0; k < UPT; ++k) U::max_add(mx, w[k]);
            const float z = rs.owns(x) ? rs.token(x) : -INFINITY;
            if (z != z) bad = 1u;
            zx = fmaxf(zx, z);
            const float t = warp_max_f32(fmaxf(U::max_val(mx, bad), z));    // (every lane's loads from the stage have ended)
            if (t == INFINITY) bad = 1u;
            if (h == 0) next();
            rs.release();
            ask(h);
            const Shift c = sum_shift(t, c1, L2);
            float2 S2 = make_float2(0.f, 0.f), T2 = make_float2(0.f, 0.f);
            if (sum_big(t, c1)) for_units<UPT>(nk, [&](int k) { add_unit<T, ENT, true>(w[k], c, S2, T2); });
            else for_units<UPT>(nk, [&](int k) { add_unit<T, ENT, false>(w[k], c, S2, T2); });
            const float2 r = finish_sums<ENT>(S2, T2, t, c1);
            if (h == 0) {
                m = t;
                S = r.x;
                Ts = r.y;
            } else {
                fold_sums(m, S, Ts, t, r, c1);
            }
        }
        const int set = done >> 5 & 1, at = done & 31;
        const bool any_bad = __any_sync(0xFFFFFFFFu, bad);
        if (lane == 0) {
            keep[set][warp][at] = make_float4(m, any_bad ? NAN : S, Ts, zx);
            if (warp == 0) rows_s[set][at] = row;
        }
        ++done;
        if (at == 31 || nrow < 0) {
            // (whoever comes here has folded the set before: its place may be written again)
            if (CS > 1) cluster.sync();
            else __syncthreads();
            RowStats st;
            int cnt = 0, which = 0;
            for (int j = rank * NW + warp; j <= at; j += CS * NW, ++cnt) {
                RowStats f = fold_partials<kScMaxCluster * NW>(
                    [&](int k) { return *cluster.map_shared_rank(&keep[set][k % NW][j], k / NW); }, CS * NW, c1, floor_v);
                if (lane == cnt) {
                    st = f;
                    which = rows_s[set][j];
                }
            }
            if (lane < cnt) row_report(p, which, row_in(p, which), st);
        }
    }
    if (CS > 1) cluster.sync();                              // (nobody leaves while others read its partials)
}

}  // namespace adasd
