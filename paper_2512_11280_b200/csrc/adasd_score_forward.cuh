// Log-probs, entropies and losses without a gradient on many rows (same outputs as score_kernel): a cluster (of one CTA, where there
// are rows enough) takes row after row, and no warp waits for another's sums.  A warp owns a stretch of units of every row and goes
// through it piece by piece: a piece is taken into registers when it has landed, the piece after the next is asked for, and
// the lanes add to their sums of the row.  A warp keeps its partials of 32 rows; then all warps of the cluster fold them, a few rows
// each, and report them a row a lane.
#pragma once

#include "adasd_score_stream.cuh"

namespace adasd {

constexpr int kSfUPT = 8;                                    // units a lane holds
constexpr int kSfPiece = kSfUPT * 32;                        // units of a piece, at most
constexpr int kSfStage = kSfPiece * 16;

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

    // (per_cta: units of a WARP here, p.pieces pieces of them)
    const int ua = (rank * NW + warp) * p.per_cta, NP = p.pieces, size = p.per_cta / NP;
    auto units = [&](int row) {
        const T* const z = reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride;
        return RowUnits<T, L>(z, z, p.V);
    };

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
    struct Row {
        int row, x;                                          // row -1: none left
    };
    auto next = [&]() -> Row {
        while (!win.todo) {
            if ((long long)cl + (long long)(win.wi + 32) * ncl >= p.n_rows) return Row{-1, 0};
            open(win.wi + 32);
        }
        const int j = __ffs(win.todo) - 1;
        win.todo &= win.todo - 1;
        return Row{__shfl_sync(0xFFFFFFFFu, win.row, j), __shfl_sync(0xFFFFFFFFu, win.x, j)};
    };
    bool alive = true;                                       // (no more copies once a wait has run out; those under way are waited for)
    unsigned asked = 0u;                                     // stages a copy is under way to
    auto ask = [&](int row, int piece, int s) {
        asked &= ~(1u << s);
        if (row < 0 || !alive) return;
        asked |= 1u << s;
        if (lane == 0) {
            const RowUnits<T, L> ru = units(row);
            const int g0 = ua + piece * size, g1 = min(g0 + size, ru.NU);
            const uint32_t bytes = (uint32_t)max(g1 - g0, 0) * 16u;
            uint64_t* const bar = reinterpret_cast<uint64_t*>(&full_s[warp][s]);
            mbar_expect_tx(bar, bytes);
            if (bytes) bulk_g2s(stages + s * kSfStage, ru.src + g0, bytes, bar);
        }
    };
    open(0);
    Row cur = next(), n1 = next(), n2 = next();
    ask(cur.row, 0, 0);
    if (NP > 1) ask(cur.row, 1, 1);
    else ask(n1.row, 0, 1);

    const float c1 = p.c1;
    const float2 L2 = pair2(c1);
    int done = 0;
    uint32_t t = 0u;                                         // pieces done
    while (cur.row >= 0) {
        const int row = cur.row, x = cur.x;
        const RowUnits<T, L> ru = units(row);
        float m = -INFINITY, off = 0.f, zx = -INFINITY;      // off: what the shift lacks of m c1
        float2 S2 = make_float2(0.f, 0.f), T2 = make_float2(0.f, 0.f);
        uint32_t bad = 0u;
#pragma unroll 1
        for (int piece = 0; piece < NP; ++piece, ++t) {
            const int s = (int)(t & 1u);
            if (asked >> s & 1u) {
                const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(reinterpret_cast<uint64_t*>(&full_s[warp][s]), (t >> 1) & 1u));
                if (!ok && lane == 0) atomicOr(p.status, ADASD_STATUS_TIMEOUT);
                alive = alive && ok;
            }
            if (!alive) bad = 1u;
            const int u0 = min(ua + piece * size, ru.NU), un = min(u0 + size, ru.NU), nk = (un - u0 + 31) >> 5;
            const RowStage<T, L> rs(stages + s * kSfStage, ru, u0, un);
            rs.clean(0);
            uint4 w[UPT];
            typename U::Max mx = U::max0();
            if (un - u0 == kSfPiece) {
#pragma unroll
                for (int k = 0; k < UPT; ++k) w[k] = rs.held(u0 + k * 32 + lane);
            } else {
#pragma unroll
                for (int k = 0; k < UPT; ++k) {
                    const int u = u0 + k * 32 + lane;
                    w[k] = u < un ? rs.held(u) : U::none4();
                }
            }
#pragma unroll
            for (int k = 0; k < UPT; ++k) U::max_add(mx, w[k]);
            const float z = rs.owns(x) ? rs.token(x) : -INFINITY;
            if (z != z) bad = 1u;
            zx = fmaxf(zx, z);
            const float v = warp_max_f32(fmaxf(U::max_val(mx, bad), z));    // (every lane's loads from the stage have ended)
            rs.release();
            if (piece + 2 < NP) ask(row, piece + 2, s);
            else if (NP > 1) ask(n1.row, piece + 2 - NP, s);
            else ask(n2.row, 0, s);
            if (v > m) {                                     // a larger maximum: the sums move to its shift
                const float o = sum_big(v, c1) ? 0.f : fmaf(v, c1, -(v * c1));
                const float d = m > -INFINITY ? fmaxf((m - v) * c1 - off + o, kLowT) : kLowT, f = ex2(d);
                if (ENT) {
                    T2.x = f * fmaf(d, S2.x, T2.x);
                    T2.y = f * fmaf(d, S2.y, T2.y);
                }
                S2.x *= f;
                S2.y *= f;
                m = v;
                off = o;
            }
            const Shift c = sum_shift(m, c1, L2);
            if (sum_big(m, c1)) for_units<UPT>(nk, [&](int k) { add_unit<T, ENT, true>(w[k], c, S2, T2); });
            else for_units<UPT>(nk, [&](int k) { add_unit<T, ENT, false>(w[k], c, S2, T2); });
        }
        if (m == INFINITY) bad = 1u;
        const float2 sums = finish_sums<ENT>(S2, T2, m, c1);
        cur = n1;
        n1 = n2;
        n2 = next();
        const int set = done >> 5 & 1, at = done & 31;
        const bool any_bad = __any_sync(0xFFFFFFFFu, bad);
        if (lane == 0) {
            keep[set][warp][at] = make_float4(m, any_bad ? NAN : sums.x, sums.y, zx);
            if (warp == 0) rows_s[set][at] = row;
        }
        ++done;
        if (at == 31 || cur.row < 0) {
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
