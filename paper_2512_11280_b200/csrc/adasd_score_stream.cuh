// score_kernel for launches of many rows (same rows, same outputs): a cluster takes row after row, and while a row is summed
// and its gradient formed from the registers that hold it, the next one is on its way into shared memory.
//
// A warp owns a stretch of units of every row: it asks for it with one bulk copy, takes it into registers when it has landed,
// and asks for the next row's at once, so that an SM has up to 128 KB of loads under way whatever its warps are at.  The warps'
// statistics go to every CTA of the cluster with stores that count their bytes on a barrier there; a warp waits for nothing else.
#pragma once

#include "adasd_score.cuh"

namespace adasd {

constexpr int kSsUPT = 16;                                   // units a lane holds
constexpr int kSsStage = (kSsUPT * 32 + 1) * 16;             // a warp's stretch (+ one unit: rows off 16-byte boundaries)

// What a warp keeps of 32 rows: inputs of their losses, until they are used (GRAD); its partials and the rows, until they are
// folded (forward pass); the rows' statistics, until they are reported (GRAD, one warp of a cluster).
struct __align__(16) RowHist {
    RowStats s;
    int32_t row, pad[3];
};

// The rows a cluster has to do, 32 at a time: lane j holds row first + (wi + j) clusters.  Rows left out are set aside.
struct RowWindow {
    int wi, row, x;
    unsigned todo, zero;                                     // lanes with rows to do, with gradient rows to zero
};

template <typename T, bool WHOLE, int NW, bool GRAD, bool ENT>
__global__ void __launch_bounds__(NW * 32, 16 / NW) score_stream_kernel(const __grid_constant__ ScoreParams p) {
    using U = Unit<T>;
    constexpr int N = U::N, UPT = kSsUPT;
    const float floor_v = N == 8 ? ADASD_FLOOR_BF : kFloor;
    extern __shared__ __align__(128) unsigned char dyn_smem[];
    __shared__ float4 part[2][GRAD ? kScMaxCluster * NW : 1];
    __shared__ unsigned long long full_s[NW], got_s[2];
    __shared__ RowHist hist[GRAD ? 32 : 1];
    __shared__ float4 keep[NW][32];                          // GRAD: RowIn of the window's rows; else the partials of 32 rows
    __shared__ int2 rows_s[GRAD ? 1 : 32];                   // ... and which rows, with their tokens
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CS = p.cs, ncl = (int)(gridDim.x / (unsigned)CS), cl = (int)(blockIdx.x / (unsigned)CS);
    const int rank = (int)(blockIdx.x - (unsigned)cl * (unsigned)CS);
    const bool keeper = rank == 0 && warp == 0;              // the warp that reports
    uint64_t* const full = reinterpret_cast<uint64_t*>(&full_s[warp]);
    unsigned char* const stage = dyn_smem + warp * kSsStage;
    cg::cluster_group cluster = cg::this_cluster();
    if (lane == 0) {
        mbar_init(full, 1);
        if (warp == 0) {
            mbar_init(reinterpret_cast<uint64_t*>(&got_s[0]), 1);
            mbar_init(reinterpret_cast<uint64_t*>(&got_s[1]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (CS > 1) cluster.sync();
    else __syncthreads();
    pdl_wait();
    pdl_trigger();

    const int ua = (rank * NW + warp) * p.per_cta, ub = ua + p.per_cta;          // (per_cta: units of a WARP here)
    auto units = [&](int row) {
        const T* const z = reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride;
        return RowUnits<T, WHOLE>(z, GRAD ? reinterpret_cast<const T*>(p.grad) + (long long)row * p.g_stride : z, p.V);
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
            if (keeper && kind != 1) row_report_out(p, (int)r, kind);
        }
        if (GRAD) {
            RowIn in{0.f, 0.f, 0.f, 0.f};
            if (kind == 1) in = row_in(p, (int)r);
            __syncwarp();
            keep[warp][lane] = make_float4(in.adv, in.old, in.ref, in.w);
            __syncwarp();
        }
        win.todo = __ballot_sync(0xFFFFFFFFu, kind == 1);
        win.zero = GRAD ? __ballot_sync(0xFFFFFFFFu, kind == 0) : 0u;
    };
    auto zero_row = [&]() {                                  // one row set aside
        const int j = __ffs(win.zero) - 1, row = __shfl_sync(0xFFFFFFFFu, win.row, j);
        win.zero &= win.zero - 1;
        const RowUnits<T, WHOLE> ru = units(row);
        T* const g = reinterpret_cast<T*>(p.grad) + (long long)row * p.g_stride;
        for (int u = ua + lane; u < min(ub, ru.NU); u += 32) ru.store(g, u, make_uint4(0u, 0u, 0u, 0u));
    };
    int row = -1, x = 0;                                     // the row asked for; -1: none left
    float4 inputs;                                           // of its loss
    auto next = [&]() {
        while (!win.todo) {
            while (GRAD && win.zero) zero_row();
            row = -1;
            if ((long long)cl + (long long)(win.wi + 32) * ncl >= p.n_rows) return;
            open(win.wi + 32);
        }
        const int j = __ffs(win.todo) - 1;
        win.todo &= win.todo - 1;
        row = __shfl_sync(0xFFFFFFFFu, win.row, j);
        x = __shfl_sync(0xFFFFFFFFu, win.x, j);
        if (GRAD) inputs = keep[warp][j];
    };
    auto ask = [&]() {                                       // its stretch: granules from unit ua's first on that hold elements
        if (lane == 0) {
            const RowUnits<T, WHOLE> ru = units(row);
            const int g0 = max(ua, ru.glo), g1 = min(min(ub, ru.NU) + (!WHOLE && ru.sh ? 1 : 0), ru.ghi);
            const uint32_t bytes = (uint32_t)max(g1 - g0, 0) * 16u;
            mbar_expect_tx(full, bytes);
            if (bytes) bulk_g2s(stage + (g0 - ua) * 16, ru.src + g0, bytes, full);
        }
    };
    bool alive = true, asked = false;                        // (no more copies once a wait has run out; one under way is waited for)
    open(0);
    next();
    if (row >= 0) {
        ask();
        asked = true;
    }

    const float c1 = p.c1;
    const float2 L2 = pair2(c1);
    uint32_t ph = 0u;
    int done = 0;
    while (row >= 0) {
        const int my_row = row, my_x = x, par = done & 1;
        const RowUnits<T, WHOLE> ru = units(my_row);
        const int un = min(ub, ru.NU);
        const RowIn in{inputs.x, inputs.y, inputs.z, inputs.w};
        uint64_t* const got = reinterpret_cast<uint64_t*>(&got_s[par]);
        if (GRAD && CS > 1 && warp == 0 && lane == 0) mbar_expect_tx(got, (uint32_t)(CS * NW) * 16u);
        if (asked) {
            const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(full, ph));
            if (!ok && lane == 0) atomicOr(p.status, ADASD_STATUS_TIMEOUT);
            alive = alive && ok;
        }
        ph ^= 1u;
        uint32_t bad = alive ? 0u : 1u;
        uint4 w[UPT];
        typename U::Max mx = U::max0();
#pragma unroll
        for (int k = 0; k < UPT; ++k) {
            const int u = ua + k * 32 + lane;
            w[k] = u < un ? ru.unit(u, [&](int g) { return *reinterpret_cast<const uint4*>(stage + (g - ua) * 16); }) : U::none4();
        }
#pragma unroll
        for (int k = 0; k < UPT; ++k) U::max_add(mx, w[k]);
        // the token's logit, if it is in this stretch
        const int ox = ru.unit_of(my_x) - ua;
        float zx = -INFINITY;
        if (ox >= 0 && ox < un - ua) {
            const int e = my_x - ((ua + ox) * N - ru.m0) + ru.sh;           // (of the two granules that hold its unit)
            zx = to_f32(*reinterpret_cast<const T*>(stage + ox * 16 + e * (int)sizeof(T)));
        }
        if (zx != zx) bad = 1u;
        const float m = warp_max_f32(fmaxf(U::max_val(mx, bad), zx));       // (every lane's loads from the stage have ended)
        if (m == INFINITY) bad = 1u;
        next();
        asked = row >= 0 && alive;
        if (asked) ask();
        const float2 sums = sum_units<T, ENT, UPT>(w, m, c1, L2, [&](int k) { return ua + k * 32 < un; });
        const float4 mine = make_float4(m, __any_sync(0xFFFFFFFFu, bad) ? NAN : sums.x, sums.y, zx);
        if (!GRAD) {
            // forward pass: nothing waits for the totals; 32 rows are folded and reported at a time, by all warps of the cluster
            if (lane == 0) {
                keep[warp][done & 31] = mine;
                if (warp == 0) rows_s[done & 31] = make_int2(my_row, my_x);
            }
            ++done;
            if ((done & 31) == 0 || row < 0) {
                const int n = ((done - 1) & 31) + 1;
                if (CS > 1) cluster.sync();
                else __syncthreads();
                RowStats st;
                int cnt = 0, which = 0;
                for (int j = rank * NW + warp; j < n; j += CS * NW, ++cnt) {
                    const RowStats f = fold_partials<kScMaxCluster * NW>(
                        [&](int k) { return *cluster.map_shared_rank(&keep[k % NW][j], k / NW); }, CS * NW, c1, floor_v);
                    if (lane == cnt) {
                        st = f;
                        which = j;
                    }
                }
                if (lane < cnt) row_report(p, rows_s[which].x, row_in(p, rows_s[which].x), st);
                if (CS > 1) cluster.sync();
                else __syncthreads();
            }
            continue;
        }
        if (CS > 1) {
            if (lane < CS) st_async_v4(mapa_u32(&part[par][rank * NW + warp], lane), mine, mapa_u32(got, lane));
            if (alive) {
                alive = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(got, (uint32_t)(done >> 1) & 1u));
                if (!alive && lane == 0) atomicOr(p.status, ADASD_STATUS_TIMEOUT);
            }
        } else if (NW > 1) {
            if (lane == 0) part[par][warp] = mine;
            __syncthreads();
        }
        RowStats st;
        if (NW == 1 && CS == 1) {
            st.M = m;
            st.S = m > floor_v ? mine.y : NAN;
            st.Ts = mine.z;
            st.zx = zx;
        } else {
            st = fold_partials<kScMaxCluster * NW>([&](int k) { return part[par][k]; }, CS * NW, c1, floor_v);
        }
        if (!alive) st.S = NAN;
        if (GRAD) {
            const RowGrad r = row_grad(p, in, st, c1, L2, ENT);
            T* const g = reinterpret_cast<T*>(p.grad) + (long long)my_row * p.g_stride;
            auto write = [&](auto big) {
#pragma unroll
                for (int k = 0; k < UPT; k += 4) {
                    if (ua + k * 32 < un) {
#pragma unroll
                        for (int i = k; i < k + 4; ++i) {
                            const int u = ua + i * 32 + lane;
                            const uint4 v = grad_unit<T, ENT, decltype(big)::value>(w[i], r.c);
                            if (u < un) ru.store(g, u, v);
                        }
                    }
                }
            };
            if (r.zero) {
                for (int u = ua + lane; u < un; u += 32) ru.store(g, u, make_uint4(0u, 0u, 0u, 0u));
            } else {
                if (r.big) write(std::true_type{});
                else write(std::false_type{});
                // (the lane that wrote the token's element writes it again)
                if (ox >= 0 && ox < un - ua && lane == (ox & 31)) grad_token<T, ENT>(g, my_x, zx, st.M, c1, r);
            }
        }
        if (keeper && lane == 0) {
            RowHist& h = hist[done & 31];
            h.s = st;
            h.row = my_row;
        }
        ++done;
        if (keeper && ((done & 31) == 0 || row < 0)) {       // 32 rows' reports, a lane each
            __syncwarp();
            if (lane < ((done - 1) & 31) + 1) row_report(p, hist[lane].row, row_in(p, hist[lane].row), hist[lane].s);
            __syncwarp();
        }
    }
    if (GRAD && CS > 1) cluster.sync();                      // (nobody leaves while a warp's partials are on their way to it)
}

}  // namespace adasd
