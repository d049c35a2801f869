// Losses with a gradient on many rows that leave room for two of them on an SM (score_kernel's outputs): a row is read once and
// its gradient written once, and nothing waits for the totals of the row it has just summed.
//
// A cluster takes item after item, an item being a row to do and the rows left out ahead of it.  A CTA holds a stretch of the row and
// has eight workers and a control warp.  The control warp asks for the stretches with bulk copies, two items ahead, folds the
// partials of the whole cluster's workers and works out what a row's gradient takes: 400 instructions a row, which took
// a third of the issue slots where every warp did it.  A worker, with the gradient of item n still to write, moves item n into its registers
// (its stage is free then), sums item n + 1 from the other stage, sends these partials, and only then takes the constants of
// item n and writes.
//
// What bounds it: no unit is saturated (counters at 1120 rows of 128256 bf16: special-function pipe 57 %, issue slots 49 %, DRAM 56 %);
// what was taken off the special-function pipe and the issue slots made it faster.  2048 rows of 128256 bf16 logits 192 us (5.5 TB/s both
// ways; 212 with all 2^t on one pipe).  A cluster's rows are every ncl-th, whether they are left out or not: with rows left out at random
// the cluster with the most rows to do sets the time (2048 rows of 128256, a tenth left out: as long as with none).  13 units a lane
// and two CTAs an SM: 12 workers of 9 units measured 202 us; the lanes' own copies (as score_forward_kernel's) in place of the bulk
// copies 198 us against 183 on 2065 rows and 219 against 149 on 4000 rows of 50257: their instructions come on top.
#pragma once

#include "adasd_score_stream.cuh"

namespace adasd {

constexpr int kSdUPT = 13;                                   // units a lane holds
constexpr int kSdNW = 8;                                     // workers
constexpr int kSdThreads = (kSdNW + 1) * 32;
constexpr int kSdUnits = kSdNW * kSdUPT * 32;                // units of a CTA, at most: two CTAs' stages fill the shared memory
constexpr int kSdStage = (kSdUnits + 1) * 16;
constexpr int kSdSmem = 2 * kSdStage;

struct __align__(16) DeepItem {
    int32_t row, x, kind;                                    // kind 1: a row to do, -1: none left
    int32_t zeros;                                           // rows left out ahead of it: row - ncl, row - 2 ncl, ..
    float4 in;                                               // RowIn
};
struct __align__(16) DeepCoef {
    float ns, a2, b2, a;                                     // RowGrad
    float b, top, M, zx;
    int32_t zero, big, pad[2];
};

template <typename T, int L, bool ENT>
__global__ void __launch_bounds__(kSdThreads, 2) score_deep_kernel(const __grid_constant__ ScoreParams p) {
    using U = Unit<T>;
    constexpr int N = U::N, UPT = kSdUPT, NW = kSdNW;
    constexpr bool WHOLE = L == ROWS_WHOLE;
    const float floor_v = N == 8 ? ADASD_FLOOR_BF : kFloor;
    extern __shared__ __align__(128) unsigned char dyn_smem[];
    // Four rows' worth: a worker sends the partials of row n once it has the constants of row n - 2, for which every
    // worker had to send its partials of that row, which it did after its own control warp had folded row n - 4.
    __shared__ float4 part[4][kScMaxCluster * NW];
    __shared__ DeepItem items[4];
    __shared__ DeepCoef coefs[4];
    __shared__ RowHist hist[32];
    __shared__ unsigned long long full_s[2], empty_s[2], got_s[4], ready_s[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CS = p.cs, ncl = (int)(gridDim.x / (unsigned)CS), cl = (int)(blockIdx.x / (unsigned)CS);
    const int rank = (int)(blockIdx.x - (unsigned)cl * (unsigned)CS);
    auto bar = [](unsigned long long& b) { return reinterpret_cast<uint64_t*>(&b); };
    cg::cluster_group cluster = cg::this_cluster();
    if (threadIdx.x == 0) {
        items[3].row = 0;
        for (int k = 0; k < 2; ++k) {
            mbar_init(bar(full_s[k]), 1);
            mbar_init(bar(empty_s[k]), NW);
        }
        for (int k = 0; k < 4; ++k) {
            mbar_init(bar(got_s[k]), 1);
            mbar_init(bar(ready_s[k]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // the stages: what no copy ever fills reads as -inf
    for (int k = threadIdx.x; k < kSdSmem / 16; k += kSdThreads) reinterpret_cast<uint4*>(dyn_smem)[k] = U::none4();
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    cluster.sync();
    pdl_wait();
    pdl_trigger();

    const int ua = rank * p.per_cta;                         // the CTA's stretch: units [ua, ua + per_cta), a multiple of 32
    auto units = [&](int row) {
        return RowUnits<T, L>(reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride,
                                  reinterpret_cast<const T*>(p.grad) + (long long)row * p.g_stride, p.V);
    };
    const float c1 = p.c1;
    const float2 L2 = pair2(c1);
    // A wait that runs out ends its warp's work, and so, a wait later, everybody's: the rows that were left are not written.
    bool alive = true;
    auto wait = [&](unsigned long long& b, uint32_t parity) {
        if (!alive) return;
        alive = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar(b), parity));
        if (!alive && lane == 0) atomicOr(p.status, ADASD_STATUS_TIMEOUT);
    };

    if (warp == NW) {
        // ---- control ------------------------------------------------------------------------
        // 32 rows at a time: lane j holds row cl + (wi + j) ncl, its token, kind and inputs
        int wi = -32, left = 0, w_x = 0, w_kind = -1;
        RowIn w_in{0.f, 0.f, 0.f, 0.f};
        int j = 0;
        auto post = [&](int n) {                             // item n, and the copy of its stretch
            DeepItem it;
            it.zeros = 0;
            it.kind = -1;
            for (;;) {
                const unsigned todo = __ballot_sync(0xFFFFFFFFu, w_kind == 1 && lane >= j);
                const int to = todo ? __ffs(todo) - 1 : left;
                it.zeros += to - j;
                j = to;
                if (todo) it.kind = 1;
                if (todo || (long long)cl + (long long)(wi + 32) * ncl >= p.n_rows) break;
                wi += 32;
                const long long r = (long long)cl + (long long)(wi + lane) * ncl;
                w_kind = -1;
                if (r < p.n_rows) {
                    w_x = __ldcg(p.tok + r);
                    w_kind = row_kind(p, (int)r, w_x);
                    if (w_kind == 1) w_in = row_in(p, (int)r);
                    if (rank == 0 && w_kind != 1) row_report_out(p, (int)r, w_kind);
                }
                left = __popc(__ballot_sync(0xFFFFFFFFu, r < p.n_rows));
                j = 0;
            }
            it.row = cl + (wi + j) * ncl;                    // (none left: the one after the last)
            it.x = __shfl_sync(0xFFFFFFFFu, w_x, j & 31);
            it.in = make_float4(__shfl_sync(0xFFFFFFFFu, w_in.adv, j & 31), __shfl_sync(0xFFFFFFFFu, w_in.old, j & 31),
                                __shfl_sync(0xFFFFFFFFu, w_in.ref, j & 31), __shfl_sync(0xFFFFFFFFu, w_in.w, j & 31));
            if (it.kind == 1) ++j;
            if (lane == 0) {
                items[n & 3] = it;
                uint64_t* const f = bar(full_s[n & 1]);
                if (it.kind == 1) {
                    const RowUnits<T, L> ru = units(it.row);
                    const int g0 = max(ua, ru.glo), g1 = min(min(ua + p.per_cta, ru.NU), ru.ghi);
                    const uint32_t bytes = (uint32_t)max(g1 - g0, 0) * 16u;
                    mbar_expect_tx(f, bytes);
                    if (bytes) bulk_g2s(dyn_smem + (n & 1) * kSdStage + (g0 - ua) * 16, ru.src + g0, bytes, f);
                } else {
                    mbar_expect_tx(f, 0u);
                }
            }
            __syncwarp();
        };
        if (lane == 0)
            for (int k = 0; k < 4; ++k) mbar_expect_tx(bar(got_s[k]), (uint32_t)(CS * NW) * 16u);
        post(0);
        post(1);
        int posted = 1;
        for (int n = 0;; ++n) {
            const DeepItem it = items[n & 3];
            if (it.kind < 0) break;
            wait(got_s[n & 3], (uint32_t)(n >> 2) & 1u);
            if (!alive) break;
            const RowStats st = fold_partials<kScMaxCluster * NW>([&](int k) { return part[n & 3][k]; }, CS * NW, c1, floor_v);
            const RowIn in{it.in.x, it.in.y, it.in.z, it.in.w};
            const RowGrad r = row_grad(p, in, st, c1, L2, ENT);
            if (lane == 0) {
                mbar_expect_tx(bar(got_s[n & 3]), (uint32_t)(CS * NW) * 16u);        // for row n + 4
                DeepCoef c;
                c.ns = r.c.s.ns2.x;
                c.a2 = r.c.a2.x;
                c.b2 = r.c.b2.x;
                c.a = r.a;
                c.b = r.b;
                c.top = r.top;
                c.M = st.M;
                c.zx = st.zx;
                c.zero = r.zero;
                c.big = r.big;
                coefs[n & 3] = c;
                mbar_arrive_cta(bar(ready_s[n & 3]));
                hist[n & 31].s = st;
                hist[n & 31].row = it.row;
            }
            __syncwarp();
            // (its constants first: the workers are at the gradient of the row before, and will ask for them after the next sums)
            wait(empty_s[n & 1], (uint32_t)(n >> 1) & 1u);
            if (!alive) break;
            post(n + 2);
            posted = n + 2;
            if (rank == 0 && ((n & 31) == 31 || items[(n + 1) & 3].kind < 0)) {          // 32 rows' reports, a lane each
                if (lane <= (n & 31)) row_report(p, hist[lane].row, row_in(p, hist[lane].row), hist[lane].s);
                __syncwarp();
            }
        }
        for (int n = posted - 1; n <= posted; ++n) mbar_wait_bounded(bar(full_s[n & 1]), (uint32_t)(n >> 1) & 1u);   // (no copy outlives the CTA)
    } else {
        // ---- workers ------------------------------------------------------------------------
        // A worker's units: ua + (k NW + warp) 32 + lane
        auto unit_at = [&](int k) { return ua + (k * NW + warp) * 32 + lane; };
        // ... k = 0 .. count_of(un) - 1, un: end of the CTA's stretch
        auto count_of = [&](int un) { return max(0, (un - ua - warp * 32 + NW * 32 - 1) / (NW * 32)); };
        // the worker that reads an end of the row
        auto cleans = [&](const RowUnits<T, L>& ru, int un) {
            return !WHOLE && ua < un && ((ua == 0 && warp == 0) || (un == ru.NU && ((un - 1 - ua) >> 5) % NW == warp));
        };
        auto sum_row = [&](const DeepItem& it, int n) {
            const RowUnits<T, L> ru = units(it.row);
            const int un = min(ua + p.per_cta, ru.NU);
            const RowStage<T, L> st(dyn_smem + (n & 1) * kSdStage, ru, ua, un);
            uint32_t bad = 0u;
            // The ends of the row, by the worker that reads them.  (A row that starts elsewhere may have had a unit more.)
            if (cleans(ru, un)) st.clean(1);
            typename U::Max mx = U::max0();
            const int nk = count_of(un);
            for_units<UPT>(nk, [&](int k) { U::max_add(mx, st.held(unit_at(k))); });
            float zx = -INFINITY;
            const int ux = ru.unit_of(it.x);
            if (ux >= ua && ux < un && ((ux - ua) >> 5) % NW == warp) zx = st.token(it.x);
            if (zx != zx) bad = 1u;
            const float m = warp_max_f32(U::max_val(mx, bad));
            if (m == INFINITY) bad = 1u;
            const Shift c = sum_shift(m, c1, L2);
            float2 S2 = make_float2(0.f, 0.f), T2 = make_float2(0.f, 0.f);
            auto add = [&](auto big) {
                for_units<UPT>(nk, [&](int k) { add_unit<T, ENT, decltype(big)::value>(st.held(unit_at(k)), c, S2, T2); });
            };
            if (sum_big(m, c1)) add(std::true_type{});
            else add(std::false_type{});
            const float2 sums = finish_sums<ENT>(S2, T2, m, c1);
            const float4 mine = make_float4(m, __any_sync(0xFFFFFFFFu, bad) ? NAN : sums.x, sums.y, zx);
            if (lane < CS) st_async_v4(mapa_u32(&part[n & 3][rank * NW + warp], lane), mine, mapa_u32(bar(got_s[n & 3]), lane));
        };
        // n = -1: nothing to write yet
        for (int n = -1; alive; ++n) {
            const int row = items[n & 3].row, x = items[n & 3].x;
            const RowUnits<T, L> ru = units(max(row, 0));
            const int un = min(ua + p.per_cta, ru.NU), nk = count_of(un);
            uint4 w[UPT], last;
            const bool has_last = !WHOLE && ua < un && un > ru.whole_hi() && ru.NU - 1 >= ru.whole_lo() && ((un - 1 - ua) >> 5) % NW == warp;
            if (n >= 0) {
                for (int k = items[n & 3].zeros; k > 0; --k) {
                    const RowUnits<T, L> rz = units(row - k * ncl);
                    rz.store_zeros(reinterpret_cast<T*>(p.grad) + (long long)(row - k * ncl) * p.g_stride, ua, min(ua + p.per_cta, rz.NU), (int)threadIdx.x, NW * 32);
                }
                if (items[n & 3].kind < 0) break;
                const RowStage<T, L> st(dyn_smem + (n & 1) * kSdStage, ru, ua, un);
                uint32_t v = 0u;
                for_units<UPT>(nk, [&](int k) {
                    w[k] = st.held(unit_at(k));
                    v |= w[k].x;
                });
                if (has_last) last = st.held(ru.NU - 1);
                __reduce_or_sync(0xFFFFFFFFu, v);            // (the loads have ended)
                if (cleans(ru, un)) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_cta(bar(empty_s[n & 1]));
            }
            wait(full_s[(n + 1) & 1], (uint32_t)((n + 1) >> 1) & 1u);
            if (!alive) break;
            if (items[(n + 1) & 3].kind == 1) sum_row(items[(n + 1) & 3], n + 1);
            if (n < 0) continue;
            T* const g = reinterpret_cast<T*>(p.grad) + (long long)row * p.g_stride;
            wait(ready_s[n & 3], (uint32_t)(n >> 2) & 1u);
            if (!alive) break;
            const DeepCoef cf = coefs[n & 3];
            if (cf.zero) {
                ru.store_zeros(g, ua, un, (int)threadIdx.x, NW * 32);
                continue;
            }
            RowGrad r;
            r.c.s.L2 = L2;
            r.c.s.ns2 = r.c.s.nm2 = pair2(cf.ns);
            r.c.a2 = pair2(cf.a2);
            r.c.b2 = pair2(cf.b2);
            r.a = cf.a;
            r.b = cf.b;
            r.top = cf.top;
            const int lo = max(ua, ru.whole_lo()), hi = min(un, ru.whole_hi());
            auto write = [&](auto big) {
                constexpr bool BIG = decltype(big)::value;
                for_units<UPT>(nk, [&](int k) {
                    const uint4 v = grad_unit<T, ENT, BIG, kFmaPairs<L, ENT>>(w[k], r.c);
                    const int u = unit_at(k);
                    if ((WHOLE || k > 0 || u >= lo) && u < hi) __stcs(ru.frame(g) + u, v);
                });
                if (!WHOLE && ua == 0 && warp == 0 && ua < un && ru.whole_lo() > 0) {
                    const uint4 f = make_uint4(__shfl_sync(0xFFFFFFFFu, w[0].x, 0), __shfl_sync(0xFFFFFFFFu, w[0].y, 0),
                                               __shfl_sync(0xFFFFFFFFu, w[0].z, 0), __shfl_sync(0xFFFFFFFFu, w[0].w, 0));
                    ru.store_end(g, 0, grad_unit<T, ENT, BIG>(f, r.c));
                }
                if (has_last) ru.store_end(g, ru.NU - 1, grad_unit<T, ENT, BIG>(last, r.c));
            };
            if (cf.big) write(std::true_type{});
            else write(std::false_type{});
            // the token's own element, by a lane of the warp that wrote it
            __syncwarp();
            const int ox = ru.unit_of(x) - ua;
            if (ox >= 0 && ox < un - ua && (ox >> 5) % NW == warp && lane == (ox & 31)) grad_token<T, ENT>(g, x, cf.zx, cf.M, c1, r);
        }
    }
    cluster.sync();                                          // (nobody leaves while partials are on their way to it)
}

}  // namespace adasd
