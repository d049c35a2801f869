// Losses with a gradient on many rows (same outputs as score_kernel), where rows are short or too long for score_deep_kernel: a
// cluster takes row after row, and while a row is summed and its gradient formed from the registers that hold it, the next
// one is on its way into shared memory.
//
// A warp owns a stretch of units of every row: it asks for it with one bulk copy, takes it into registers when it has landed,
// and asks for the next row's at once, so that an SM has up to 128 KB of loads under way whatever its warps are at.  The warps'
// statistics go to every CTA of the cluster with stores that count their bytes on a barrier there; a warp waits for nothing else.
// 517 fp32 rows of 128256 logits: 93 us, 5.7 TB/s; 2000 bf16 rows of 32000: 55 us, 4.7 TB/s (the exchange of every row's totals).
#pragma once

#include "adasd_score.cuh"

namespace adasd {

constexpr int kSsUPT = 16;                                   // units a lane holds
constexpr int kSsStage = kSsUPT * 32 * 16;                   // a warp's stretch

// Statistics of a row until it is reported, 32 at a time.
struct __align__(16) RowHist {
    RowStats s;
    int32_t row, pad[3];
};

// f(k) for k < n of UPT, four at a time without a branch between them (n: warp-uniform).
template <int UPT, typename F>
__device__ __forceinline__ void for_units(int n, F f) {
#pragma unroll
    for (int k = 0; k < UPT; k += 4) {
        if (k + 4 <= UPT && n >= k + 4) {
#pragma unroll
            for (int i = k; i < (k + 4 < UPT ? k + 4 : UPT); ++i) f(i);
        } else {
#pragma unroll
            for (int i = k; i < (k + 4 < UPT ? k + 4 : UPT); ++i)
                if (i < n) f(i);
        }
    }
}

// The rows a cluster has to do, 32 at a time: lane j holds row first + (wi + j) clusters.  Rows left out are set aside.
struct RowWindow {
    int wi, row, x;
    unsigned todo, zero;                                     // lanes with rows to do, with gradient rows to zero
};

// A warp's stretch [ua, un) of a row in its stage: granule ua first.  Element e of the row is element e + off of the granules.
template <typename T, int L>
struct RowStage {
    using U = Unit<T>;
    static constexpr int N = U::N;
    static constexpr bool WHOLE = L == ROWS_WHOLE;
    unsigned char* at;
    const RowUnits<T, L>& ru;
    int ua, un, off;
    __device__ __forceinline__ RowStage(unsigned char* at_, const RowUnits<T, L>& ru_, int ua_, int un_)
        : at(at_), ru(ru_), ua(ua_), un(un_), off(WHOLE ? 0 : ru_.m0 + ru_.sh) {}
    __device__ __forceinline__ bool ends() const { return !WHOLE && ua < un && (ua == 0 || un == ru.NU); }
    // what the row's first and last granules hold of its neighbours becomes -inf, and `more` granules behind them
    __device__ __forceinline__ void clean(int more) const {
        if (!ends()) return;
        const int lane = threadIdx.x & 31;
        T* const s = reinterpret_cast<T*>(at) - (long long)ua * N;
        const long long after = (long long)off + ru.V + lane;
        if (ua == 0 && lane < off) put(s + lane, -INFINITY);
        if (un == ru.NU && after < (long long)(ru.NU + more) * N) put(s + after, -INFINITY);
        __syncwarp();
    }
    __device__ __forceinline__ uint4 held(int u) const {
        const uint4* const g = reinterpret_cast<const uint4*>(at) + (u - ua);
        static_assert(L != ROWS_ANY, "units that lie across granules are score_kernel's");
        return *g;
    }
    __device__ __forceinline__ bool owns(int x) const {
        const int u = ru.unit_of(x);
        return u >= ua && u < un;
    }
    __device__ __forceinline__ float token(int x) const {
        return to_f32(*(reinterpret_cast<const T*>(at) + (x + (long long)off - (long long)ua * N)));
    }
    // before another copy is asked for: after what every lane has read and written here
    __device__ __forceinline__ void release() const {
        if (ends()) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
    }
};

// One pair in four of a gradient's exponentials on the FMA pipe, where issue slots are left: rows without ends to look at, no
// entropy.  2048 rows of 128256 bf16: 212 -> 192 us; two pairs 203; with an entropy 407 -> 429 (4096 rows of 151936), rows off
// 16-byte boundaries 167 -> 178 (4000 rows of 50257).
template <int L, bool ENT>
constexpr int kFmaPairs = L == ROWS_WHOLE && !ENT ? 1 : 0;

// Gradient of a warp's stretch, from its registers.  last: the row's last unit where it is not whole and in this stretch.
template <typename T, int L, bool ENT, int UPT>
__device__ __forceinline__ void write_row(T* g, const uint4 (&w)[UPT], const uint4& last, bool has_last, const RowUnits<T, L>& ru, int ua,
                                          int un, int x, const RowGrad& r, const RowStats& st, float c1) {
    constexpr bool WHOLE = L == ROWS_WHOLE;
    const int lane = threadIdx.x & 31;
    if (r.zero) {
        ru.store_zeros(g, ua, un, lane, 32);
        return;
    }
    const int lo = max(ua, ru.whole_lo()), hi = min(un, ru.whole_hi());
    auto write = [&](auto big) {
        constexpr bool BIG = decltype(big)::value;
#pragma unroll
        for (int k = 0; k < UPT; k += 4) {
            if (ua + k * 32 < un) {
#pragma unroll
                for (int i = k; i < (k + 4 < UPT ? k + 4 : UPT); ++i) {
                    const int u = ua + i * 32 + lane;
                    const uint4 v = grad_unit<T, ENT, BIG, kFmaPairs<L, ENT>>(w[i], r.c);
                    if ((WHOLE || i > 0 || u >= lo) && u < hi) __stcs(ru.frame(g) + u, v);
                }
            }
        }
        if (!WHOLE && ua == 0 && ua < un && ru.whole_lo() > 0) {
            const uint4 f = make_uint4(__shfl_sync(0xFFFFFFFFu, w[0].x, 0), __shfl_sync(0xFFFFFFFFu, w[0].y, 0),
                                       __shfl_sync(0xFFFFFFFFu, w[0].z, 0), __shfl_sync(0xFFFFFFFFu, w[0].w, 0));
            ru.store_end(g, 0, grad_unit<T, ENT, BIG>(f, r.c));
        }
        if (has_last) ru.store_end(g, ru.NU - 1, grad_unit<T, ENT, BIG>(last, r.c));
    };
    if (r.big) write(std::true_type{});
    else write(std::false_type{});
    // the token's own element, by a lane of the warp that wrote it
    __syncwarp();
    const int ox = ru.unit_of(x) - ua;
    if (ox >= 0 && ox < un - ua && lane == (ox & 31)) grad_token<T, ENT>(g, x, st.zx, st.M, c1, r);
}

template <typename T, int L, int NW, bool ENT>
__global__ void __launch_bounds__(NW * 32, 16 / NW) score_stream_kernel(const __grid_constant__ ScoreParams p) {
    using U = Unit<T>;
    constexpr int N = U::N, UPT = kSsUPT;
    constexpr bool WHOLE = L == ROWS_WHOLE;
    const float floor_v = N == 8 ? ADASD_FLOOR_BF : kFloor;
    extern __shared__ __align__(128) unsigned char dyn_smem[];
    __shared__ float4 part[2][kScMaxCluster * NW];
    __shared__ unsigned long long full_s[NW], got_s[2];
    __shared__ RowHist hist[32];
    __shared__ float4 keep[NW][32];                          // RowIn of the window's rows
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
        return RowUnits<T, L>(z, reinterpret_cast<const T*>(p.grad) + (long long)row * p.g_stride, p.V);
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
        RowIn in{0.f, 0.f, 0.f, 0.f};
        if (kind == 1) in = row_in(p, (int)r);
        __syncwarp();
        keep[warp][lane] = make_float4(in.adv, in.old, in.ref, in.w);
        __syncwarp();
        win.todo = __ballot_sync(0xFFFFFFFFu, kind == 1);
        win.zero = __ballot_sync(0xFFFFFFFFu, kind == 0);
    };
    auto zero_row = [&]() {                                  // one row set aside
        const int j = __ffs(win.zero) - 1, row = __shfl_sync(0xFFFFFFFFu, win.row, j);
        win.zero &= win.zero - 1;
        const RowUnits<T, L> ru = units(row);
        T* const g = reinterpret_cast<T*>(p.grad) + (long long)row * p.g_stride;
        ru.store_zeros(g, ua, min(ub, ru.NU), lane, 32);
    };
    int row = -1, x = 0;                                     // the row asked for; -1: none left
    float4 inputs;                                           // of its loss
    auto next = [&]() {
        while (!win.todo) {
            while (win.zero) zero_row();
            row = -1;
            if ((long long)cl + (long long)(win.wi + 32) * ncl >= p.n_rows) return;
            open(win.wi + 32);
        }
        const int j = __ffs(win.todo) - 1;
        win.todo &= win.todo - 1;
        row = __shfl_sync(0xFFFFFFFFu, win.row, j);
        x = __shfl_sync(0xFFFFFFFFu, win.x, j);
        inputs = keep[warp][j];
    };
    auto ask = [&]() {                                       // its stretch: granules from unit ua's first on that hold elements
        if (lane == 0) {
            const RowUnits<T, L> ru = units(row);
            const int g0 = max(ua, ru.glo), g1 = min(min(ub, ru.NU), ru.ghi);
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
        const RowUnits<T, L> ru = units(my_row);
        const int un = min(ub, ru.NU);
        const RowIn in{inputs.x, inputs.y, inputs.z, inputs.w};
        uint64_t* const got = reinterpret_cast<uint64_t*>(&got_s[par]);
        if (CS > 1 && warp == 0 && lane == 0) mbar_expect_tx(got, (uint32_t)(CS * NW) * 16u);
        if (asked) {
            const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(full, ph));
            if (!ok && lane == 0) atomicOr(p.status, ADASD_STATUS_TIMEOUT);
            alive = alive && ok;
        }
        ph ^= 1u;
        uint32_t bad = alive ? 0u : 1u;
        const RowStage<T, L> rs(stage, ru, ua, un);
        rs.clean(0);
        uint4 w[UPT], last;
        typename U::Max mx = U::max0();
#pragma unroll
        for (int k = 0; k < UPT; ++k) {
            const int u = ua + k * 32 + lane;
            w[k] = u < un ? rs.held(u) : U::none4();
        }
        const bool has_last = !WHOLE && ua < un && un > ru.whole_hi() && ru.NU - 1 >= ru.whole_lo();
        if (has_last) last = rs.held(ru.NU - 1);
#pragma unroll
        for (int k = 0; k < UPT; ++k) U::max_add(mx, w[k]);
        const float zx = rs.owns(my_x) ? rs.token(my_x) : -INFINITY;
        if (zx != zx) bad = 1u;
        const float m = warp_max_f32(fmaxf(U::max_val(mx, bad), zx));       // (every lane's loads from the stage have ended)
        if (m == INFINITY) bad = 1u;
        next();
        asked = row >= 0 && alive;
        rs.release();
        if (asked) ask();
        const float2 sums = sum_units<T, ENT, UPT>(w, m, c1, L2, [&](int k) { return ua + k * 32 < un; });
        const float4 mine = make_float4(m, __any_sync(0xFFFFFFFFu, bad) ? NAN : sums.x, sums.y, zx);
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
        const RowGrad r = row_grad(p, in, st, c1, L2, ENT);
        T* const g = reinterpret_cast<T*>(p.grad) + (long long)my_row * p.g_stride;
        write_row<T, L, ENT, UPT>(g, w, last, has_last, ru, ua, un, my_x, r, st, c1);
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
    if (CS > 1) cluster.sync();                      // (nobody leaves while a warp's partials are on their way to it)
}

}  // namespace adasd
