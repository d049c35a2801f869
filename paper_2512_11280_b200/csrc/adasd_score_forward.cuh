// Log-probs, entropies and losses without a gradient on many rows (same outputs as score_kernel): a cluster (of one CTA, where there
// are rows enough) takes row after row, and no warp waits for another's sums.
//
// A warp owns a stretch of units of every row.  Its lanes fetch their own 16-byte units through a ring in shared memory, sixteen
// ahead, across the ends of rows: a lane reads only what it has fetched itself, so that nothing is signalled or waited for but its
// own copies.  A lane keeps the sums of its units under its own shift s (raised with its largest logit): S = sum 2^(z c1 - s),
// one rounding in every exponent.  Rows whose largest logit has a shift beyond 1e7 are summed again (big_sums).  A warp keeps its partials of 32 rows; then all warps of the cluster fold them, a few
// rows each, and report them a row a lane.
//
// What bounds it: memory for fp32, memory and the special-function pipe (75 % busy: one 2^t a logit) for bf16.  3300 rows of
// 128256 bf16 logits 138 us (6.1 TB/s), 1776 fp32 rows of 50256 63 us (5.7 TB/s).  Bulk copies instead of the lanes' own, each
// with as many bytes under way: a warp's stretch of 8 KB 168 us, pieces of 4 KB 168 and 86, a CTA's pieces of 32 KB asked for
// by a control warp 152 and 92: a stage is free only when its last reader has read it, and waiting for it is polling.
#pragma once

#include "adasd_score_stream.cuh"

namespace adasd {

constexpr int kSfGroup = 4;                                  // units of a lane that are fetched and summed together
constexpr int kSfRing = 4;                                   // groups of a warp's ring
constexpr int kSfGroupB = kSfGroup * 32 * 16;
constexpr int kSfRingB = kSfRing * kSfGroupB;
constexpr int kSfWarps = 24;                                 // of an SM

__device__ __forceinline__ void fetch16(uint32_t smem, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(src) : "memory");
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void fetch_wait() {               // until LEFT groups are under way
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// Sums of a warp's stretch [u0, un) of a row under its largest logit m, from memory: logits (or 1 / T) so large that a shift
// m c1 lies whole powers of two off.
template <typename T, int L, bool ENT>
__device__ __noinline__ float2 big_sums(const RowUnits<T, L>& ru, int u0, int un, float m, float c1) {
    float2 S2 = make_float2(0.f, 0.f), T2 = make_float2(0.f, 0.f);
    const Shift c = sum_shift(m, c1, pair2(c1));
    for (int u = u0 + (int)(threadIdx.x & 31); u < un; u += 32) add_unit<T, ENT, true>(ru.load(u), c, S2, T2);
    return make_float2(warp_sum(S2.x + S2.y), ENT ? warp_sum(T2.x + T2.y) : 0.f);
}

// {S, T} of a warp under its largest logit M from its lanes' under their shifts s.
template <bool ENT>
__device__ __forceinline__ float2 join_lanes(float2 S2, float2 T2, float s, float M, float c1, float floor_v) {
    if (!(M > floor_v)) return make_float2(0.f, 0.f);
    const float sM = M * c1, d = fmaxf(s - sM, kLowT), f = ex2(d);
    float2 r;
    r.x = warp_sum(f * (S2.x + S2.y));
    r.y = ENT ? warp_sum(f * fmaf(d, S2.x + S2.y, T2.x + T2.y)) : 0.f;
    const float tm = fmaf(M, c1, -sM), em = ex2(tm);         // (as finish_sums)
    if (ENT) r.y = (r.y - __fmul_rn(tm, r.x)) / em;
    r.x /= em;
    return r;
}

template <typename T, int L, int NW, bool ENT>
__global__ void __launch_bounds__(NW * 32, kSfWarps / NW) score_forward_kernel(const __grid_constant__ ScoreParams p) {
    using U = Unit<T>;
    constexpr int N = U::N, G = kSfGroup;
    const float floor_v = N == 8 ? ADASD_FLOOR_BF : kFloor;
    extern __shared__ __align__(128) unsigned char dyn_smem[];
    // 32 rows of partials, twice: those of one set of rows are folded by others while the next set's are formed
    __shared__ float4 keep[2][NW][32];
    __shared__ int rows_s[2][32];
    __shared__ int2 ahead[NW][8];                            // rows whose units are being fetched: row, token
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CS = p.cs, ncl = (int)(gridDim.x / (unsigned)CS), cl = (int)(blockIdx.x / (unsigned)CS);
    const int rank = (int)(blockIdx.x - (unsigned)cl * (unsigned)CS);
    unsigned char* const ring = dyn_smem + warp * kSfRingB + lane * 16;
    const uint32_t ring_u = smem_u32(ring);
    cg::cluster_group cluster = cg::this_cluster();
    pdl_wait();
    pdl_trigger();

    const int ua = (rank * NW + warp) * p.per_cta, NG = p.pieces;        // (per_cta: units of a WARP here, in p.pieces groups)
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
    // ---- fetching: group far_g of row far, kSfRing groups ahead of the one that is summed -----------
    const uint4* far_src = nullptr;                          // this lane's unit of the group (null: no more rows)
    int far_row = -1, far_left = 0, far_g = 0, head = 0, tail = 0;       // far_left: units of the stretch from the lane's on
    auto next = [&]() {
        far_row = -1;
        far_g = 0;
        int x = 0;
        while (!win.todo) {
            if ((long long)cl + (long long)(win.wi + 32) * ncl >= p.n_rows) break;
            open(win.wi + 32);
        }
        if (win.todo) {
            const int j = __ffs(win.todo) - 1;
            win.todo &= win.todo - 1;
            far_row = __shfl_sync(0xFFFFFFFFu, win.row, j);
            x = __shfl_sync(0xFFFFFFFFu, win.x, j);
            const RowUnits<T, L> ru = units(far_row);
            far_src = ru.src + ua + lane;
            far_left = min(ua + p.per_cta, ru.NU) - ua - lane;
        }
        if (lane == 0) ahead[warp][head & 7] = make_int2(far_row, x);
        ++head;
        __syncwarp();
    };
    auto fetch = [&](int slot) {                             // (a group is committed, of however few copies: they are counted)
        if (far_row >= 0) {
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (32 * i < far_left) fetch16(ring_u + slot * kSfGroupB + i * 512, far_src + 32 * i);
            far_src += 32 * G;
            far_left -= 32 * G;
        }
        fetch_commit();
        if (far_row >= 0 && ++far_g == NG) next();
    };
    open(0);
    next();
#pragma unroll 1
    for (int k = 0; k < kSfRing; ++k) fetch(k);

    const float c1 = p.c1;
    const float2 L2 = pair2(c1);
    int slot = 0;
    for (int done = 0;; ++done) {
        const int2 cur = ahead[warp][tail & 7];
        ++tail;
        const int row = cur.x, x = cur.y, set = done >> 5 & 1, at = done & 31;
        if ((at == 0 && done > 0) || row < 0) {
            // 32 rows, or the last ones.  (Whoever comes here has folded the set before: its place may be written again.)
            const int fold = (done - 1) >> 5 & 1, n = done == 0 ? 0 : ((done - 1) & 31) + 1;
            if (CS > 1) cluster.sync();
            else __syncthreads();
            RowStats st;
            int cnt = 0, which = 0;
            for (int j = rank * NW + warp; j < n; j += CS * NW, ++cnt) {
                const RowStats f = fold_partials<kScMaxCluster * NW>(
                    [&](int k) { return *cluster.map_shared_rank(&keep[fold][k % NW][j], k / NW); }, CS * NW, c1, floor_v);
                if (lane == cnt) {
                    st = f;
                    which = rows_s[fold][j];
                }
            }
            if (lane < cnt) row_report(p, which, row_in(p, which), st);
            if (row < 0) break;
        }
        const RowUnits<T, L> ru = units(row);
        const int un = min(ua + p.per_cta, ru.NU);
        const float zx = to_f32((reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride)[x]);
        float m = -INFINITY, s = -kBigShift;                 // the lane's largest logit and its shift (nothing big: see below)
        float2 S2 = make_float2(0.f, 0.f), T2 = make_float2(0.f, 0.f);
        typename U::Max mx = U::max0();
#pragma unroll 1
        for (int g = 0; g < NG; ++g) {
            fetch_wait<kSfRing - 1>();
            const int u0 = ua + g * 32 * G + lane;
            uint4 w[G];
#pragma unroll
            for (int i = 0; i < G; ++i) w[i] = *reinterpret_cast<const uint4*>(ring + slot * kSfGroupB + i * 512);
            if (ua + (g + 1) * 32 * G > un || (L != ROWS_WHOLE && (g == 0 || ua + (g + 1) * 32 * G == ru.NU))) {
#pragma unroll
                for (int i = 0; i < G; ++i) {                // ends of the stretch and of the row
                    const int u = u0 + 32 * i;
                    if (u >= un) w[i] = U::none4();
                    else if (L != ROWS_WHOLE && (u == 0 || u == ru.NU - 1))
                        U::mask(w[i], u == 0 ? ru.m0 : 0, (int)min((long long)N, (long long)ru.V + ru.m0 - (long long)u * N));
                }
            }
            typename U::Max h = U::unit_max(w[0]);
#pragma unroll
            for (int i = 1; i < G; ++i) U::max_add(h, w[i]);
            U::max_join(mx, h);
            asm volatile("" ::"r"(U::bits(h)) : "memory");      // (the lane's loads from the slot have ended)
            fetch(slot);
            if (++slot == kSfRing) slot = 0;
            // the sums move to the shift of the largest logit so far
            m = fmaxf(m, U::top(h));
            const float ns = fmaxf(m * c1, -kBigShift), d = s - ns, f = ex2(d);
            if (ENT) {
                const float dc = fmaxf(d, kLowT);
                T2.x = f * fmaf(dc, S2.x, T2.x);
                T2.y = f * fmaf(dc, S2.y, T2.y);
            }
            S2.x *= f;
            S2.y *= f;
            s = ns;
            Shift c;
            c.L2 = L2;
            c.ns2 = c.nm2 = make_float2(-s, -s);
#pragma unroll
            for (int i = 0; i < G; ++i) add_unit<T, ENT, false>(w[i], c, S2, T2);
        }
        uint32_t bad = 0u;
        const float v = U::max_val(mx, bad), M = warp_max_f32(v);
        if (M == INFINITY) bad = 1u;
        const float2 r = M > floor_v && big_shift(M, c1) ? big_sums<T, L, ENT>(ru, ua, un, M, c1) : join_lanes<ENT>(S2, T2, s, M, c1, floor_v);
        const bool any_bad = __any_sync(0xFFFFFFFFu, bad);
        if (lane == 0) {
            keep[set][warp][at] = make_float4(M, any_bad ? NAN : r.x, r.y, zx);
            if (warp == 0) rows_s[set][at] = row;
        }
    }
    if (CS > 1) cluster.sync();                              // (nobody leaves while others read its partials)
}

}  // namespace adasd
