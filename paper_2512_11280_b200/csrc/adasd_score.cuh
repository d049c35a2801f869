// Scoring and losses of given tokens for sm_100a: log-probs and entropies of rows of logits, and the gradients
// with respect to the logits of losses made of them.
//
// A row z, the token x that stands there, T the temperature, m the largest logit, S = sum 2^((z - m) log2 e / T):
//   l = (z_x - m) / T - ln S,   p_v = 2^((z_v - m) log2 e / T) / S,   H = ln S - (1/S) sum p'_v ln p'_v  (p' = S p)
//   dL/dz_v = (dL/dl (1[v = x] - p_v) - dL/dH p_v (ln p_v + H)) / T
// dL/dl and dL/dH hang on the row's own l and H alone (policy loss) or are given, so one launch reads a row, forms
// its statistics and writes its gradient.  In a preference loss they hang on all rows of a pair: score_kernel leaves
// the statistics, pref_pair_kernel forms the pairs' losses, pref_grad_kernel reads the rows again.
//
// score_kernel takes few rows, rows whose gradient lies elsewhere relative to 16 bytes, and rows too long for the
// others: a cluster of CTAs a row; a thread loads its 16-byte units into registers, and they stay
// there between the sums and the gradient, so that a row crosses the memory once each way.  (Rows of more than 32768 units are
// read again: policy loss with a gradient, 1000 fp32 rows of 131072 by score_stream_kernel 180 us, of 151936 by this one 369.  Without a
// pipeline of rows: 2000 rows of 128249 bf16 that are a slice of 128256, gradient dense, 470 us; 2000 of 128256 the ordinary way 186.)  The warps' statistics go
// to every CTA of the cluster (one barrier) and are folded by each warp in the same order.  What bounds it is the chain
// launch -> load -> cluster barrier -> fold -> store: 7 fp32 rows of 32000 logits with a gradient 7 us.
//
// Many rows: score_forward_kernel (no gradient; adasd_score_forward.cuh), score_deep_kernel and score_stream_kernel (with one).
// pref_grad_kernel is bound by memory: 3300 rows of 128256 bf16 logits 244 us, 6.9 TB/s; with the rows' statistics 138 us.
#pragma once

#include "adasd_async.cuh"
#include "adasd_score_types.cuh"

#include <type_traits>

namespace adasd {

constexpr int kScMaxCluster = 8;
constexpr float kLowT = -16384.f;          // 2^t = 0 from here down; keeps 0 * (-inf) out of the sums

// A row's units of 16 bytes, aligned in the memory of the array that decides: the gradient's row where one is written
// (so that whole units are stored at once), else the logits'.  Unit u holds elements u N - m0 .. u N - m0 + N - 1; logits that
// lie elsewhere relative to 16 bytes are put together from two granules (ROWS_ANY).  ROWS_SAME: no row does.  ROWS_WHOLE: rows start
// on 16-byte boundaries and V is a multiple of N, so that no unit needs a look at its ends.
enum Layout : int { ROWS_WHOLE, ROWS_SAME, ROWS_ANY };
template <typename T, int L>
struct RowUnits {
    using U = Unit<T>;
    static constexpr int N = U::N;
    static constexpr bool WHOLE = L == ROWS_WHOLE;
    const uint4* src;                      // granule that unit 0 starts in
    int m0, sh;                            // elements before the row in unit 0; elements of src's granule before unit 0
    int glo, ghi;                          // granules that hold elements of the row
    int V, NU;

    __device__ __forceinline__ RowUnits(const T* z, const T* frame, int V_) : V(V_) {
        const unsigned long long a = reinterpret_cast<unsigned long long>(z);
        if (WHOLE) {
            src = reinterpret_cast<const uint4*>(z);
            m0 = sh = glo = 0;
            NU = ghi = V / N;
        } else {
            m0 = (int)((reinterpret_cast<unsigned long long>(frame) & 15ull) / sizeof(T));
            NU = (int)(((long long)m0 + V + N - 1) / N);
            const unsigned long long s = a - (unsigned long long)m0 * sizeof(T), b = s & ~15ull;
            src = reinterpret_cast<const uint4*>(b);
            sh = L == ROWS_ANY ? (int)((s & 15ull) / sizeof(T)) : 0;
            glo = (int)(((a & ~15ull) - b) >> 4);
            ghi = (int)((a + (unsigned long long)V * sizeof(T) + 15ull - b) >> 4);
        }
    }
    // unit u from its granule and the next (get(g): granule g of those that hold elements); elements outside the row: -inf
    template <typename F>
    __device__ __forceinline__ uint4 unit(int u, F get) const {
        if (WHOLE) return get(u);
        uint4 w = u >= glo && u < ghi ? get(u) : U::none4();
        if (L == ROWS_ANY && sh) w = U::realign(w, u + 1 < ghi ? get(u + 1) : U::none4(), sh);
        if (u == 0 || u == NU - 1) U::mask(w, u == 0 ? m0 : 0, (int)min((long long)N, (long long)V + m0 - (long long)u * N));
        return w;
    }
    __device__ __forceinline__ uint4 load(int u) const {
        return unit(u, [&](int g) { return __ldcg(src + g); });
    }
    __device__ __forceinline__ int unit_of(int v) const { return (int)(((long long)v + (WHOLE ? 0 : m0)) / N); }
    // where unit 0 of row g would start
    __device__ __forceinline__ uint4* frame(T* g) const { return reinterpret_cast<uint4*>(g - (WHOLE ? 0 : m0)); }
    // units that lie in the row from end to end: [whole_lo, whole_hi)
    __device__ __forceinline__ int whole_lo() const { return WHOLE || m0 == 0 ? 0 : 1; }
    __device__ __forceinline__ int whole_hi() const { return WHOLE || (m0 + V) % N == 0 ? NU : NU - 1; }
    // for the gradient alone: unit u whose elements outside the row hold anything (the nearest granules that may be read)
    __device__ __forceinline__ uint4 load_any(int u) const {
        if (WHOLE) return __ldcg(src + u);
        uint4 w = __ldcg(src + min(max(u, glo), ghi - 1));
        if (L == ROWS_ANY && sh) w = U::realign(w, __ldcg(src + min(max(u + 1, glo), ghi - 1)), sh);
        return w;
    }
    // unit u of row g where it is the row's first or last and not whole: its elements, one a lane (by a whole warp)
    __device__ __forceinline__ void store_end(T* g, int u, const uint4& w) const {
        const int j = threadIdx.x & 31;
        const long long e = (long long)u * N - m0 + j;
        const uint32_t q = j * (int)sizeof(T) < 8 ? (j * (int)sizeof(T) < 4 ? w.x : w.y) : (j * (int)sizeof(T) < 12 ? w.z : w.w);
        if (j < N && e >= 0 && e < V) {
            if (sizeof(T) == 2) reinterpret_cast<uint16_t*>(g)[e] = (uint16_t)(q >> (16 * (j & 1)));
            else reinterpret_cast<uint32_t*>(g)[e] = q;
        }
    }
    // ... and units of zeros, [u0, u1) by the threads t, t + n, .. of a group of whole warps
    __device__ __forceinline__ void store_zeros(T* g, int u0, int u1, int t, int n) const {
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        const int lo = max(u0, whole_lo()), hi = min(u1, whole_hi());
        for (int u = lo + t; u < hi; u += n) __stcs(frame(g) + u, zero);
        if (!WHOLE && t < 32) {
            if (u0 < u1 && u0 < whole_lo()) store_end(g, 0, zero);
            if (u0 < u1 && u1 > whole_hi() && NU - 1 >= whole_lo()) store_end(g, NU - 1, zero);
        }
    }
};

__device__ __forceinline__ uint4 pack16(const float2 (&v)[4]) {
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r[j]) : "f"(v[j].y), "f"(v[j].x));
    return make_uint4(r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ uint4 pack16(const float2 (&v)[2]) {
    return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
}
__device__ __forceinline__ void put(__nv_bfloat16* at, float v) { *at = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* at, float v) { *at = v; }

// Exponents.  t = (z - m) log2 e / T is formed as fma(z, c1, -s) with s = fl(m c1), one rounding, good however large the
// logits' common offset; what s is off by is taken back from the sums (at t_m = fma(m, c1, -s), the exponent that the
// largest logit gets instead of 0).  BIG: (z - m) c1, where offsets or 1 / T are so large that t_m is off by whole powers of
// two, or T so large that the exponent of -1e30, which stands for a masked logit there, is not small.
constexpr float kBigShift = 1e7f, kLowScale = 1e-20f;
__device__ __forceinline__ bool big_shift(float m, float c1) {
    return !(fabsf(m * c1) < (c1 < kBigShift && c1 >= kLowScale ? kBigShift : 0.f));
}
struct Shift {
    float2 L2, ns2, nm2;                   // c1; -s; -m
};
// ENT: the exponents are factors too and have to be finite: logits of -inf (of bf16 rows: two at a time) or exponents are clamped.
template <typename T, bool ENT, bool BIG>
__device__ __forceinline__ void exponents(const uint4& w, const Shift& c, float2 (&q)[Unit<T>::N / 2]) {
    constexpr bool CLAMP = ENT && !BIG;
    if (CLAMP && sizeof(T) == 2) Unit<T>::unpack(w, q);
    else Unit<T>::unpack_raw(w, q);
#pragma unroll
    for (int j = 0; j < Unit<T>::N / 2; ++j) {
        q[j] = BIG ? __fmul2_rn(__fadd2_rn(q[j], c.nm2), c.L2) : __ffma2_rn(q[j], c.L2, c.ns2);
        if (ENT && !(CLAMP && sizeof(T) == 2)) q[j] = make_float2(fmaxf(q[j].x, kLowT), fmaxf(q[j].y, kLowT));
    }
}

// 2^q on the FMA pipe, q <= 126: 2^n 2^f with n = q rounded, f in [-1/2, 1/2], 2^f by the degree-4 polynomial of least relative
// error there (fitted by reweighted least squares): 2.64e-6, 2.7e-6 with its roundings, against 2^-22 of ex2.  For gradients that are
// rounded to bf16 alone (up to 2^-8 of the value).  0 from -125 down, exactly: what the clamped argument gives is taken off every value.
__device__ __forceinline__ float2 exp2_fma(float2 q) {
    const float2 big = make_float2(12582912.f, 12582912.f);              // 1.5 2^23: the sum's last bit is 1
    constexpr float least = 9.999992847442627e-1f * 0x1p-125f;           // (exact)
    q = make_float2(fmaxf(q.x, -125.f), fmaxf(q.y, -125.f));
    const float2 r = __fadd2_rn(q, big);
    const float2 f = __ffma2_rn(__fadd2_rn(r, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), q);
    float2 y = __ffma2_rn(f, make_float2(9.570102207362652e-3f, 9.570102207362652e-3f), make_float2(5.591785907745361e-2f, 5.591785907745361e-2f));
    y = __ffma2_rn(y, f, make_float2(2.40247443318367e-1f, 2.40247443318367e-1f));
    y = __ffma2_rn(y, f, make_float2(6.931217908859253e-1f, 6.931217908859253e-1f));
    y = __ffma2_rn(y, f, make_float2(9.999992847442627e-1f, 9.999992847442627e-1f));
    y = make_float2(__int_as_float(__float_as_int(y.x) + (__float_as_int(r.x) << 23)), __int_as_float(__float_as_int(y.y) + (__float_as_int(r.y) << 23)));
    return __fadd2_rn(y, make_float2(-least, -least));
}

// dL/dz of a unit: 2^q (b + a q); BIG: 2^q b + (2^q q) a, where 2^q q is 0 however large a is.  FMA: pairs (of a bf16 unit's
// four) whose 2^q comes from the FMA pipe.
struct GradConsts {
    Shift s;
    float2 a2, b2;
};
template <typename T, bool ENT, bool BIG, int FMA = 0>
__device__ __forceinline__ uint4 grad_unit(const uint4& w, const GradConsts& c) {
    using U = Unit<T>;
    float2 q[U::N / 2];
    exponents<T, ENT, BIG>(w, c.s, q);
#pragma unroll
    for (int j = 0; j < U::N / 2; ++j) {
        const float2 e = sizeof(T) == 2 && !BIG && j < FMA ? exp2_fma(q[j]) : make_float2(ex2(q[j].x), ex2(q[j].y));
        q[j] = ENT && BIG ? __ffma2_rn(__fmul2_rn(e, q[j]), c.a2, __fmul2_rn(e, c.b2)) : __fmul2_rn(e, ENT ? __ffma2_rn(q[j], c.a2, c.b2) : c.b2);
    }
    return pack16(q);
}

// Inputs of a row's loss.
struct RowIn {
    float adv, old, ref, w;                // SCORE_GIVEN: dL/dl, dL/dH in the first two
};
__device__ __forceinline__ RowIn row_in(const ScoreParams& p, int row) {
    RowIn r{0.f, 0.f, 0.f, 1.f};
    if (p.op == SCORE_GIVEN) {
        r.adv = __ldcg(p.g_logp + row);
        if (p.g_H) r.old = __ldcg(p.g_H + row);
    } else if (p.op == SCORE_POLICY) {
        r.adv = __ldcg(p.adv + row);
        if (p.old_logp) r.old = __ldcg(p.old_logp + row);
        if (p.ref_logp) r.ref = __ldcg(p.ref_logp + row);
        if (p.weight) r.w = __ldcg(p.weight + row);
    }
    return r;
}
// Whether a row is left out.
__device__ __forceinline__ bool row_out(const ScoreParams& p, int row, int x) {
    bool out = x < 0 || x >= p.V;
    if (p.op == SCORE_POLICY && p.weight) out = out || __ldcg(p.weight + row) == 0.f;
    if (p.op == SCORE_GIVEN) out = out || (__ldcg(p.g_logp + row) == 0.f && (!p.g_H || __ldcg(p.g_H + row) == 0.f));
    return out;
}

// Terms of the policy loss and its derivatives, without the weight.  F: float for the gradient's coefficients, double for what
// is reported (KL estimates of 1e-3 and less, totals of terms of either sign).  The differences of log-probs come as such:
// rounded after they are formed.
template <typename F>
__device__ __forceinline__ void policy_terms(const ScoreParams& p, const RowIn& in, F l_old, F ref_l, F H, F& loss, F& k3, F& dl, F& dH) {
    const F A = (F)in.adv, ratio = p.old_logp ? exp(l_old) : l_old == l_old ? (F)1 : l_old;
    loss = dl = dH = k3 = (F)0;
    if (A != (F)0) {                       // (0 times an overflowed ratio is no term either)
        const F lo = (F)1 - (F)p.clip_low, hi = (F)1 + (F)p.clip_high;
        const F s1 = ratio * A, s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * A;
        loss = s1 <= s2 ? -s1 : s2 == s2 ? -s2 : s1;
        if (!(s1 > s2)) dl = -s1;
    } else if (ratio != ratio) {
        loss = dl = ratio;
    }
    if (p.ref_logp) {
        const F e = expm1(ref_l);
        k3 = e < (F)INFINITY ? e - ref_l : e;
        if (p.kl_coef != 0.f) {
            loss += (F)p.kl_coef * k3;
            dl -= (F)p.kl_coef * e;
        }
    }
    if (p.ent_coef != 0.f) {
        loss -= (F)p.ent_coef * H;
        dH = -(F)p.ent_coef;
    }
}

// Statistics of a row: largest logit, S, T = sum 2^t t, the token's logit.
struct RowStats {
    float M, S, Ts, zx;
};

// dL/dl and dL/dH.  lnS: its logarithm in 32 bits, which is as good as S.
__device__ __forceinline__ float2 row_coefs(const ScoreParams& p, const RowIn& in, const RowStats& s, float lnS, float H) {
    const double l = ((double)s.zx - (double)s.M) * p.inv_temp - (double)lnS;
    if (p.op == SCORE_GIVEN) return make_float2(l == l ? in.adv : (float)l, in.old);
    float loss, k3, dl, dH;
    policy_terms<float>(p, in, (float)(l - (double)in.old), (float)((double)in.ref - l), H, loss, k3, dl, dH);
    const float w = p.scale * in.w;
    return make_float2(w * dl, w * dH);
}

// What a row reports, by one thread, in 64 bits.
__device__ __forceinline__ void row_report(const ScoreParams& p, int row, const RowIn& in, const RowStats& s) {
    if (s.S != s.S) atomicOr(p.status, ADASD_STATUS_NAN);
    if (p.op == SCORE_PREF) {
        p.pref[row] = PrefRow{s.M, s.S, s.zx - s.M, 1};
        return;
    }
    if (p.op == SCORE_GIVEN) return;
    const double lnS = log((double)s.S), l = ((double)s.zx - (double)s.M) * p.inv_temp - lnS;
    const double H = lnS - 0.69314718055994530942 * ((double)s.Ts / (double)s.S);
    if (p.logp) p.logp[row] = (float)l;
    if (p.H) p.H[row] = (float)H;
    if (p.lse) p.lse[row] = (float)((double)s.M * p.inv_temp + lnS);
    if (p.op == SCORE_POLICY) {
        double loss, k3, dl, dH;
        policy_terms<double>(p, in, l - (double)in.old, (double)in.ref - l, H, loss, k3, dl, dH);
        p.row_loss[row] = (float)((double)p.scale * (double)in.w * loss);
        if (p.kl) p.kl[row] = (float)k3;
    }
}
// ... and one that is left out.  kind: -1 in no sequence (SCORE_PREF)
__device__ __forceinline__ void row_report_out(const ScoreParams& p, int row, int kind) {
    if (p.logp) p.logp[row] = 0.f;
    if (p.H) p.H[row] = 0.f;
    if (p.lse) p.lse[row] = 0.f;
    if (p.row_loss) p.row_loss[row] = 0.f;
    if (p.kl) p.kl[row] = 0.f;
    if (p.op == SCORE_PREF) p.pref[row] = PrefRow{0.f, 0.f, 0.f, kind};
}
// kind of a row of SCORE_PREF (-1: in no sequence), 0 left out, 1 counted
__device__ __forceinline__ int row_kind(const ScoreParams& p, int row, int x) {
    if (p.op == SCORE_PREF) {
        const int first = max(0, __ldcg(p.seq_start)), end = min(p.n_rows, __ldcg(p.seq_start + p.n_seqs));
        if (row < first || row >= end) return -1;
    }
    return row_out(p, row, x) ? 0 : 1;
}

// Totals of a row from its warps' partials {m, S (NaN: unusable), T, the token's logit or -inf}, by a whole warp, in the same
// order in every warp.  get(k): partial k of n.
template <int MOST, typename F>
__device__ __forceinline__ RowStats fold_partials(F get, int n, float c1, float floor_v) {
    constexpr int PL = (MOST + 31) / 32;      // partials of a lane
    const int lane = threadIdx.x & 31;
    float4 q[PL];
    RowStats r;
    r.M = r.zx = -INFINITY;
#pragma unroll
    for (int k = 0; k < PL; ++k) {
        q[k] = lane + 32 * k < n ? get(lane + 32 * k) : make_float4(-INFINITY, 0.f, 0.f, -INFINITY);
        r.M = fmaxf(r.M, q[k].x);
        r.zx = fmaxf(r.zx, q[k].w);
    }
    r.M = warp_max_f32(r.M);
    r.zx = warp_max_f32(r.zx);
    r.S = r.Ts = 0.f;
#pragma unroll
    for (int k = 0; k < PL; ++k) {
        const float d = fmaxf((q[k].x - r.M) * c1, kLowT), f = ex2(d);
        r.S = fmaf(f, q[k].y, r.S);
        r.Ts = fmaf(f, fmaf(d, q[k].y, q[k].z), r.Ts);
    }
    r.S = warp_sum(r.S);
    r.Ts = warp_sum(r.Ts);
    if (!(r.M > floor_v)) r.S = NAN;
    return r;
}

// Sums of a warp's units under their largest logit m: what sum_units returns is {S, T} of the whole warp.  (m = -inf: a warp
// without a logit, whose exponents at a small 1 / c1 have to be clamped like everybody's.)
__device__ __forceinline__ bool sum_big(float m, float c1) { return big_shift(m > -INFINITY ? m : 0.f, c1); }
__device__ __forceinline__ Shift sum_shift(float m, float c1, float2 L2) {
    Shift c;
    c.L2 = L2;
    const float mm = m > -INFINITY ? m : 0.f;
    c.ns2 = c.nm2 = pair2(sum_big(m, c1) ? -mm : -(mm * c1));
    return c;
}
template <typename T, bool ENT, bool BIG>
__device__ __forceinline__ void add_unit(const uint4& w, const Shift& c, float2& S2, float2& T2) {
    using U = Unit<T>;
    float2 q[U::N / 2];
    exponents<T, ENT, BIG>(w, c, q);
#pragma unroll
    for (int j = 0; j < U::N / 2; ++j) {
        const float2 e = make_float2(ex2(q[j].x), ex2(q[j].y));
        S2 = __fadd2_rn(S2, e);
        if (ENT) T2 = __ffma2_rn(e, q[j], T2);
    }
}
template <bool ENT>
__device__ __forceinline__ float2 finish_sums(float2 S2, float2 T2, float m, float c1) {
    float2 r = make_float2(warp_sum(S2.x + S2.y), ENT ? warp_sum(T2.x + T2.y) : 0.f);
    if (sum_big(m, c1)) return r;
    const float mm = m > -INFINITY ? m : 0.f, tm = fmaf(mm, c1, -(mm * c1)), em = ex2(tm);
    if (ENT) r.y = (r.y - __fmul_rn(tm, r.x)) / em;
    r.x /= em;
    return r;
}
// Adds sums {S, T} = r under the largest logit t to those under m.
__device__ __forceinline__ void fold_sums(float& m, float& S, float& Ts, float t, float2 r, float c1) {
    const float n = fmaxf(m, t), d0 = m > -INFINITY ? fmaxf((m - n) * c1, kLowT) : kLowT, d1 = t > -INFINITY ? fmaxf((t - n) * c1, kLowT) : kLowT;
    const float f0 = ex2(d0), f1 = ex2(d1);
    Ts = f0 * fmaf(d0, S, Ts) + f1 * fmaf(d1, r.x, r.y);
    S = f0 * S + f1 * r.x;
    m = n;
}
// Units held in registers, in groups of four; used(k): whether group k can hold anything (warp-uniform).
template <typename T, bool ENT, int UPT, typename F>
__device__ __forceinline__ float2 sum_units(const uint4 (&w)[UPT], float m, float c1, float2 L2, F used) {
    const Shift c = sum_shift(m, c1, L2);
    float2 S2 = make_float2(0.f, 0.f), T2 = make_float2(0.f, 0.f);
    auto all = [&](auto big) {
#pragma unroll
        for (int k = 0; k < UPT; k += 4) {
            if (used(k)) {
#pragma unroll
                for (int i = k; i < k + 4; ++i) add_unit<T, ENT, decltype(big)::value>(w[i], c, S2, T2);
            }
        }
    };
    if (sum_big(m, c1)) all(std::true_type{});
    else all(std::false_type{});
    return finish_sums<ENT>(S2, T2, m, c1);
}

// What the gradient of a row takes: its constants, and the token's own element.
struct RowGrad {
    GradConsts c;
    float a, b, top;
    bool zero, big;
};
// dL/dz_v = p_v (b + a log2 p_v) = 2^t / S (b + a (t - log2 S)), t = (z_v - M) c1
__device__ __forceinline__ void grad_consts(RowGrad& r, const RowStats& s, float c1, float2 L2, float a, float b) {
    const float rS = 1.f / s.S, h = s.M * c1;
    r.a = a * rS;
    r.b = fmaf(-a, log2f(s.S), b) * rS;
    // (a q has to be finite at a masked logit too, whose 2^q is 0: bf16 units clamp the logit, to -1e30, not the exponent)
    r.big = big_shift(s.M, c1) || (a != 0.f && !(fabsf(r.a) * (1e30f * c1 + fabsf(h)) < 1e38f));
    r.c.s.L2 = L2;
    // t = fma(z, c1, -h) + x, x = h - M c1 exactly: 2^x goes to the constants
    const float x = r.big ? 0.f : -fmaf(s.M, c1, -h), f = ex2(x);
    r.c.s.ns2 = r.c.s.nm2 = pair2(r.big ? -s.M : -h);
    r.c.a2 = pair2(f * r.a);
    r.c.b2 = pair2(f * fmaf(r.a, x, r.b));
}
// The token's own element has dL/dl / T on top.
template <typename T, bool ENT>
__device__ __forceinline__ void grad_token(T* g, int x, float zx, float m, float c1, const RowGrad& r) {
    float t = (zx - m) * c1;
    if (ENT) t = fmaxf(t, kLowT);
    const float e = ex2(t), v = fmaf(e, r.b, r.top);
    put(g + x, ENT ? fmaf(e * t, r.a, v) : v);
}
__device__ __forceinline__ RowGrad row_grad(const ScoreParams& p, const RowIn& in, const RowStats& s, float c1, float2 L2, bool ent) {
    RowGrad r;
    const float lnS = logf(s.S), H = ent ? lnS - kLn2 * (s.Ts / s.S) : 0.f, iT = (float)p.inv_temp;
    const float2 d = row_coefs(p, in, s, lnS, H);
    r.zero = d.x == 0.f && d.y == 0.f;
    r.top = d.x * iT;
    grad_consts(r, s, c1, L2, ent ? -kLn2 * d.y * iT : 0.f, (ent ? fmaf(-d.y, H, -d.x) : -d.x) * iT);
    return r;
}
// ... by the thread that wrote it: of the NT that dealt units [u0, u1) among themselves, whole ones lo .. hi - 1; the ends' by
// the first warp
template <typename T, bool ENT, int NT>
__device__ __forceinline__ void grad_token_by(T* g, int x, int ux, int u0, int u1, int lo, int hi, float zx, float m, float c1,
                                              const RowGrad& r) {
    if (ux < u0 || ux >= u1) return;
    const unsigned t = ux >= lo && ux < hi ? (unsigned)(ux - u0) % NT : 0u;
    if ((threadIdx.x >> 5) == (t >> 5)) {
        __syncwarp();
        if (threadIdx.x == t) grad_token<T, ENT>(g, x, zx, m, c1, r);
    }
}

// L: as RowUnits.  NW warps a CTA, UPT units a thread.  HOLD: a CTA's units
// fit its registers; else (rows longer than the cluster holds) they are taken in turn and read again for the gradient.
// GRAD: a gradient is written.  ENT: the entropy or its gradient is wanted.
template <typename T, int L, int NW, int UPT, bool HOLD, bool GRAD, bool ENT>
__global__ void __launch_bounds__(NW * 32, 16 / NW) score_kernel(const __grid_constant__ ScoreParams p) {
    using U = Unit<T>;
    constexpr int N = U::N, NT = NW * 32;
    constexpr bool WHOLE = L == ROWS_WHOLE;
    const float floor_v = N == 8 ? ADASD_FLOOR_BF : kFloor;
    __shared__ float4 part[kScMaxCluster * NW];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CS = p.cs, row = (int)(blockIdx.x / (unsigned)CS), rank = (int)(blockIdx.x - (unsigned)row * (unsigned)CS);
    cg::cluster_group cluster = cg::this_cluster();
    pdl_wait();
    pdl_trigger();

    const T* const z = reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride;
    T* const g = GRAD ? reinterpret_cast<T*>(p.grad) + (long long)row * p.g_stride : nullptr;
    const RowUnits<T, L> ru(z, GRAD ? g : z, p.V);
    const int u0 = min(rank * p.per_cta, ru.NU), u1 = min(u0 + p.per_cta, ru.NU);
    const int x = __ldcg(p.tok + row), kind = row_kind(p, row, x);       // (the same in every CTA of the cluster)
    if (kind != 1) {
        if (GRAD)
            ru.store_zeros(g, u0, u1, (int)threadIdx.x, NT);
        if (rank == 0 && threadIdx.x == 0) row_report_out(p, row, kind);
        return;
    }
    if (CS > 1) cluster.barrier_arrive();           // (waited for before the first remote store: that CTA has started)
    const float zx = to_f32(z[x]);
    const RowIn in = row_in(p, row);

    // ---- sums -----------------------------------------------------------------------------
    const float c1 = p.c1;
    const float2 L2 = pair2(c1);
    float m = -INFINITY, S = 0.f, Ts = 0.f;
    uint32_t bad = 0u;
    uint4 w[UPT];
    for (int base = u0; base < u1; base += NT * UPT) {
#pragma unroll
        for (int k = 0; k < UPT; ++k) {
            const int u = base + k * NT + (int)threadIdx.x;
            w[k] = u < u1 ? ru.load(u) : U::none4();
        }
        typename U::Max mx = U::max0();
#pragma unroll
        for (int k = 0; k < UPT; ++k) U::max_add(mx, w[k]);
        const float t = warp_max_f32(U::max_val(mx, bad));
        if (t == INFINITY) bad = 1u;
        const float2 r = sum_units<T, ENT, UPT>(w, t, c1, L2, [&](int k) { return base + k * NT < u1; });
        if (HOLD) {
            m = t;
            S = r.x;
            Ts = r.y;
        } else {
            fold_sums(m, S, Ts, t, r, c1);
        }
    }
    const float4 mine = make_float4(m, __any_sync(0xFFFFFFFFu, bad) ? NAN : S, Ts, zx);
    if (CS > 1) {
        cluster.barrier_wait();
        if (lane < CS) *cluster.map_shared_rank(part + rank * NW + warp, lane) = mine;
        cluster.sync();
    } else {
        if (lane == 0) part[warp] = mine;
        __syncthreads();
    }
    if (!GRAD && (rank != 0 || warp != 0)) return;
    const RowStats st = fold_partials<kScMaxCluster * NW>([&](int k) { return part[k]; }, CS * NW, c1, floor_v);

    // ---- gradient ---------------------------------------------------------------------------
    if (GRAD) {
        const RowGrad r = row_grad(p, in, st, c1, L2, ENT);
        if (r.zero) {
            ru.store_zeros(g, u0, u1, (int)threadIdx.x, NT);
        } else {
            const int lo = max(u0, ru.whole_lo()), hi = min(u1, ru.whole_hi());
            auto write = [&](auto big) {
                constexpr bool BIG = decltype(big)::value;
                // (the ends first: what follows may overwrite the logits they are made of)
                if (!WHOLE && warp == 0 && u0 < u1) {
                    if (u0 < ru.whole_lo()) ru.store_end(g, 0, grad_unit<T, ENT, BIG>(ru.load_any(0), r.c));
                    if (u1 > ru.whole_hi() && ru.NU - 1 >= ru.whole_lo()) ru.store_end(g, ru.NU - 1, grad_unit<T, ENT, BIG>(ru.load_any(ru.NU - 1), r.c));
                }
                for (int base = u0; base < u1; base += NT * UPT) {
#pragma unroll
                    for (int k = 0; k < UPT; ++k) {
                        const int u = base + k * NT + (int)threadIdx.x;
                        if (u >= lo && u < hi) __stcs(ru.frame(g) + u, grad_unit<T, ENT, BIG>(HOLD ? w[k] : ru.load_any(u), r.c));
                    }
                    if (HOLD) break;
                }
            };
            if (r.big) write(std::true_type{});
            else write(std::false_type{});
            const int ux = ru.unit_of(x);
            grad_token_by<T, ENT, NT>(g, x, ux, u0, u1, lo, hi, zx, st.M, c1, r);
        }
    }
    if (rank == 0 && threadIdx.x == 0) row_report(p, row, in, st);
}

// ---- preference loss -----------------------------------------------------------------------

template <int NT>
__device__ __forceinline__ double block_sum_f64(double v, double* s) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_sum_f64(v);
    __syncthreads();
    if (lane == 0) s[warp] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int k = 0; k < NT / 32; ++k) t += s[k];
    return t;
}

// Sum of n terms in a fixed order.
constexpr int kTotThreads = 512;
__global__ void __launch_bounds__(kTotThreads) total_kernel(const float* terms, int n, float* out) {
    __shared__ double s[kTotThreads / 32];
    pdl_wait();
    pdl_trigger();
    double v = 0.0;
    for (int k = threadIdx.x; k < n; k += kTotThreads) v += (double)__ldcg(terms + k);
    v = block_sum_f64<kTotThreads>(v, s);
    if (threadIdx.x == 0) *out = (float)v;
}

// Pairs: log-probs of the two sequences, the loss, and dL/dl of their rows; either sequence has half of a CTA's threads.  total: the
// launch is one cluster (of at most kPairSum pairs), which adds the losses up in the pairs' order; else a CTA a pair.
constexpr int kPairThreads = 512, kPairHalf = kPairThreads / 2, kPairSum = 64;
__global__ void __launch_bounds__(kPairThreads) pref_pair_kernel(const __grid_constant__ PrefParams p, int total) {
    __shared__ double s[2][kPairThreads / 32];
    __shared__ float losses[kPairSum];
    const int P = p.n_pairs, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k = threadIdx.x >= kPairHalf ? 1 : 0, t0 = (int)threadIdx.x - k * kPairHalf;      // 1: the rejected sequence
    cg::cluster_group cluster = cg::this_cluster();
    if (total) cluster.barrier_arrive();            // (CTA 0 has started before anyone stores a loss into it)
    pdl_wait();
    pdl_trigger();
    if (total) cluster.barrier_wait();
    const double iT = 1.0 / (double)p.temperature;
    for (int i = blockIdx.x; i < P; i += (int)gridDim.x) {
        const int q = i + k * P;
        const int first = min(max(__ldcg(p.seq_start + q), 0), p.n_rows), end = min(max(__ldcg(p.seq_start + q + 1), first), p.n_rows);
        double t = 0.0, n = 0.0;
        for (int r = first + t0; r < end; r += kPairHalf) {
            const float4 e = __ldcg(reinterpret_cast<const float4*>(p.pref + r));
            if (__float_as_int(e.w) == 1) {
                t += (double)e.z * iT - log((double)e.y);
                n += 1.0;
            }
        }
        t = warp_sum_f64(t);
        n = warp_sum_f64(n);
        __syncthreads();                                     // (the pair before has been read)
        if (lane == 0) {
            s[0][warp] = t;
            s[1][warp] = n;
        }
        __syncthreads();
        double l[2] = {0.0, 0.0}, count[2] = {0.0, 0.0};
#pragma unroll
        for (int w = 0; w < kPairThreads / 32; ++w) {
            l[w / (kPairHalf / 32)] += s[0][w];
            count[w / (kPairHalf / 32)] += s[1][w];
        }
        if (p.average) {
            if (count[0] > 0.0) l[0] /= count[0];
            if (count[1] > 0.0) l[1] /= count[1];
        }
        const double w = (double)p.scale * (p.pair_weight ? (double)__ldcg(p.pair_weight + i) : 1.0);
        const double D = p.ref_logp ? (l[0] - (double)__ldcg(p.ref_logp + i)) - (l[1] - (double)__ldcg(p.ref_logp + P + i)) : l[0] - l[1];
        const double beta = (double)p.beta, margin = (double)p.margin;
        double loss, dD;
        if (p.rule == ADASD_PREF_SIGMOID) {
            // -(1 - s) ln sigma(u) - s ln sigma(-u) = ln(1 + e^-|u|) + (1 - s) max(-u, 0) + s max(u, 0), for infinite u too
            const double u = beta * D - margin, ls = (double)p.label_smoothing, e = exp(-fabs(u));
            loss = log1p(e) + (u < 0.0 ? (ls - 1.0) * u : ls != 0.0 || u != u ? ls * u : 0.0);
            dD = beta * (ls - (u >= 0.0 ? e / (1.0 + e) : 1.0 / (1.0 + e)));
        } else if (p.rule == ADASD_PREF_SQUARED) {
            const double u = D - margin - 0.5 / beta;
            loss = u * u;
            dD = 2.0 * u;
        } else {
            const double u = 1.0 - (beta * D - margin);
            loss = u > 0.0 ? u : u == u ? 0.0 : u;
            dD = u > 0.0 ? -beta : u == u ? 0.0 : u;
        }
        const bool off = w == 0.0;
        const float term = off ? 0.f : (float)(w * loss);
        if (threadIdx.x == 0) {
            p.seq_logp[i] = (float)l[0];
            p.seq_logp[i + P] = (float)l[1];
            p.pair_loss[i] = term;
            if (total) *cluster.map_shared_rank(losses + i, 0) = term;
        }
        if (p.grad) {
            double d = off ? 0.0 : (k ? -w : w) * dD;
            if (p.average && count[k] > 0.0) d /= count[k];
            const float df = (float)d;
            for (int r = first + t0; r < end; r += kPairHalf) p.pref[r].dz = df;
        }
    }
    if (total) {
        cluster.sync();
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            double v = 0.0;
            for (int i = 0; i < P; ++i) v += (double)losses[i];
            *p.loss = (float)v;
        }
    }
}

// Gradient of rows whose statistics and dL/dl are known: dL/dz_v = dL/dl (1[v = x] - p_v) / T.  From the last row to the
// first: what the L2 still holds of score_kernel's reads is read first.
constexpr int kPgThreads = 256, kPgUnits = 8;
template <typename T, int L>
__global__ void __launch_bounds__(kPgThreads) pref_grad_kernel(const __grid_constant__ PrefParams p) {
    constexpr bool WHOLE = L == ROWS_WHOLE;
    const int back = (int)(blockIdx.x / (unsigned)p.segs), seg = (int)(blockIdx.x - (unsigned)back * (unsigned)p.segs);
    const int row = p.n_rows - 1 - back;
    pdl_wait();
    pdl_trigger();
    const float4 e = __ldcg(reinterpret_cast<const float4*>(p.pref + row));
    const int kind = __float_as_int(e.w);
    if (kind < 0) return;
    const T* const z = reinterpret_cast<const T*>(p.z) + (long long)row * p.row_stride;
    T* const g = reinterpret_cast<T*>(p.grad) + (long long)row * p.g_stride;
    const RowUnits<T, L> ru(z, g, p.V);
    const int u0 = min(seg * p.per_cta, ru.NU), u1 = min(u0 + p.per_cta, ru.NU);
    if (u0 >= u1) return;                           // (of rows of 2048 segments and more, the last may be empty)
    if (kind == 0 || e.z == 0.f) {
        ru.store_zeros(g, u0, u1, (int)threadIdx.x, kPgThreads);
        return;
    }
    const int x = __ldcg(p.tok + row), ux = ru.unit_of(x);
    uint4 w[kPgUnits], first, last;
#pragma unroll
    for (int k = 0; k < kPgUnits; ++k) w[k] = ru.load_any(min(u0 + k * kPgThreads + (int)threadIdx.x, u1 - 1));
    const int lo = max(u0, ru.whole_lo()), hi = min(u1, ru.whole_hi());
    const bool has_first = !WHOLE && u0 < ru.whole_lo(), has_last = !WHOLE && u1 > ru.whole_hi() && ru.NU - 1 >= ru.whole_lo();
    if (has_first) first = ru.load_any(0);
    if (has_last) last = ru.load_any(ru.NU - 1);
    float zx = 0.f;
    if (ux >= u0 && ux < u1) zx = to_f32(z[x]);      // (of its CTA alone: another may have written its gradient there)
    __syncthreads();
    RowGrad r;
    const RowStats st{e.x, e.y, 0.f, zx};
    r.top = e.z / p.temperature;
    grad_consts(r, st, p.c1, pair2(p.c1), 0.f, -r.top);
    auto write = [&](auto big) {
        constexpr bool BIG = decltype(big)::value;
#pragma unroll
        for (int k = 0; k < kPgUnits; ++k) {
            const int u = u0 + k * kPgThreads + (int)threadIdx.x;
            if (u >= lo && u < hi) __stcs(ru.frame(g) + u, grad_unit<T, false, BIG>(w[k], r.c));
        }
        if (threadIdx.x < 32) {
            if (has_first) ru.store_end(g, 0, grad_unit<T, false, BIG>(first, r.c));
            if (has_last) ru.store_end(g, ru.NU - 1, grad_unit<T, false, BIG>(last, r.c));
        }
    };
    if (r.big) write(std::true_type{});
    else write(std::false_type{});
    grad_token_by<T, false, kPgThreads>(g, x, ux, u0, u1, lo, hi, zx, e.x, p.c1, r);
}

}  // namespace adasd
