// One AdamW step over many tensors.
//
//   m' = b1 m + (1 - b1) g        v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// Every element is read and written once: the step is bound by memory.  A warp takes a block of 256 consecutive elements of a
// tensor, eight a lane (one or two 16-byte loads of each array); a block is also what shares a scale where states are held in 8
// bits, so that its largest |m| and v are found by shuffles and nothing but the block itself is looked at.
#pragma once

#include "adasd_adamw_types.cuh"
#include "adasd_device.cuh"
#include "adasd_pdl.cuh"

#include <cuda_fp8.h>

#include <type_traits>

namespace adasd {

constexpr float kAdAvgMax = 448.f, kAdSqMax = 57344.f;       // largest e4m3, e5m2
constexpr float kAdLeast = 7.888609052210118e-31f;          // 2^-100: a block with nothing larger is held as zeros (the quotient below stays finite)

// The published mixer of 32-bit integers known as lowbias32 (shifts and factors found by search): every bit in changes every bit out about half of the time.
__device__ __forceinline__ uint32_t ad_mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}
__device__ __forceinline__ float ad_max(float a, float b) {  // NaN kept
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// Square root and reciprocal are 2^-23 of themselves off: they make the step, whose size is lr, far below p.  (Both flush: eps is 1e-16 at the least.)
__device__ __forceinline__ float ad_sqrt(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ad_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 ad_two(float x) { return make_float2(x, x); }
// Products that are rounded by themselves, whatever they are added to: as single numbers (products and sums of pairs get joined to multiply-adds).
__device__ __forceinline__ float2 ad_mul(float2 a, float b) { return make_float2(__fmul_rn(a.x, b), __fmul_rn(a.y, b)); }

// y moved towards 0 to a value of a small float, once DROP bits of `bits` / 2^DROP of a step have been added to its size: of DROP bits fewer than fp32 where it
// is normal, in steps of 1 / PER below.  In the mean over the bits this is y itself.  (The bits become a fraction as the mantissa of a number in [1, 2); the floor is
// an addition of 2^23, rounded down: conversions would wait for the special-function unit, which roots and reciprocals need.)
template <int DROP, int PER, bool SIGNED>
__device__ __forceinline__ float2 ad_to_grid(float2 y, uint32_t bits0, uint32_t bits1) {
    constexpr uint32_t kMask = (1u << DROP) - 1u;
    constexpr float kNormal = (float)(1 << (23 - DROP)) / (float)PER;
    const float2 r = __fadd2_rn(make_float2(__uint_as_float(0x3F800000u | (bits0 << (23 - DROP) & kMask << (23 - DROP))),
                                            __uint_as_float(0x3F800000u | (bits1 << (23 - DROP) & kMask << (23 - DROP)))),
                                ad_two(-1.f));
    const float2 t = SIGNED ? make_float2(fmaf(fabsf(y.x), (float)PER, r.x), fmaf(fabsf(y.y), (float)PER, r.y)) : __ffma2_rn(y, ad_two((float)PER), r);
    float2 f = __fmul2_rn(__fadd2_rn(make_float2(__fadd_rd(t.x, 8388608.f), __fadd_rd(t.y, 8388608.f)), ad_two(-8388608.f)), ad_two(1.f / (float)PER));
    if (SIGNED) f = make_float2(copysignf(f.x, y.x), copysignf(f.y, y.y));
    return make_float2(fabsf(y.x) < kNormal ? f.x : __uint_as_float((__float_as_uint(y.x) + (bits0 & kMask)) & ~kMask),
                       fabsf(y.y) < kNormal ? f.y : __uint_as_float((__float_as_uint(y.y) + (bits1 & kMask)) & ~kMask));
}
// q, or 2^-16 if that is more and v is above 0
__device__ __forceinline__ float ad_some(float q, float v) {
    asm("{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %1, 0f00000000;\n\t@p max.NaN.f32 %0, %0, 0f37800000;\n\t}" : "+f"(q) : "f"(v));
    return q;
}

// ---- eight elements of a lane ------------------------------------------------------------------
// WHOLE: the block has 256 elements and its arrays start at 16 bytes (8-bit codes: 8): lane l holds elements 8 l .. 8 l + 7.  Else elements
// l + 32 j, one by one, those at or beyond n as zeros: a tensor with any array off these boundaries goes this way (100M elements: bf16 with 8-bit states 386 us instead of
// 259, with states in 32 bits 393 instead of 337; fp32 431 instead of 421).  What is loaded is kept as it lies until it is needed, so that the next block's can be on
// its way.
template <bool WHOLE, typename T>
struct AdNumbers {                       // of T float or bf16
    uint4 w[sizeof(T) == 4 || !WHOLE ? 2 : 1];
    __device__ __forceinline__ void load(const void* p, long long first, int lane, int n) {
        const T* a = static_cast<const T*>(p) + first;
        if constexpr (WHOLE) {
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) w[k] = __ldcg(reinterpret_cast<const uint4*>(a) + (int)sizeof(T) / 2 * lane + k);
        } else {
            uint32_t* u = &w[0].x;
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = lane + 32 * j < n ? __float_as_uint(to_f32(a[lane + 32 * j])) : 0u;
        }
    }
    __device__ __forceinline__ void get(float2 (&x)[4]) const {
        const uint32_t* u = &w[0].x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (WHOLE && sizeof(T) == 2) x[j] = make_float2(__uint_as_float(u[j] << 16), __uint_as_float(u[j] & 0xFFFF0000u));
            else x[j] = make_float2(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1]));
        }
    }
};
__device__ __forceinline__ uint32_t ad_pack2(float2 v) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(v.y), "f"(v.x));
    return d;
}
// Of numbers whose lower 16 bits are to be dropped.
template <bool WHOLE>
__device__ __forceinline__ void ad_store_high(void* p, long long first, int lane, int n, const uint32_t (&x)[8]) {
    uint16_t* a = static_cast<uint16_t*>(p) + first;
    if constexpr (WHOLE) {
        reinterpret_cast<uint4*>(a)[lane] = make_uint4(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632), __byte_perm(x[4], x[5], 0x7632),
                                                       __byte_perm(x[6], x[7], 0x7632));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (lane + 32 * j < n) a[lane + 32 * j] = (uint16_t)(x[j] >> 16);
    }
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void ad_store(void* p, long long first, int lane, int n, const float2 (&x)[4]) {
    T* a = static_cast<T*>(p) + first;
    if constexpr (WHOLE && sizeof(T) == 4) {
        reinterpret_cast<float4*>(a)[2 * lane] = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
        reinterpret_cast<float4*>(a)[2 * lane + 1] = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
    } else if constexpr (WHOLE) {
        reinterpret_cast<uint4*>(a)[lane] = make_uint4(ad_pack2(x[0]), ad_pack2(x[1]), ad_pack2(x[2]), ad_pack2(x[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (lane + 32 * j < n) {
                const float v = j & 1 ? x[j / 2].y : x[j / 2].x;
                if constexpr (sizeof(T) == 4) a[lane + 32 * j] = v;
                else a[lane + 32 * j] = __float2bfloat16_rn(v);
            }
    }
}
// Codes.  E5M2 false: e4m3, true: e5m2.
template <bool WHOLE, bool E5M2>
struct AdCodes {
    uint2 w;
    __device__ __forceinline__ void load(const void* p, long long first, int lane, int n) {
        const uint8_t* a = static_cast<const uint8_t*>(p) + first;
        if constexpr (WHOLE) {
            w = __ldcg(reinterpret_cast<const uint2*>(a) + lane);
        } else {
            uint32_t u[2] = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (lane + 32 * j < n) u[j / 4] |= (uint32_t)a[lane + 32 * j] << (8 * (j & 3));
            w = make_uint2(u[0], u[1]);
        }
    }
    __device__ __forceinline__ void get(float2 (&x)[4]) const {
        const uint32_t u[2] = {w.x, w.y};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_fp8x2_storage_t two = (__nv_fp8x2_storage_t)(u[j / 2] >> (16 * (j & 1)));
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, E5M2 ? __NV_E5M2 : __NV_E4M3);
            x[j] = __half22float2(*reinterpret_cast<const __half2*>(&h));
        }
    }
    static __device__ __forceinline__ void put(void* p, long long first, int lane, int n, const float2 (&x)[4]) {
        uint8_t* a = static_cast<uint8_t*>(p) + first;
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = __nv_cvt_float2_to_fp8x2(x[j], __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
        if constexpr (WHOLE) {
            reinterpret_cast<uint2*>(a)[lane] = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (lane + 32 * j < n) a[lane + 32 * j] = (uint8_t)(c[j / 2] >> (8 * (j & 1)));
        }
    }
};

// ---- a block ---------------------------------------------------------------------------------
// Products and sums of the states are rounded one by one (no multiply-add), so that what is held in 8 bits does not hang on how the compiler joins
// them: a state that another program works out by the formula gets the same codes.
template <typename P, typename G, bool EIGHT, bool WHOLE>
struct AdBlock {
    AdNumbers<WHOLE, P> p;
    AdNumbers<WHOLE, G> g;
    std::conditional_t<EIGHT, AdCodes<WHOLE, false>, AdNumbers<WHOLE, float>> m;
    std::conditional_t<EIGHT, AdCodes<WHOLE, true>, AdNumbers<WHOLE, float>> v;
    float sm, sv;

    __device__ __forceinline__ void load(const AdTensor& t, long long first, int lane, int n) {
        p.load(t.param, first, lane, n);
        g.load(t.grad, first, lane, n);
        m.load(t.exp_avg, first, lane, n);
        v.load(t.exp_avg_sq, first, lane, n);
        if constexpr (EIGHT) {
            sm = __ldcg(t.avg_scale + first / kAdBlock);
            sv = __ldcg(t.sq_scale + first / kAdBlock);
        }
    }
    __device__ __forceinline__ void step(const AdParams& a, const AdCoef& c, float keep, const AdTensor& t, uint32_t key, long long first, int lane, int n) const {
        float2 x[4], y[4], q[4], d[4];
        m.get(y);
        v.get(q);
        g.get(d);
        p.get(x);
        float m_top = 0.f, v_top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 gj = __fmul2_rn(d[j], ad_two(c.grad_scale));
            if constexpr (EIGHT) {
                y[j] = __fmul2_rn(y[j], ad_two(sm));
                q[j] = __fmul2_rn(q[j], ad_two(sv));
            }
            y[j] = __fadd2_rn(ad_mul(y[j], a.b1), ad_mul(gj, a.b1c));
            q[j] = __fadd2_rn(ad_mul(q[j], a.b2), ad_mul(__fmul2_rn(gj, gj), a.b2c));
            const float2 denom = __ffma2_rn(make_float2(ad_sqrt(q[j].x), ad_sqrt(q[j].y)), ad_two(c.root), ad_two(a.eps));
            x[j] = __ffma2_rn(__fmul2_rn(y[j], make_float2(ad_rcp(denom.x), ad_rcp(denom.y))), ad_two(-c.rate), __fmul2_rn(x[j], ad_two(keep)));
            if constexpr (EIGHT) {
                m_top = ad_max(ad_max(m_top, fabsf(y[j].x)), fabsf(y[j].y));
                v_top = ad_max(ad_max(v_top, q[j].x), q[j].y);
            }
        }
        uint32_t h[8];
        if (a.stochastic && (EIGHT || sizeof(P) == 2)) {
            const uint32_t at = (uint32_t)first + key + (WHOLE ? 8 * lane : lane);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = ad_mix(at + (WHOLE ? j : 32 * j));
        }
        if (sizeof(P) == 2 && a.stochastic) {                // up or down by 16 bits of noise; a NaN, whose bits are all ones here, stays one
            uint32_t u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t b = __float_as_uint(j & 1 ? x[j / 2].y : x[j / 2].x);
                u[j] = min(b + ((h[j] * 0x9E3779B1u) >> 16), b | 0x7FFFFFFFu);
            }
            ad_store_high<WHOLE>(t.param, first, lane, n, u);
        } else {
            ad_store<WHOLE, P>(t.param, first, lane, n, x);
        }
        if constexpr (sizeof(P) == 4)
            if (t.param_copy) ad_store<WHOLE, __nv_bfloat16>(t.param_copy, first, lane, n, x);
        if constexpr (!EIGHT) {
            ad_store<WHOLE, float>(t.exp_avg, first, lane, n, y);
            ad_store<WHOLE, float>(t.exp_avg_sq, first, lane, n, q);
        } else {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                m_top = ad_max(m_top, __shfl_xor_sync(0xFFFFFFFFu, m_top, o));
                v_top = ad_max(v_top, __shfl_xor_sync(0xFFFFFFFFu, v_top, o));
            }
            if (lane == 0) {
                t.avg_scale[first / kAdBlock] = __fmul_rn(m_top, 1.f / kAdAvgMax);
                t.sq_scale[first / kAdBlock] = __fmul_rn(v_top, 1.f / kAdSqMax);
            }
            const float im = m_top >= kAdLeast ? __fdiv_rn(kAdAvgMax, m_top) : 0.f, iv = v_top >= kAdLeast ? __fdiv_rn(kAdSqMax, v_top) : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // a v above 0 is never held as 0: m might be kept where it is not, and m / eps is no step
                const float2 v0 = q[j];
                y[j] = __fmul2_rn(y[j], ad_two(im));
                q[j] = __fmul2_rn(q[j], ad_two(iv));
                if (a.stochastic) {
                    y[j] = ad_to_grid<20, 512, true>(y[j], h[2 * j], h[2 * j + 1]);
                    q[j] = ad_to_grid<21, 65536, false>(q[j], h[2 * j] >> 11, h[2 * j + 1] >> 11);
                }
                q[j] = make_float2(ad_some(q[j].x, v0.x), ad_some(q[j].y, v0.y));
            }
            AdCodes<WHOLE, false>::put(t.exp_avg, first, lane, n, y);
            AdCodes<WHOLE, true>::put(t.exp_avg_sq, first, lane, n, q);
        }
    }
};

// A warp's blocks of an item, one for each round of its CTA: the next one's loads are under way while one is worked on.
template <typename P, typename G, bool EIGHT>
__device__ __forceinline__ void ad_blocks(const AdParams& a, const AdCoef& c, float keep, const AdTensor& t, uint32_t key, long long first, int rounds, int lane) {
    long long left = t.n - first;
    if (t.aligned && left >= kAdBlock) {
        AdBlock<P, G, EIGHT, true> b;
        b.load(t, first, lane, kAdBlock);
        for (;;) {
            --rounds;
            left -= kAdRound;
            const bool more = rounds > 0 && left >= kAdBlock;
            AdBlock<P, G, EIGHT, true> next;
            if (more) next.load(t, first + kAdRound, lane, kAdBlock);
            b.step(a, c, keep, t, key, first, lane, kAdBlock);
            first += kAdRound;
            if (!more) break;
            b = next;
        }
    }
    for (; rounds > 0 && left > 0; --rounds, first += kAdRound, left -= kAdRound) {
        const int n = (int)min(left, (long long)kAdBlock);
        AdBlock<P, G, EIGHT, false> b;
        b.load(t, first, lane, n);
        b.step(a, c, keep, t, key, first, lane, n);
    }
}

template <bool EIGHT, typename Table>
__device__ __forceinline__ void adamw_items(const AdParams& a, const Table& table) {
    __shared__ AdCoef s_coef;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    AdCoef c = a.coef;
    if (a.lr_dev || a.step_dev || a.grad_scale_dev) {
        if (threadIdx.x == 0) {
            const double lr = a.lr_dev ? (double)__ldcg(a.lr_dev) : a.lr;
            const double step = a.step_dev ? (double)max(__ldcg(a.step_dev), 1) : (double)a.step;
            s_coef.step = (uint32_t)step;
            s_coef.lr = (float)lr;
            s_coef.rate = (float)(lr / -expm1(step * a.log_b1));
            s_coef.root = (float)rsqrt(-expm1(step * a.log_b2));
            s_coef.grad_scale = a.grad_scale_dev ? __fmul_rn(__ldcg(a.grad_scale_dev), a.coef.grad_scale) : a.coef.grad_scale;
        }
        __syncthreads();
        c = s_coef;
        if (!isfinite(c.grad_scale)) {                       // (a norm that was not finite: nothing changes)
            if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, ADASD_STATUS_NAN);
            return;
        }
    }
    const int item = blockIdx.x;
    int lo = 0, hi = table.n - 1;                            // the last tensor that starts at or before the item
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table.t[mid].first_item <= item) lo = mid;
        else hi = mid - 1;
    }
    const AdTensor& t = table.t[lo];
    const long long first = (long long)(item - t.first_item) * table.rounds * kAdRound + warp * kAdBlock;
    const float keep = fmaf(-c.lr, t.weight_decay, 1.f);
    const uint32_t key = ad_mix(a.seed ^ ad_mix(c.step + 0x9E3779B9u * (uint32_t)(t.index + 1)));
    switch (t.kind) {
        case 0: ad_blocks<__nv_bfloat16, __nv_bfloat16, EIGHT>(a, c, keep, t, key, first, table.rounds, lane); break;
        case 1: ad_blocks<float, __nv_bfloat16, EIGHT>(a, c, keep, t, key, first, table.rounds, lane); break;
        case 2: ad_blocks<__nv_bfloat16, float, EIGHT>(a, c, keep, t, key, first, table.rounds, lane); break;
        default: ad_blocks<float, float, EIGHT>(a, c, keep, t, key, first, table.rounds, lane); break;
    }
}

template <int TABLE>
__global__ void __launch_bounds__(kAdThreads) adamw_kernel(const __grid_constant__ AdParams a, const __grid_constant__ AdTable<TABLE> table) {
    pdl_wait();
    pdl_trigger();
    adamw_items<false>(a, table);
}
// States in 8 bits.  The arithmetic is the bound, 81 instructions an element, 34 of them on the integer pipe, and needs warps: with registers for 32
// of them a SM 797 us (300M bf16 elements, up or down), for 24 901, for 40 904.
template <int TABLE>
__global__ void __launch_bounds__(kAdThreads, 4) adamw8_kernel(const __grid_constant__ AdParams a, const __grid_constant__ AdTable<TABLE> table) {
    pdl_wait();
    pdl_trigger();
    adamw_items<true>(a, table);
}

}  // namespace adasd
