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

namespace adasd {

constexpr float kAdAvgMax = 448.f, kAdSqMax = 57344.f;       // largest e4m3, e5m2
constexpr float kAdLeast = 7.888609052210118e-31f;          // 2^-100: a block with nothing larger is held as zeros (the quotient below stays finite)

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
__device__ __forceinline__ float ad_sqrt(float x) {          // 2^-23 of itself: the step's size is lr, far below p
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ad_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// |y| moved down to a value of a small float, once `bits` / 2^DROP of a step have been added: of DROP bits fewer than fp32 where it is normal, in
// steps of `least` below.  In the mean over the bits this is y itself.
template <int DROP>
__device__ __forceinline__ float ad_to_grid(float y, uint32_t bits, float least) {
    const float a = fabsf(y), per = 1.f / least;             // (least is a power of two)
    const float big = __uint_as_float((__float_as_uint(a) + bits) & ~((1u << DROP) - 1u));
    const float small = floorf(__fadd_rn(__fmul_rn(a, per), __fmul_rn((float)bits, 1.f / (float)(1u << DROP)))) * least;
    return copysignf(a < least * (float)(1 << (23 - DROP)) ? small : big, y);
}

// ---- eight elements of a lane ------------------------------------------------------------------
// WHOLE: the block has 256 elements and its arrays start at 16 bytes (8-bit codes: 8): lane l holds elements 8 l .. 8 l + 7.  Else elements
// l + 32 j, one by one, those at or beyond n as zeros.
template <bool WHOLE, typename T>
__device__ __forceinline__ void ad_load(const T* a, int lane, int n, float (&x)[8]) {
    if constexpr (WHOLE && sizeof(T) == 4) {
        const float4 u = __ldcg(reinterpret_cast<const float4*>(a) + 2 * lane), w = __ldcg(reinterpret_cast<const float4*>(a) + 2 * lane + 1);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
        x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    } else if constexpr (WHOLE) {
        unpack16(__ldcg(reinterpret_cast<const uint4*>(a) + lane), x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = lane + 32 * j < n ? to_f32(a[lane + 32 * j]) : 0.f;
    }
}
__device__ __forceinline__ uint32_t ad_pack2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void ad_store(T* a, int lane, int n, const float (&x)[8]) {
    if constexpr (WHOLE && sizeof(T) == 4) {
        reinterpret_cast<float4*>(a)[2 * lane] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(a)[2 * lane + 1] = make_float4(x[4], x[5], x[6], x[7]);
    } else if constexpr (WHOLE) {
        reinterpret_cast<uint4*>(a)[lane] = make_uint4(ad_pack2(x[0], x[1]), ad_pack2(x[2], x[3]), ad_pack2(x[4], x[5]), ad_pack2(x[6], x[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (lane + 32 * j < n) {
                if constexpr (sizeof(T) == 4) a[lane + 32 * j] = x[j];
                else a[lane + 32 * j] = __float2bfloat16_rn(x[j]);
            }
    }
}
// Codes: E5M2 false: e4m3, true: e5m2.
template <bool E5M2>
__device__ __forceinline__ float2 ad_decode2(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, E5M2 ? __NV_E5M2 : __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
template <bool E5M2>
__device__ __forceinline__ uint32_t ad_encode2(float a, float b) {
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
}
template <bool WHOLE, bool E5M2>
__device__ __forceinline__ void ad_load_codes(const uint8_t* a, int lane, int n, float (&x)[8]) {
    uint32_t c[4];
    if constexpr (WHOLE) {
        const uint2 w = __ldcg(reinterpret_cast<const uint2*>(a) + lane);
        c[0] = w.x & 0xFFFFu; c[1] = w.x >> 16; c[2] = w.y & 0xFFFFu; c[3] = w.y >> 16;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c[j] = (lane + 64 * j < n ? (uint32_t)a[lane + 64 * j] : 0u) | (lane + 64 * j + 32 < n ? (uint32_t)a[lane + 64 * j + 32] << 8 : 0u);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = ad_decode2<E5M2>(c[j]);
        x[2 * j] = f.x;
        x[2 * j + 1] = f.y;
    }
}
template <bool WHOLE>
__device__ __forceinline__ void ad_store_codes(uint8_t* a, int lane, int n, const uint32_t (&c)[4]) {
    if constexpr (WHOLE) {
        reinterpret_cast<uint2*>(a)[lane] = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (lane + 64 * j < n) a[lane + 64 * j] = (uint8_t)c[j];
            if (lane + 64 * j + 32 < n) a[lane + 64 * j + 32] = (uint8_t)(c[j] >> 8);
        }
    }
}

// ---- a block ---------------------------------------------------------------------------------
// Products and sums of the states are rounded one by one (no multiply-add), so that what is held in 8 bits does not hang on how the compiler joins
// them: a state that another program works out by the formula gets the same codes.
template <typename P, typename G, bool EIGHT, bool WHOLE>
struct AdBlock {
    float p[8], g[8], m[8], v[8], sm, sv;

    __device__ __forceinline__ void load(const AdTensor& t, long long first, int lane, int n) {
        ad_load<WHOLE>(static_cast<const P*>(t.param) + first, lane, n, p);
        ad_load<WHOLE>(static_cast<const G*>(t.grad) + first, lane, n, g);
        if constexpr (EIGHT) {
            ad_load_codes<WHOLE, false>(static_cast<const uint8_t*>(t.exp_avg) + first, lane, n, m);
            ad_load_codes<WHOLE, true>(static_cast<const uint8_t*>(t.exp_avg_sq) + first, lane, n, v);
            sm = __ldcg(t.avg_scale + first / kAdBlock);
            sv = __ldcg(t.sq_scale + first / kAdBlock);
        } else {
            ad_load<WHOLE>(static_cast<const float*>(t.exp_avg) + first, lane, n, m);
            ad_load<WHOLE>(static_cast<const float*>(t.exp_avg_sq) + first, lane, n, v);
        }
    }
    __device__ __forceinline__ void step(const AdParams& a, const AdCoef& c, float keep, const AdTensor& t, uint32_t key, long long first, int lane, int n) {
        float m_top = 0.f, v_top = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float gj = __fmul_rn(g[j], c.grad_scale);
            if constexpr (EIGHT) {
                m[j] = __fmul_rn(m[j], sm);
                v[j] = __fmul_rn(v[j], sv);
            }
            m[j] = __fadd_rn(__fmul_rn(m[j], a.b1), __fmul_rn(gj, a.b1c));
            v[j] = __fadd_rn(__fmul_rn(v[j], a.b2), __fmul_rn(__fmul_rn(gj, gj), a.b2c));
            const float denom = fmaf(ad_sqrt(v[j]), c.root, a.eps);
            p[j] = fmaf(-c.rate, m[j] * ad_rcp(denom), p[j] * keep);
            if constexpr (EIGHT) {
                m_top = ad_max(m_top, fabsf(m[j]));
                v_top = ad_max(v_top, v[j]);
            }
        }
        uint32_t h[8];
        if (a.stochastic && (EIGHT || sizeof(P) == 2)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = ad_mix((uint32_t)first + (WHOLE ? 8 * lane + j : lane + 32 * j) + key);
            if constexpr (sizeof(P) == 2) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {                // (infinities and NaN as they are)
                    const uint32_t b = __float_as_uint(p[j]);
                    if ((b & 0x7F800000u) != 0x7F800000u) p[j] = __uint_as_float((b + ((h[j] * 0x9E3779B1u) >> 16)) & 0xFFFF0000u);
                }
            }
        }
        ad_store<WHOLE>(static_cast<P*>(t.param) + first, lane, n, p);
        if constexpr (sizeof(P) == 4)
            if (t.param_copy) ad_store<WHOLE>(static_cast<__nv_bfloat16*>(t.param_copy) + first, lane, n, p);
        if constexpr (!EIGHT) {
            ad_store<WHOLE>(static_cast<float*>(t.exp_avg) + first, lane, n, m);
            ad_store<WHOLE>(static_cast<float*>(t.exp_avg_sq) + first, lane, n, v);
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
            uint32_t cm[4], cv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float y[2], q[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    y[k] = __fmul_rn(m[2 * j + k], im);
                    q[k] = __fmul_rn(v[2 * j + k], iv);
                    if (a.stochastic) {
                        y[k] = ad_to_grid<20>(y[k], h[2 * j + k] & 0xFFFFFu, 0x1p-9f);
                        q[k] = ad_to_grid<21>(q[k], h[2 * j + k] >> 11, 0x1p-16f);
                    }
                }
                cm[j] = ad_encode2<false>(y[0], y[1]);
                cv[j] = ad_encode2<true>(q[0], q[1]);
                // a v above 0 is never held as 0: m might be kept where it is not, and m / eps is no step
                if (v[2 * j] > 0.f && (cv[j] & 0xFFu) == 0u) cv[j] |= 1u;
                if (v[2 * j + 1] > 0.f && (cv[j] >> 8) == 0u) cv[j] |= 0x100u;
            }
            ad_store_codes<WHOLE>(static_cast<uint8_t*>(t.exp_avg) + first, lane, n, cm);
            ad_store_codes<WHOLE>(static_cast<uint8_t*>(t.exp_avg_sq) + first, lane, n, cv);
        }
    }
};

// A warp's block of an item.
template <typename P, typename G, bool EIGHT>
__device__ __forceinline__ void ad_blocks(const AdParams& a, const AdCoef& c, float keep, const AdTensor& t, uint32_t key, long long first, int lane) {
    const long long left = t.n - first;
    if (left <= 0) return;
    if (t.aligned && left >= kAdBlock) {
        AdBlock<P, G, EIGHT, true> b;
        b.load(t, first, lane, kAdBlock);
        b.step(a, c, keep, t, key, first, lane, kAdBlock);
    } else {
        const int n = (int)min(left, (long long)kAdBlock);
        AdBlock<P, G, EIGHT, false> b;
        b.load(t, first, lane, n);
        b.step(a, c, keep, t, key, first, lane, n);
    }
}

template <int TABLE>
__global__ void __launch_bounds__(kAdThreads) adamw_kernel(const __grid_constant__ AdParams a, const __grid_constant__ AdTable<TABLE> table) {
    __shared__ AdCoef s_coef;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    pdl_trigger();
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
    for (int item = blockIdx.x; item < table.items; item += gridDim.x) {
        int lo = 0, hi = table.n - 1;                        // the last tensor that starts at or before the item
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (table.t[mid].first_item <= item) lo = mid;
            else hi = mid - 1;
        }
        const AdTensor& t = table.t[lo];
        const long long first = (long long)(item - t.first_item) * kAdItem + warp * kAdBlock;
        const float keep = fmaf(-c.lr, t.weight_decay, 1.f);
        const uint32_t key = ad_mix(a.seed ^ ad_mix(c.step + 0x9E3779B9u * (uint32_t)(t.index + 1)));
        switch (t.kind) {
            case 0: ad_blocks<__nv_bfloat16, __nv_bfloat16, false>(a, c, keep, t, key, first, lane); break;
            case 1: ad_blocks<float, __nv_bfloat16, false>(a, c, keep, t, key, first, lane); break;
            case 2: ad_blocks<__nv_bfloat16, float, false>(a, c, keep, t, key, first, lane); break;
            case 3: ad_blocks<float, float, false>(a, c, keep, t, key, first, lane); break;
            case 4: ad_blocks<__nv_bfloat16, __nv_bfloat16, true>(a, c, keep, t, key, first, lane); break;
            case 5: ad_blocks<float, __nv_bfloat16, true>(a, c, keep, t, key, first, lane); break;
            case 6: ad_blocks<__nv_bfloat16, float, true>(a, c, keep, t, key, first, lane); break;
            default: ad_blocks<float, float, true>(a, c, keep, t, key, first, lane); break;
        }
    }
}

}  // namespace adasd
