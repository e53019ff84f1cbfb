// One AdamW step over all tensors of a network (the fine-tuning of Algorithm 1), states in 32 or in 8 bits.
//
//   g = grad * scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w = w (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every element is read and written once, so the bytes bound it: 28 an element for fp32 weights, gradients and states, 10 for bf16 weights and
// gradients with 8-bit states.  A thread takes eight consecutive elements (16 or 32 bytes of each tensor, 8 of an 8-bit state), so that half a warp
// holds the 128 elements of a scale and finds their largest value by shuffles; the tensors of a call are numbered through in pieces of
// 2048 elements, one CTA each, and their table travels as a kernel parameter.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "crisp_internal.h"

namespace crisp {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kPer = 8;                                       // elements a thread
constexpr int kPiece = kAdamThreads * kPer;

struct AdamTensor {
    void *w;
    uint16_t *copy;
    const void *g;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    const uint32_t *mask;
    int64_t total, ldw, ldc, ldg;
    uint32_t k, wpr;
    uint32_t key, spread;    // of the hash: the tensor's, and what elements below 2^32 take (filled in for the step of the call)
    uint32_t ordinal;
    uint8_t g32;             // gradients are fp32
    uint8_t flat;            // w, g and copy are packed: element e lies at e
    uint8_t vec;             // eight elements from a multiple of eight on lie in a row and at multiples of 16 bytes
    uint8_t bytes;           // k is a multiple of 8: eight elements' mask bits are one byte
    uint8_t plain;           // flat, vec and, under a mask, bytes
};

// Powers of two as parameters of the kernel.  The 8-bit kernel is bound by the integer pipe, and a product with a number that the compiler does not
// know goes to the multiply-add pipe instead of becoming a shift.
struct Powers { uint32_t p1 = 1u << 1, p4 = 1u << 4, p5 = 1u << 5, p7 = 1u << 7, p9 = 1u << 9, p19 = 1u << 19; };

struct AdamScalars {
    float lr, beta1, one_beta1, beta2, one_beta2, eps, decay, weight_decay;
    float step_size, root_scale;                              // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float log_beta1, log_beta2;
    uint32_t seed_key;
    Powers by;
    const float *d_lr, *d_grad_scale;
    const int64_t *d_step;
};

// A bijection of 32-bit words in which every bit of the input moves every bit of the output (xorshift-multiply with the constants that Wellons'
// search published as lowbias32).
__host__ __device__ __forceinline__ uint32_t mix_rest(uint32_t h) {
    h *= 0x7FEB352Du;
    h ^= h >> 15; h *= 0x846CA68Bu;
    return h ^ (h >> 16);
}
__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) { return mix_rest(h ^ (h >> 16)); }

// Eight elements at a multiple of 16 bytes.
__device__ __forceinline__ void load8(const float *p, float (&x)[kPer]) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(float *p, const float (&x)[kPer]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void unpack8(const uint4 &a, float (&x)[kPer]) {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ uint32_t nearest2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float from_bf16(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t nearest(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

// The 8-bit forms.  A code is the top of an fp32 number whose exponent field has been brought down by 120 (127 - 7), so that small codes are
// subnormal as fp32's are: reading sqrt(v) is a shift and a product by 2^120, rounding an addition to the bits below the code.
__device__ __forceinline__ float power_of(uint32_t biased) { return __uint_as_float(biased << 23); }       // 2^(biased - 127), 0 for 0
// One power of two for both factors, 2^120 and the scale; the product of the two exponents' rest, beyond fp32's range, is `beyond` (1 for scales up to 2^7).
__device__ __forceinline__ float power_120(uint32_t biased, float *beyond) {
    const uint32_t near = min(biased, 134u);
    *beyond = power_of(127u + biased - near);
    return power_of(near + 120u);
}
__device__ __forceinline__ float root_bits(uint32_t codes, int byte, uint32_t p19) {                         // code << 19 as fp32
    return __uint_as_float(__byte_perm(codes, 0, 0x4440 | (uint32_t)byte) * p19);
}
// The top bytes of four words.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ float2 values_m(uint32_t codes, int pair) {                                       // two e4m3 codes
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> (16 * pair)), __NV_E4M3);
    return __half22float2(__half2(h));
}
// Biased exponent of the scale under which `largest` (bits of a value >= 0) is at most 448 (`fraction` 0x600000) or 496 (0x780000): its own exponent less 8,
// one more where the fraction is above that one's.
__device__ __forceinline__ uint32_t scale_of(float largest, uint32_t fraction) {
    return (uint32_t)max((int)((__float_as_uint(largest) + (0x7FFFFFu - fraction)) >> 23) - 8, 1);
}
// The larger of each half over the 16 lanes of a block.
__device__ __forceinline__ uint32_t max_of_block(uint32_t v) {
#pragma unroll
    for (int d = 8; d; d >>= 1) v = __vmaxu2(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    return v;
}
__device__ __forceinline__ float sqrt_near(float x) {          // two units of the last place, subnormal numbers too
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal_near(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Bit i of the byte in every bit of byte i of (lo, hi).
__device__ __forceinline__ uint2 bytes_of_bits(uint32_t keep) {
    return make_uint2(((keep & 15u) * 0x00204081u & 0x01010101u) * 255u, ((keep >> 4) * 0x00204081u & 0x01010101u) * 255u);
}

// Eight elements of a thread, from e0 on.  kPlain: all of the CTA's elements are the tensor's, lie packed at multiples of 16 bytes, and their mask bits in whole
// bytes; what every other piece has to ask for each element is left out (8-bit states, 4 x 4096 x 4096: MEASURE us against MEASURE).
template <bool kNarrow, bool kW32, bool kPlain>
__device__ __forceinline__ void eight(const AdamTensor &T, const AdamScalars &s, const int64_t e0) {
    const int count = kPlain ? kPer : (int)max((int64_t)0, min((int64_t)kPer, T.total - e0));
    const bool whole = kPlain || count == kPer, vec = kPlain || (T.vec && whole), flat = kPlain || T.flat, bytes = kPlain || T.bytes;

    // where the elements lie: row and column of the first one, needed for rows that are not packed and for masks
    int64_t row = 0;
    uint32_t col = 0;
    if (T.mask || !flat) {
        if (T.total <= 0xFFFFFFFFll) {
            const uint32_t r = (uint32_t)e0 / T.k;
            row = r; col = (uint32_t)e0 - r * T.k;
        } else {
            row = e0 / T.k; col = (uint32_t)(e0 - row * T.k);
        }
    }
    const auto at = [&](int64_t ld, int i) -> int64_t {       // the address of element i, for rows of pitch ld
        if (flat) return e0 + i;
        int64_t r = row;
        uint32_t c = col + i;
        while (c >= T.k) { c -= T.k; ++r; }
        return r * ld + c;
    };

    float w[kPer] = {}, g[kPer] = {}, m[kPer] = {}, v[kPer] = {};
    uint32_t keep = 0xFFu;
    uint2 mc = make_uint2(0, 0), vc = make_uint2(0, 0);
    uint32_t m_exp = 0, v_exp = 0;
    if (vec) {
        if constexpr (kW32) load8(reinterpret_cast<const float *>(T.w) + at(T.ldw, 0), w);
        else unpack8(*reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(T.w) + at(T.ldw, 0)), w);
        if (T.g32) load8(reinterpret_cast<const float *>(T.g) + at(T.ldg, 0), g);
        else unpack8(*reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(T.g) + at(T.ldg, 0)), g);
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < count) {
                if constexpr (kW32) w[i] = reinterpret_cast<const float *>(T.w)[at(T.ldw, i)];
                else w[i] = from_bf16(reinterpret_cast<const uint16_t *>(T.w)[at(T.ldw, i)]);
                if (T.g32) g[i] = reinterpret_cast<const float *>(T.g)[at(T.ldg, i)];
                else g[i] = from_bf16(reinterpret_cast<const uint16_t *>(T.g)[at(T.ldg, i)]);
            }
    }
    if constexpr (!kNarrow) {
        const float *pm = reinterpret_cast<const float *>(T.m) + e0, *pv = reinterpret_cast<const float *>(T.v) + e0;
        if (whole) {
            load8(pm, m); load8(pv, v);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) { m[i] = pm[i]; v[i] = pv[i]; }
        }
    } else {
        const uint8_t *pm = reinterpret_cast<const uint8_t *>(T.m) + e0, *pv = reinterpret_cast<const uint8_t *>(T.v) + e0;
        if (whole) {
            mc = *reinterpret_cast<const uint2 *>(pm); vc = *reinterpret_cast<const uint2 *>(pv);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) {
                    (i < 4 ? mc.x : mc.y) |= (uint32_t)pm[i] << (8 * (i & 3));
                    (i < 4 ? vc.x : vc.y) |= (uint32_t)pv[i] << (8 * (i & 3));
                }
        }
        if (count) { m_exp = T.m_exp[e0 >> 7]; v_exp = T.v_exp[e0 >> 7]; }
    }
    if (T.mask && count) {
        if (bytes) {
            keep = reinterpret_cast<const uint8_t *>(T.mask + row * T.wpr)[col >> 3];
        } else {
            int64_t r = row;
            uint32_t c = col;
            keep = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) {
                    keep |= (T.mask[r * T.wpr + (c >> 5)] >> (c & 31) & 1u) << i;
                    if (++c == T.k) { c = 0; ++r; }
                }
        }
    }

    float step_size = s.step_size, root_scale = s.root_scale, decay = s.decay;
    uint32_t key = T.key, spread = T.spread;
    if (s.d_step || s.d_lr) {
        const float lr = s.d_lr ? *s.d_lr : s.lr;
        const float t = s.d_step ? (float)*s.d_step : 0.f;
        // 1 - b^t = -expm1(t log b): to a rounding or two of fp32 for any t
        if (s.d_step) {
            root_scale = 1.f / sqrtf(-expm1f(t * s.log_beta2));
            key = mix(mix(s.seed_key ^ (uint32_t)*s.d_step) ^ T.ordinal);
            spread = mix(key);
        }
        step_size = s.d_step ? lr / -expm1f(t * s.log_beta1) : s.step_size / s.lr * lr;
        decay = 1.f - lr * s.weight_decay;
    }
    const float grad_scale = s.d_grad_scale ? *s.d_grad_scale : 1.f;
    if (kNarrow || !kW32)
        if (e0 >> 32) spread = mix((uint32_t)(e0 >> 32) ^ key);

    // Where the mask has no bit: zeros go in and zeros come out (eps is above 0).
    if (T.mask) {
        if constexpr (kNarrow) {
            const uint2 b8 = bytes_of_bits(keep);
            mc.x &= b8.x; mc.y &= b8.y; vc.x &= b8.x; vc.y &= b8.y;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (!(keep >> i & 1u)) { w[i] = 0.f; g[i] = 0.f; m[i] = 0.f; v[i] = 0.f; }
    }
    float v_beyond;
    const float m_scale = power_of(m_exp), v_scale = power_120(v_exp, &v_beyond);
    const bool wide_scale = kNarrow && v_beyond != 1.f;

    // (e0 is a multiple of 8: the hash of e0 + i differs from that of e0 in three low bits until its first product)
    const uint32_t first = ((uint32_t)e0 ^ spread) ^ (((uint32_t)e0 ^ spread) >> 16);
    uint32_t h[kPer];
    float root[kPer], bad = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if constexpr (kNarrow) {
            if ((i & 1) == 0) {
                const float2 two = values_m(i < 4 ? mc.x : mc.y, i >> 1 & 1);
                m[i] = two.x * m_scale; m[i + 1] = two.y * m_scale;
            }
            float u = root_bits(i < 4 ? vc.x : vc.y, i & 3, s.by.p19) * v_scale;
            if (wide_scale) u *= v_beyond;
            v[i] = u * u;
        }
        const float gi = g[i] * grad_scale;
        m[i] = s.beta1 * m[i] + s.one_beta1 * gi;
        v[i] = s.beta2 * v[i] + s.one_beta2 * gi * gi;
        root[i] = sqrt_near(v[i]);
        w[i] = w[i] * decay - step_size * (m[i] * reciprocal_near(root[i] * root_scale + s.eps));
        bad = fmaf(w[i], 0.f, bad);
        if constexpr (kNarrow || !kW32) h[i] = mix_rest(first ^ (uint32_t)i);
    }

    if constexpr (kW32) {
        if (vec) {
            store8(reinterpret_cast<float *>(T.w) + at(T.ldw, 0), w);
            if (T.copy)
                *reinterpret_cast<uint4 *>(T.copy + at(T.ldc, 0)) =
                    make_uint4(nearest2(w[0], w[1]), nearest2(w[2], w[3]), nearest2(w[4], w[5]), nearest2(w[6], w[7]));
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) {
                    reinterpret_cast<float *>(T.w)[at(T.ldw, i)] = w[i];
                    if (T.copy) T.copy[at(T.ldc, i)] = nearest(w[i]);
                }
        }
    } else {
        uint32_t r[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i)                        // bf16 weights: 11 bits of the hash decide about the 16 that do not fit
            r[i] = (h[i] >> 20 | 1u) * s.by.p4 + __float_as_uint(w[i]);
        if (bad != 0.f)                                       // (NaN: a weight is not finite, and adding to its bits may have made a number of it)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (!(fabsf(w[i]) <= 3.402823466e38f)) r[i] = (uint32_t)nearest(w[i]) << 16;
        if (vec) {
            *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(T.w) + at(T.ldw, 0)) =
                make_uint4(__byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632), __byte_perm(r[4], r[5], 0x7632), __byte_perm(r[6], r[7], 0x7632));
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) reinterpret_cast<uint16_t *>(T.w)[at(T.ldw, i)] = (uint16_t)(r[i] >> 16);
        }
    }
    if constexpr (!kNarrow) {
        float *pm = reinterpret_cast<float *>(T.m) + e0, *pv = reinterpret_cast<float *>(T.v) + e0;
        if (whole) {
            store8(pm, m); store8(pv, v);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) { pm[i] = m[i]; pv[i] = v[i]; }
        }
    } else {
        // (elements beyond the tensor's last one are zero: g, m and v were not read there)
        float am = 0.f, av = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) { am = fmaxf(am, fabsf(m[i])); av = fmaxf(av, root[i]); }
        if (bad != 0.f || !(am <= 3.402823466e38f) || !(av <= 3.402823466e38f)) {       // what is not finite is held as 0 (NaN in m or root is one in w)
            am = av = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (!(fabsf(m[i]) <= 3.402823466e38f)) m[i] = 0.f;
                if (!(root[i] <= 3.402823466e38f)) root[i] = 0.f;
                am = fmaxf(am, fabsf(m[i])); av = fmaxf(av, root[i]);
            }
        }
        // (the exponent of a block's scale is the largest of its threads': their two travel in one word)
        const uint32_t both = max_of_block(scale_of(am, 0x600000u) | scale_of(av, 0x780000u) << 16);
        const uint32_t em = both & 0xFFFFu, ev = both >> 16;
        // 2^-E 2^-120 in one factor; where that is below fp32's range, the values come down by 2^-120 first
        float down_m = power_of(134u - min(em, 133u)), down_v = power_of(134u - min(ev, 133u));
        if (em > 133u || ev > 133u) {
            const float first_m = em > 133u ? 0x1p-120f : 1.f, first_v = ev > 133u ? 0x1p-120f : 1.f;
            if (em > 133u) down_m = power_of(254u - em);
            if (ev > 133u) down_v = power_of(254u - ev);
#pragma unroll
            for (int i = 0; i < kPer; ++i) { m[i] *= first_m; root[i] *= first_v; }
        }
        uint32_t cm[kPer], cv[kPer];                          // codes as top bytes
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            // 20 (19) bits below the code, of which the hash gives the upper ten (eleven) and the one below them is set
            cm[i] = (((h[i] * s.by.p1 + 1u) & 0x7FFu) * s.by.p9 + __float_as_uint(m[i] * down_m)) * s.by.p4;
            const uint32_t t = ((h[i] >> 9 & 0xFFEu) | 1u) * s.by.p7 + __float_as_uint(root[i] * down_v);
            cv[i] = max(t, __float_as_uint(__saturatef(root[i] * 0x1p80f) * 0x1p-130f)) * s.by.p5;             // at least 1 where root is above 0
        }
        mc.x = top_bytes(cm[0], cm[1], cm[2], cm[3]);
        mc.y = top_bytes(cm[4], cm[5], cm[6], cm[7]);
        const auto sign = [&](int i) { return top_bytes(__float_as_uint(m[i]), __float_as_uint(m[i + 1]), __float_as_uint(m[i + 2]), __float_as_uint(m[i + 3])) & 0x80808080u; };
        mc.x |= sign(0);
        mc.y |= sign(4);
        vc = make_uint2(top_bytes(cv[0], cv[1], cv[2], cv[3]), top_bytes(cv[4], cv[5], cv[6], cv[7]));
        uint8_t *pm = reinterpret_cast<uint8_t *>(T.m) + e0, *pv = reinterpret_cast<uint8_t *>(T.v) + e0;
        if (whole) {
            *reinterpret_cast<uint2 *>(pm) = mc; *reinterpret_cast<uint2 *>(pv) = vc;
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < count) {
                    pm[i] = (uint8_t)((i < 4 ? mc.x : mc.y) >> (8 * (i & 3)));
                    pv[i] = (uint8_t)((i < 4 ? vc.x : vc.y) >> (8 * (i & 3)));
                }
        }
        if ((threadIdx.x & 15) == 0 && count) { T.m_exp[e0 >> 7] = (uint8_t)em; T.v_exp[e0 >> 7] = (uint8_t)ev; }
    }
}

template <bool kNarrow, bool kW32, int CAP>
__global__ void __launch_bounds__(kAdamThreads, kNarrow ? 5 : 4)
adamw_kernel(const __grid_constant__ Batch<AdamTensor, CAP> b, const __grid_constant__ AdamScalars s) {
    wait_for_prerequisites();
    const int l = b.find(blockIdx.x);
    const AdamTensor &T = b.layer[l];
    const int64_t first = (int64_t)(blockIdx.x - b.first[l]) * kPiece;
    if (T.plain && first + kPiece <= T.total) eight<kNarrow, kW32, true>(T, s, first + threadIdx.x * kPer);
    else eight<kNarrow, kW32, false>(T, s, first + threadIdx.x * kPer);
}

__global__ void __launch_bounds__(kAdamThreads)
moments_kernel(const uint8_t *m, const uint8_t *m_exp, const uint8_t *v, const uint8_t *v_exp, int64_t count, uint16_t *m_out, uint16_t *root_out, int vec) {
    wait_for_prerequisites();
    const int64_t e0 = ((int64_t)blockIdx.x * kAdamThreads + threadIdx.x) * kPer;
    if (e0 >= count) return;
    float beyond;
    const float sm = power_of(m_exp[e0 >> 7]), sv = power_120(v_exp[e0 >> 7], &beyond);
    const int here = (int)min((int64_t)kPer, count - e0);
    uint2 mc = make_uint2(0, 0), vc = make_uint2(0, 0);
    if (here == kPer) {
        mc = *reinterpret_cast<const uint2 *>(m + e0); vc = *reinterpret_cast<const uint2 *>(v + e0);
    } else {
        for (int i = 0; i < here; ++i) {
            (i < 4 ? mc.x : mc.y) |= (uint32_t)m[e0 + i] << (8 * (i & 3));
            (i < 4 ? vc.x : vc.y) |= (uint32_t)v[e0 + i] << (8 * (i & 3));
        }
    }
    uint32_t a[4], r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 two = values_m(i < 2 ? mc.x : mc.y, i & 1);
        const uint32_t c = i < 2 ? vc.x : vc.y;
        a[i] = nearest2(two.x * sm, two.y * sm);
        r[i] = nearest2(root_bits(c, 2 * (i & 1), 1u << 19) * sv * beyond, root_bits(c, 2 * (i & 1) + 1, 1u << 19) * sv * beyond);
    }
    if (vec && here == kPer) {
        *reinterpret_cast<uint4 *>(m_out + e0) = make_uint4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<uint4 *>(root_out + e0) = make_uint4(r[0], r[1], r[2], r[3]);
        return;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < here) {
            m_out[e0 + i] = (uint16_t)(a[i >> 1] >> (16 * (i & 1)));
            root_out[e0 + i] = (uint16_t)(r[i >> 1] >> (16 * (i & 1)));
        }
}

template <int CAP>
cudaError_t launch_pieces(const AdamTensor *tensors, int n, bool narrow, bool w32, const AdamScalars &s, cudaStream_t st) {
    std::unique_ptr<Batch<AdamTensor, CAP>> b(new (std::nothrow) Batch<AdamTensor, CAP>);
    if (!b) return cudaErrorMemoryAllocation;
    for (int l = 0; l < n;) {
        int count = 0;
        int64_t pieces = 0;
        for (; l < n && count < CAP; ++l) {
            const int64_t here = (tensors[l].total + kPiece - 1) / kPiece;
            if (pieces + here > 0x7FFFFFFFll) {
                if (count == 0) return cudaErrorInvalidValue;
                break;
            }
            b->layer[count] = tensors[l];
            b->first[count++] = pieces;
            pieces += here;
        }
        b->n = count;
        b->first[count] = pieces;
        cudaError_t e;
        if (narrow) e = w32 ? launch_chained(adamw_kernel<true, true, CAP>, (unsigned)pieces, kAdamThreads, 0, st, *b, s)
                            : launch_chained(adamw_kernel<true, false, CAP>, (unsigned)pieces, kAdamThreads, 0, st, *b, s);
        else e = w32 ? launch_chained(adamw_kernel<false, true, CAP>, (unsigned)pieces, kAdamThreads, 0, st, *b, s)
                     : launch_chained(adamw_kernel<false, false, CAP>, (unsigned)pieces, kAdamThreads, 0, st, *b, s);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The entry of one tensor (all arguments but the mask's shape are checked here).
crisp_status_t entry(const crisp_adamw_tensor_t &t, int32_t ordinal, const crisp_adamw_t &p, AdamTensor *T) {
    if (t.rows < 0 || t.k < 0) return CRISP_BAD_SHAPE;
    if (t.k > 0x7FFFFFFFll) return CRISP_UNSUPPORTED;
    if (t.k > 0 && t.rows > ((int64_t)1 << 44) / t.k) return CRISP_UNSUPPORTED;
    T->total = t.rows * t.k;
    if (T->total == 0 || !t.d_grad) { T->total = 0; return CRISP_OK; }
    if ((t.w_dtype != 0 && t.w_dtype != 1) || (t.grad_dtype != 0 && t.grad_dtype != 1)) return CRISP_INVALID_ARG;
    if (!t.d_w || !t.d_m || !t.d_v || (t.d_copy_bf16 && t.w_dtype != 1)) return CRISP_INVALID_ARG;
    const size_t ws = t.w_dtype ? 4 : 2, gs = t.grad_dtype ? 4 : 2;
    if (!aligned_to(t.d_w, ws) || !aligned_to(t.d_grad, gs) || !aligned_to(t.d_copy_bf16, 2) || !aligned_to(t.d_m, 16) || !aligned_to(t.d_v, 16))
        return CRISP_INVALID_ARG;
    if (p.state_bits == 8 && (!t.d_m_exp || !t.d_v_exp)) return CRISP_INVALID_ARG;
    if (t.rows > 1 && (t.ld_w < t.k || t.ld_grad < t.k || (t.d_copy_bf16 && t.ld_copy < t.k))) return CRISP_BAD_SHAPE;
    T->w = t.d_w; T->copy = t.d_copy_bf16; T->g = t.d_grad; T->m = t.d_m; T->v = t.d_v; T->m_exp = t.d_m_exp; T->v_exp = t.d_v_exp;
    T->ldw = t.ld_w; T->ldc = t.ld_copy; T->ldg = t.ld_grad;
    T->k = (uint32_t)t.k;
    T->g32 = t.grad_dtype == 1;
    T->flat = t.rows == 1 || (t.ld_w == t.k && t.ld_grad == t.k && (!t.d_copy_bf16 || t.ld_copy == t.k));
    T->bytes = t.k % 8 == 0;
    const bool ends = aligned_to(t.d_w, 16) && aligned_to(t.d_grad, 16) && aligned_to(t.d_copy_bf16, 16);
    T->vec = ends && (T->flat || (T->bytes && t.ld_w * ws % 16 == 0 && t.ld_grad * gs % 16 == 0 && (!t.d_copy_bf16 || t.ld_copy % 8 == 0)));
    T->mask = nullptr; T->wpr = 0;
    if (t.mask) {
        if (t.mask->g.rows != t.rows || t.mask->g.k != t.k) return CRISP_BAD_SHAPE;
        T->mask = t.mask->d_nm_bits; T->wpr = (uint32_t)t.mask->g.wpr;
    }
    T->plain = T->flat && T->vec && (T->bytes || !T->mask);
    T->ordinal = (uint32_t)ordinal;
    return CRISP_OK;
}

}  // namespace

}  // namespace crisp

extern "C" {

crisp_status_t crisp_adamw(int32_t n, const crisp_adamw_tensor_t *tensors, const crisp_adamw_t *p, void *stream) {
    using namespace crisp;
    if (n < 0 || (n > 0 && !tensors) || !p) return CRISP_INVALID_ARG;
    if (p->state_bits != 32 && p->state_bits != 8) return CRISP_INVALID_ARG;
    if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0) || !(p->eps >= 0.0) || !std::isfinite(p->eps) ||
        !std::isfinite(p->lr) || !std::isfinite(p->weight_decay) || p->reserved != 0)
        return CRISP_INVALID_ARG;
    if (!p->d_step && p->step < 1) return CRISP_INVALID_ARG;
    if (!aligned_to(p->d_lr, 4) || !aligned_to(p->d_step, 8) || !aligned_to(p->d_grad_scale, 4)) return CRISP_INVALID_ARG;
    if (n == 0) return CRISP_OK;
    AdamScalars s{};
    s.lr = (float)p->lr;
    s.beta1 = (float)p->beta1; s.one_beta1 = (float)(1.0 - p->beta1);
    s.beta2 = (float)p->beta2; s.one_beta2 = (float)(1.0 - p->beta2);
    s.eps = std::max((float)p->eps, 1.17549435e-38f);          // 0 / 0 is 0; no root above 0 is that small
    s.weight_decay = (float)p->weight_decay;
    s.decay = (float)(1.0 - p->lr * p->weight_decay);
    // (the factor of a device lr: taken with lr = 1, so that nothing is divided by an lr of 0)
    const double t = (double)p->step;
    const double unit = p->d_step ? 1.0 : 1.0 / -std::expm1(t * std::log(p->beta1));
    if (p->d_lr) s.lr = 1.f;
    s.step_size = (float)((p->d_lr ? 1.0 : p->lr) * unit);
    s.root_scale = p->d_step ? 1.f : (float)(1.0 / std::sqrt(-std::expm1(t * std::log(p->beta2))));
    s.log_beta1 = (float)std::log(p->beta1); s.log_beta2 = (float)std::log(p->beta2);
    s.seed_key = mix(mix((uint32_t)p->seed) ^ (uint32_t)(p->seed >> 32));
    s.d_lr = p->d_lr; s.d_step = p->d_step; s.d_grad_scale = p->d_grad_scale;
    const uint32_t step_key = mix(s.seed_key ^ (uint32_t)p->step);

    // the entries, those with fp32 weights first (a launch's weights are of one type)
    std::unique_ptr<AdamTensor[]> table(new (std::nothrow) AdamTensor[(size_t)n]);
    std::unique_ptr<const void *[]> seen(new (std::nothrow) const void *[(size_t)n]);
    if (!table || !seen) return CRISP_CUDA_ERROR;
    int count[2] = {0, 0};
    for (int32_t i = 0; i < n; ++i) {
        AdamTensor T{};
        const crisp_status_t bad = entry(tensors[i], i, *p, &T);
        if (bad != CRISP_OK) return bad;
        if (T.total == 0) continue;
        T.key = mix(step_key ^ T.ordinal);
        T.spread = mix(T.key);
        seen[count[0] + count[1]] = T.w;
        if (tensors[i].w_dtype == 1) table[count[1]++] = T;
        else table[n - ++count[0]] = T;
    }
    const int all = count[0] + count[1];
    std::sort(seen.get(), seen.get() + all);
    for (int i = 1; i < all; ++i)
        if (seen[i] == seen[i - 1]) return CRISP_INVALID_ARG;
    for (int w32 = 1; w32 >= 0; --w32) {
        if (!count[w32]) continue;
        const AdamTensor *first = w32 ? table.get() : table.get() + (n - count[0]);
        const cudaError_t e = count[w32] <= 8 ? launch_pieces<8>(first, count[w32], p->state_bits == 8, w32 != 0, s, (cudaStream_t)stream)
                                              : launch_pieces<128>(first, count[w32], p->state_bits == 8, w32 != 0, s, (cudaStream_t)stream);
        if (e == cudaErrorInvalidValue) return CRISP_UNSUPPORTED;
        if (e != cudaSuccess) return CRISP_CUDA_ERROR;
    }
    return CRISP_OK;
}

crisp_status_t crisp_adamw_moments(const uint8_t *d_m, const uint8_t *d_m_exp, const uint8_t *d_v, const uint8_t *d_v_exp, int64_t count,
                                   uint16_t *d_m_bf16, uint16_t *d_root_bf16, void *stream) {
    using namespace crisp;
    if (count < 0) return CRISP_BAD_SHAPE;
    if (count == 0) return CRISP_OK;
    if (!d_m || !d_m_exp || !d_v || !d_v_exp || !d_m_bf16 || !d_root_bf16) return CRISP_INVALID_ARG;
    if (!aligned_to(d_m, 16) || !aligned_to(d_v, 16) || !aligned_to(d_m_bf16, 2) || !aligned_to(d_root_bf16, 2)) return CRISP_INVALID_ARG;
    const int64_t ctas = (count + kPiece - 1) / kPiece;
    if (ctas > 0x7FFFFFFFll) return CRISP_UNSUPPORTED;
    const int vec = aligned_to(d_m_bf16, 16) && aligned_to(d_root_bf16, 16);
    const cudaError_t e = launch_chained(moments_kernel, (unsigned)ctas, kAdamThreads, 0, (cudaStream_t)stream, d_m, d_m_exp, d_v, d_v_exp, count, d_m_bf16,
                                         d_root_bf16, vec);
    return e == cudaSuccess ? CRISP_OK : CRISP_CUDA_ERROR;
}

}  // extern "C"
