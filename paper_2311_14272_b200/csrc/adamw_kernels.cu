// One AdamW step over all tensors of a network (the fine-tuning of Algorithm 1), states in 32 or in 8 bits.
//
//   g = grad * scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w = w (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every element is read and written once, so the bytes bound it: 28 an element for fp32 weights, gradients and states, 10 for bf16 weights and
// gradients with 8-bit states.  A thread takes eight consecutive elements (16 or 32 bytes of each tensor, 8 of an 8-bit state), so that half a warp
// holds the 128 elements of a scale and finds their largest value by shuffles; the tensors of a call are numbered through in pieces of
// 2048 elements, one CTA each, and their table travels as a kernel parameter.
//
// Measured on four tensors of 4096 x 4096 with bf16 gradients: 32-bit states 254 us with fp32 weights under masks (6.9 TB/s), 215 with bf16 ones (6.9).
// 8-bit states 159 us with bf16 weights (4.2 TB/s), 169 under masks, 171 with fp32 weights (5.5): some 80 instructions an element, six in seven of the schedulers'
// cycles, bound these.  What brought them there from 356: no questions asked for each element in pieces that need none (287 -> 195), products instead of shifts
// (287 -> 267 before that), codes packed by byte permutes, cvt.rs for bf16 weights, five CTAs an SM (four 187, six 172 and seven 188 with spills).  Not kept: two or four turns
// of eight elements a thread (190 and 252; with the loads ahead 184).
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
constexpr float kLargest = 3.402823466e38f;

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
    uint32_t by_k, shift;    // e / k = umulhi(e, by_k) >> shift for e below 2^31 (plain tensors under masks)
    uint8_t g32;             // gradients are fp32
    uint8_t flat;            // w, g and copy are packed: element e lies at e
    uint8_t vec;             // eight elements from a multiple of eight on lie in a row and at multiples of 16 bytes
    uint8_t bytes;           // k is a multiple of 8: eight elements' mask bits are one byte
    uint8_t plain;           // flat, vec and, under a mask, bytes
};

// Powers of two as parameters of the kernel.  The 8-bit kernel is bound by the integer pipe, and a product with a number that the compiler does not
// know goes to the multiply-add pipe instead of becoming a shift.
struct Powers { uint32_t p1 = 1u << 1, p4 = 1u << 4, p5 = 1u << 5, p7 = 1u << 7, p6 = 1u << 6, p9 = 1u << 9; };

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
__device__ __forceinline__ uint32_t nearest2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint16_t nearest(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

// The 8-bit forms.  A code is the top of an fp32 number whose exponent field has been brought down by 120 (127 - 7), so that small codes are
// subnormal as fp32's are: rounding is an addition to the bits below the code.
__device__ __forceinline__ float power_of(uint32_t biased) { return __uint_as_float(biased << 23); }       // 2^(biased - 127), 0 for 0
// 2^(E + 8) of a biased scale exponent: what a code of sqrt(v) is multiplied by.  (E is 56 at most: sqrt(v) is below 2^64.)
__device__ __forceinline__ float power_8(uint32_t biased) { return power_of(min(biased + 8u, 254u)); }
// The top bytes of four words.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
// Two codes of sqrt(v), 2^8 too small: e4m4 with bias 7 is the top of an fp16 number with bias 15 whose sign and first exponent bit are 0.
__device__ __forceinline__ float2 values_root(uint32_t codes, int pair, uint32_t p6) {
    const uint32_t h = __byte_perm(codes, 0, pair ? 0x4342 : 0x4140) * p6;
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
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
// bf16 weights, rounded at random: 11 bits of each hash and a set one below them decide about the 16 bits that do not fit.
__device__ __forceinline__ uint32_t random2(float lo, float hi, uint32_t h_lo, uint32_t h_hi) {
    const uint32_t random = (__byte_perm(h_lo, h_hi, 0x7632) & 0xFFE0FFE0u) | 0x00100010u;
    uint32_t r;
    asm("cvt.rs.bf16x2.f32 %0, %1, %2, %3;" : "=r"(r) : "f"(hi), "f"(lo), "r"(random));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Bit i of the byte in every bit of byte i of (lo, hi).
__device__ __forceinline__ uint2 bytes_of_bits(uint32_t keep) {
    return make_uint2(((keep & 15u) * 0x00204081u & 0x01010101u) * 255u, ((keep >> 4) * 0x00204081u & 0x01010101u) * 255u);
}

// What a step reads of eight elements of a thread, as it lies in memory (weights and gradients: bf16 pairs or fp32).
template <bool kNarrow, bool kW32>
struct Eight {
    uint32_t w[kW32 ? 8 : 4], g[8];
    float m[kNarrow ? 1 : 8], v[kNarrow ? 1 : 8];
    uint2 mc, vc;            // codes of 8-bit states
    uint32_t m_exp, v_exp, keep;
};
// What it takes beside them.
struct Factors {
    float decay, step_size, root_scale, grad_scale;
    uint32_t key, spread;
};
// The row and column of element e0.
template <bool kPlain>
__device__ __forceinline__ void place(const AdamTensor &T, int64_t e0, int64_t *row, uint32_t *col) {
    if (kPlain && T.by_k) {                                   // (a product instead of a division of some twenty instructions)
        const uint32_t r = __umulhi((uint32_t)e0, T.by_k) >> T.shift;
        *row = r; *col = (uint32_t)e0 - r * T.k;
    } else if (T.total <= 0xFFFFFFFFll) {
        const uint32_t r = (uint32_t)e0 / T.k;
        *row = r; *col = (uint32_t)e0 - r * T.k;
    } else {
        *row = e0 / T.k; *col = (uint32_t)(e0 - *row * T.k);
    }
}
template <int N>
__device__ __forceinline__ void load_words(const void *p, uint32_t (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const uint4 a = reinterpret_cast<const uint4 *>(p)[i / 4];
        x[i] = a.x; x[i + 1] = a.y; x[i + 2] = a.z; x[i + 3] = a.w;
    }
}

// kPlain: the eight elements are the tensor's, lie packed at multiples of 16 bytes, and their mask bits in a byte.  What all others have to ask for each element
// is left out of the code.
template <bool kNarrow, bool kW32, bool kPlain>
struct Piece {
    const AdamTensor &T;
    const int64_t e0;
    int count;
    bool whole, vec, flat;
    int64_t row;
    uint32_t col;

    __device__ __forceinline__ Piece(const AdamTensor &t, int64_t e) : T(t), e0(e), row(0), col(0) {
        count = kPlain ? kPer : (int)max((int64_t)0, min((int64_t)kPer, T.total - e0));
        whole = kPlain || count == kPer; vec = kPlain || (T.vec && whole); flat = kPlain || T.flat;
        if (T.mask || !flat) place<kPlain>(T, e0, &row, &col);
    }
    // where element i of rows of pitch ld lies
    __device__ __forceinline__ int64_t at(int64_t ld, int i) const {
        if (flat) return e0 + i;
        int64_t r = row;
        uint32_t c = col + i;
        while (c >= T.k) { c -= T.k; ++r; }
        return r * ld + c;
    }
    __device__ __forceinline__ void read(Eight<kNarrow, kW32> &x) const {
        const uint16_t *w16 = reinterpret_cast<const uint16_t *>(T.w), *g16 = reinterpret_cast<const uint16_t *>(T.g);
        const uint32_t *w32 = reinterpret_cast<const uint32_t *>(T.w), *g32 = reinterpret_cast<const uint32_t *>(T.g);
        if (vec) {
            if constexpr (kW32) load_words(w32 + at(T.ldw, 0), x.w);
            else load_words(w16 + at(T.ldw, 0), x.w);
            if (T.g32) load_words(g32 + at(T.ldg, 0), x.g);
            else load_words(g16 + at(T.ldg, 0), reinterpret_cast<uint32_t (&)[4]>(x.g));
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const bool in = i < count;
                if constexpr (kW32) {
                    x.w[i] = in ? w32[at(T.ldw, i)] : 0u;
                } else {
                    const uint32_t bits = in ? (uint32_t)w16[at(T.ldw, i)] << (16 * (i & 1)) : 0u;
                    x.w[i / 2] = i & 1 ? x.w[i / 2] | bits : bits;
                }
                if (T.g32) {
                    x.g[i] = in ? g32[at(T.ldg, i)] : 0u;
                } else {
                    const uint32_t bits = in ? (uint32_t)g16[at(T.ldg, i)] << (16 * (i & 1)) : 0u;
                    x.g[i / 2] = i & 1 ? x.g[i / 2] | bits : bits;
                }
            }
        }
        if constexpr (!kNarrow) {
            const float *pm = reinterpret_cast<const float *>(T.m) + e0, *pv = reinterpret_cast<const float *>(T.v) + e0;
            if (whole) {
                load8(pm, x.m); load8(pv, x.v);
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i) { x.m[i] = i < count ? pm[i] : 0.f; x.v[i] = i < count ? pv[i] : 0.f; }
            }
        } else {
            const uint8_t *pm = reinterpret_cast<const uint8_t *>(T.m) + e0, *pv = reinterpret_cast<const uint8_t *>(T.v) + e0;
            x.mc = x.vc = make_uint2(0, 0);
            x.m_exp = x.v_exp = 0;
            if (whole) {
                x.mc = *reinterpret_cast<const uint2 *>(pm); x.vc = *reinterpret_cast<const uint2 *>(pv);
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (i < count) {
                        (i < 4 ? x.mc.x : x.mc.y) |= (uint32_t)pm[i] << (8 * (i & 3));
                        (i < 4 ? x.vc.x : x.vc.y) |= (uint32_t)pv[i] << (8 * (i & 3));
                    }
            }
            if (count) { x.m_exp = T.m_exp[e0 >> 7]; x.v_exp = T.v_exp[e0 >> 7]; }
        }
        x.keep = 0xFFu;
        if (T.mask && count) {
            if (kPlain || T.bytes) {
                x.keep = reinterpret_cast<const uint8_t *>(T.mask + row * T.wpr)[col >> 3];
            } else {
                int64_t r = row;
                uint32_t c = col;
                x.keep = 0;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (i < count) {
                        x.keep |= (T.mask[r * T.wpr + (c >> 5)] >> (c & 31) & 1u) << i;
                        if (++c == T.k) { c = 0; ++r; }
                    }
            }
        }
    }

    __device__ __forceinline__ void update(Eight<kNarrow, kW32> &x, const AdamScalars &s, const Factors &f) const {
        // Where the mask has no bit: zeros go in and zeros come out (eps is above 0).
        if (T.mask) {
            const uint2 b = bytes_of_bits(x.keep);
            if constexpr (kNarrow) { x.mc.x &= b.x; x.mc.y &= b.y; x.vc.x &= b.x; x.vc.y &= b.y; }
            uint32_t pairs[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) pairs[i] = __byte_perm(i < 2 ? b.x : b.y, 0, i & 1 ? 0x3322 : 0x1100);
            if constexpr (!kW32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x.w[i] &= pairs[i];
            }
            if (!T.g32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x.g[i] &= pairs[i];
            }
            if (kW32 || !kNarrow || T.g32) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (!(x.keep >> i & 1u)) {
                        if constexpr (kW32) x.w[i] = 0;
                        if constexpr (!kNarrow) x.m[i] = x.v[i] = 0.f;
                        if (T.g32) x.g[i] = 0;
                    }
            }
        }
        float w[kPer], g[kPer], m[kPer], root[kPer], v[kPer];
        uint32_t h[kPer];
        uint32_t spread = f.spread;
        if (kNarrow || !kW32)
            if (e0 >> 32) spread = mix((uint32_t)(e0 >> 32) ^ f.key);
        // (e0 is a multiple of 8: the hash of e0 + i differs from that of e0 in three low bits until its first product)
        const uint32_t first = ((uint32_t)e0 ^ spread) ^ (((uint32_t)e0 ^ spread) >> 16);
        float m_scale = 0.f, v_scale = 0.f;
        if constexpr (kNarrow) { m_scale = s.beta1 * power_of(x.m_exp); v_scale = power_8(x.v_exp); }
        if (T.g32) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) g[i] = __uint_as_float(x.g[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) g[i] = __uint_as_float(i & 1 ? x.g[i / 2] & 0xFFFF0000u : x.g[i / 2] << 16);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if constexpr (kW32) w[i] = __uint_as_float(x.w[i]);
            else w[i] = __uint_as_float(i & 1 ? x.w[i / 2] & 0xFFFF0000u : x.w[i / 2] << 16);
            if constexpr (kNarrow) {
                if ((i & 1) == 0) {
                    const float2 two = values_m(i < 4 ? x.mc.x : x.mc.y, i >> 1 & 1), roots = values_root(i < 4 ? x.vc.x : x.vc.y, i >> 1 & 1, s.by.p6);
                    m[i] = two.x * m_scale; m[i + 1] = two.y * m_scale;
                    v[i] = roots.x * v_scale; v[i + 1] = roots.y * v_scale;
                }
                v[i] *= v[i];
            } else {
                m[i] = x.m[i]; v[i] = x.v[i];
            }
            const float gi = g[i] * f.grad_scale;
            // (m in 8 bits comes with the factor beta1 in its scale)
            m[i] = fmaf(s.one_beta1, gi, kNarrow ? m[i] : s.beta1 * m[i]);
            v[i] = fmaf(s.one_beta2 * gi, gi, s.beta2 * v[i]);
            root[i] = sqrt_near(v[i]);
            w[i] = w[i] * f.decay - f.step_size * (m[i] * reciprocal_near(root[i] * f.root_scale + s.eps));
            if constexpr (kNarrow || !kW32) h[i] = mix_rest(first ^ (uint32_t)i);
        }

        // (zero times what is not finite is not zero)
        if (T.mask && !(fmaf(f.grad_scale, 0.f, fmaf(f.step_size, 0.f, fmaf(f.root_scale, 0.f, f.decay * 0.f))) == 0.f)) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (!(x.keep >> i & 1u)) w[i] = m[i] = v[i] = root[i] = 0.f;
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
            uint32_t r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = random2(w[2 * i], w[2 * i + 1], h[2 * i], h[2 * i + 1]);
            if (vec) {
                *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(T.w) + at(T.ldw, 0)) = make_uint4(r[0], r[1], r[2], r[3]);
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (i < count) reinterpret_cast<uint16_t *>(T.w)[at(T.ldw, i)] = (uint16_t)(r[i / 2] >> (16 * (i & 1)));
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
            hold(m, root, h, s);
        }
    }

    // m and sqrt(v) to their 8-bit forms; the 16 threads of a block come here together.
    __device__ __forceinline__ void hold(float (&m)[kPer], float (&root)[kPer], const uint32_t (&h)[kPer], const AdamScalars &s) const {
        // (elements beyond the tensor's last one are zero: g, m and v were not read there)
        float am = 0.f, av = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) { am = max_nan(am, fabsf(m[i])); av = max_nan(av, root[i]); }
        if (!(am <= kLargest) || !(av <= kLargest)) {
            // An element of which one is not finite is held as 0 in both: the square of a finite gradient may leave fp32, and its m over an sqrt(v) of 0 would be
            // the next step's update.
            am = av = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (!(fabsf(m[i]) <= kLargest) || !(root[i] <= kLargest)) m[i] = root[i] = 0.f;
                am = fmaxf(am, fabsf(m[i])); av = fmaxf(av, root[i]);
            }
        }
        // (the exponent of a block's scale is the largest of its threads': their two travel in one word)
        const uint32_t both = max_of_block(scale_of(am, 0x600000u) | scale_of(av, 0x780000u) << 16);
        const uint32_t em = both & 0xFFFFu, ev = both >> 16;
        // 2^-E 2^-120 in one factor; where that is below fp32's range, the values come down by 2^-120 first
        float down_m = power_of(134u - min(em, 133u)), down_v = power_of(134u - min(ev, 133u));
        if (em > 133u || ev > 133u) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (em > 133u) m[i] *= 0x1p-120f;
                if (ev > 133u) root[i] = root[i] > 0.f ? fmaxf(root[i] * 0x1p-120f, 0x1p-126f) : 0.f;
            }
            if (em > 133u) down_m = power_of(254u - em);
            if (ev > 133u) down_v = power_of(254u - ev);
        }
        uint32_t cm[kPer], cv[kPer];                              // codes as top bytes
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            // 20 (19) bits below the code, of which the hash gives the upper ten (eleven) and the one below them is set
            cm[i] = (((h[i] * s.by.p1 + 1u) & 0x7FFu) * s.by.p9 + __float_as_uint(m[i] * down_m)) * s.by.p4;
            const uint32_t t = ((h[i] >> 9 & 0xFFEu) | 1u) * s.by.p7 + __float_as_uint(root[i] * down_v);
            cv[i] = max(t, min(__float_as_uint(root[i]), 1u << 19)) * s.by.p5;                              // at least 1 where root is above 0 (it is 2^-126 or more)
        }
        const auto sign = [&](int i) {
            return top_bytes(__float_as_uint(m[i]), __float_as_uint(m[i + 1]), __float_as_uint(m[i + 2]), __float_as_uint(m[i + 3])) & 0x80808080u;
        };
        const uint2 mc = make_uint2(top_bytes(cm[0], cm[1], cm[2], cm[3]) | sign(0), top_bytes(cm[4], cm[5], cm[6], cm[7]) | sign(4));
        const uint2 vc = make_uint2(top_bytes(cv[0], cv[1], cv[2], cv[3]), top_bytes(cv[4], cv[5], cv[6], cv[7]));
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
};

template <bool kNarrow, bool kW32, int CAP>
__global__ void __launch_bounds__(kAdamThreads, kNarrow ? 5 : 4)
adamw_kernel(const __grid_constant__ Batch<AdamTensor, CAP> b, const __grid_constant__ AdamScalars s) {
    wait_for_prerequisites();
    const int l = b.find(blockIdx.x);
    const AdamTensor &T = b.layer[l];
    const int64_t first = (int64_t)(blockIdx.x - b.first[l]) * kPiece, e0 = first + threadIdx.x * kPer;
    Factors f{s.decay, s.step_size, s.root_scale, s.d_grad_scale ? *s.d_grad_scale : 1.f, T.key, T.spread};
    if (s.d_step || s.d_lr) {
        const float lr = s.d_lr ? *s.d_lr : s.lr;
        const float t = s.d_step ? (float)*s.d_step : 0.f;
        // 1 - b^t = -expm1(t log b): to a rounding or two of fp32 for any t
        if (s.d_step) {
            f.root_scale = 1.f / sqrtf(-expm1f(t * s.log_beta2));
            f.key = mix(mix(s.seed_key ^ (uint32_t)*s.d_step) ^ T.ordinal);
            f.spread = mix(f.key);
        }
        f.step_size = s.d_step ? lr / -expm1f(t * s.log_beta1) : s.step_size / s.lr * lr;
        f.decay = 1.f - lr * s.weight_decay;
    }
    Eight<kNarrow, kW32> x;
    if (T.plain && first + kPiece <= T.total) {
        const Piece<kNarrow, kW32, true> piece(T, e0);
        piece.read(x);
        piece.update(x, s, f);
    } else {
        const Piece<kNarrow, kW32, false> piece(T, e0);
        piece.read(x);
        piece.update(x, s, f);
    }
}

__global__ void __launch_bounds__(kAdamThreads)
moments_kernel(const uint8_t *m, const uint8_t *m_exp, const uint8_t *v, const uint8_t *v_exp, int64_t count, uint16_t *m_out, uint16_t *root_out, int vec) {
    wait_for_prerequisites();
    const int64_t e0 = ((int64_t)blockIdx.x * kAdamThreads + threadIdx.x) * kPer;
    if (e0 >= count) return;
    const float sm = power_of(m_exp[e0 >> 7]), sv = power_8(v_exp[e0 >> 7]);
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
        const float2 roots = values_root(i < 2 ? vc.x : vc.y, i & 1, 1u << 6);
        a[i] = nearest2(two.x * sm, two.y * sm);
        r[i] = nearest2(roots.x * sv, roots.y * sv);
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
    if (t.k > 0x7FFFFFFFll && (t.rows > 1 || t.mask)) return CRISP_UNSUPPORTED;        // (columns are counted in 31 bits where they count)
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
    T->by_k = T->shift = 0;
    if (T->plain && T->mask && T->total < (int64_t)1 << 31) {
        // l = ceil(log2 k) and by_k = ceil(2^(31 + l) / k) < 2^32: exact for numerators below 2^31
        uint32_t l = 0;
        while (((uint64_t)1 << l) < (uint64_t)t.k) ++l;
        T->by_k = (uint32_t)((((uint64_t)1 << (31 + l)) + (uint64_t)t.k - 1) / (uint64_t)t.k);
        T->shift = l - 1;                                     // (k is 8 or more)
    }
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
