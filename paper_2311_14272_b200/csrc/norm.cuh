// Group norm with an activation over channels-last activations, forward and backward.
//
//   of a sample's group (pixels x C / G channels):  mean, rstd = 1 / sqrt(var + eps)
//   h = (x - mean) rstd      y = act(p), p = gamma h + beta
//   backward:  e = dy act'(p)   dbeta = sum e   dgamma = sum e h   dx = rstd (gamma e - m1 - h m2),  m1, m2 = the group's means of gamma e, gamma e h
//
// Bound by memory: each value is needed twice, and what counts is that it comes from DRAM once.
//
//   small calls   one kernel: a cluster of CTAs takes a sample's slice of whole groups, every thread keeps what it has read in shared memory of its own (no barrier: it
//                 reads what it wrote) until the cluster's sums are there
//   large ones    two kernels of as many CTAs as fit, each with its part of the pixels.  The second goes over them backwards: what the first read last
//                 is still in L2 (forward, us, backwards and not: 32 x 112 x 112 x 96, 77 MB, 38 and 42; of 50 MB 25 and 24; of 200 MB 115 and 116)
//
// A thread holds V = 16 bytes' worth of consecutive channels and goes over pixels, two channels an instruction: per pair p = a (x - mean) + beta (a = gamma rstd),
// dx = a e + B (x - mean) + C.  (With a x + (beta - mean a), an addition less, mean a is rounded: equal values of -700 gave y off by 0.016; the times are the same.)  Forward sums are about the thread's first value, and then about its mean so far, so that neither a mean far from zero nor single
// values far from the mean cost digits; then mean = sum n_i mean_i / n and M2 = sum M2_i + n_i (mean_i - mean)^2 over threads and over CTAs, always in the same order.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "block8.h"
#include "block8.cuh"
#include "mask_common.cuh"

namespace crisp {
namespace norm {

using namespace block8;

constexpr int kThreads = 256;
constexpr int kForwardCtas = 3, kBackwardCtas = 2;            // an SM, in large calls
constexpr int kMaxCluster = 16;
constexpr size_t kMaxSmem = 232448 - 1024;

enum Act { kNone = 0, kRelu = 1, kRelu6 = 2, kSilu = 3 };

struct Norm {
    const void *x, *dy;                  // dy: backward
    void *out;                           // y (or nullptr), dx
    const uint8_t *from8;                // backward: x in 8 bits (x: nullptr)
    uint8_t *x8, *y8;                    // forward: 8-bit forms to write, or nullptr
    const float *gamma, *beta;           // or nullptr: 1, 0
    float *stats;                        // [batch, groups, 2]
    float *sums;                         // backward: [batch * ranks][2][channels]
    float2 *partial;                     // large calls: [batch, groups, ranks, parts]
    int64_t ldx, ld_dy, ld_out;
    int64_t groups8, chunks8;            // 8-bit form: groups of 8 and of 128 columns (pixels of all samples)
    size_t scale_off;
    int pixels, channels, groups, cpg;   // cpg: channels a group
    int width, slices;                   // channels a slice, slices a sample
    int ranks, per;                      // CTAs of a sample's slice, pixels of one
    int parts;                           // the most slices that a group lies in
    int cv, lanes;                       // threads a pixel, pixels at a time
    int some, more, some_last, more_last;    // items of a pixel lane: `some`, the first `more` lanes one more (the last rank's: ..._last)
    int resident;                        // items (V channels of a pixel) that a thread keeps
    uint32_t across_magic, cpg_magic;    // 2^32 / (entries of a whole group and lane), / cpg, rounded up (0: not exact for all channels)
    int as_stored;                       // backward from 8 bits: codes keep their order on the way (slices of whole blocks of 128 channels, an order for each place of the ring)
    int act, vec, vec_dy, vec_out;       // vec: addresses and pitches allow 16 bytes at once
    float eps;
};

// V values as pairs.
template <typename T>
struct Of;
template <>
struct Of<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void open(const uint4 &u, uint64_t (&f)[2]) {
        f[0] = f32x2(__uint_as_float(u.x), __uint_as_float(u.y)); f[1] = f32x2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ uint4 close(const uint64_t (&f)[2]) {
        const float2 a = f32x2_halves(f[0]), b = f32x2_halves(f[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
    static __device__ __forceinline__ float sigmoid(float p) { return 1.f / (1.f + expf(-p)); }
    static __device__ __forceinline__ uint64_t sigmoid2(uint64_t p) { const float2 v = f32x2_halves(p); return f32x2(sigmoid(v.x), sigmoid(v.y)); }
};
struct Of16 {
    static constexpr int V = 8;
    // (some 2^-20 of the value, far below the result's last place; 0 where it is below 2^-126)
    static __device__ __forceinline__ float sigmoid(float p) {
        float e, r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(p * -1.44269504f));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
        return r;
    }
    // Of two values, with one reciprocal of the product of both denominators: the special function unit is what the forward pass with silu is bound by (75 % of its rate with
    // four of its instructions a pair).  Where a denominator is above 2^62, or NaN, each for itself.
    static __device__ __forceinline__ uint64_t sigmoid2(uint64_t p) {
        const float2 v = f32x2_halves(mul2(p, f32x2(-1.44269504f, -1.44269504f)));
        float a, b, r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(v.x));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(v.y));
        if (!(max_nan(a, b) <= 0x1p62f)) { const float2 w = f32x2_halves(p); return f32x2(sigmoid(w.x), sigmoid(w.y)); }
        a += 1.f; b += 1.f;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a * b));
        return mul2(f32x2(r, r), f32x2(b, a));
    }
};
template <>
struct Of<__nv_bfloat16> : Of16 {
    static __device__ __forceinline__ void open(const uint4 &u, uint64_t (&f)[4]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    }
    static __device__ __forceinline__ uint4 close(const uint64_t (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = f32x2_halves(f[i]);
            const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Of<__half> : Of16 {
    static __device__ __forceinline__ void open(const uint4 &u, uint64_t (&f)[4]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[i])); f[i] = f32x2(v.x, v.y); }
    }
    static __device__ __forceinline__ uint4 close(const uint64_t (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = f32x2_halves(f[i]);
            const __half2 b = __floats2half2_rn(v.x, v.y);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t both(float v) { return f32x2(v, v); }

__device__ __forceinline__ uint32_t smem_at(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
template <int kBytes>
__device__ __forceinline__ void copy_async(void *to, const void *from) {
    if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(to)), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_at(to)), "l"(from), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// V channels of one pixel, `n` of them there (the others 0).  kVec: all of them, at a multiple of 16 bytes.
template <bool kVec, typename T>
__device__ __forceinline__ uint4 fetch(const T *p, int vec, int n) {
    constexpr int V = Of<T>::V;
    if (kVec || (vec && n == V)) return *reinterpret_cast<const uint4 *>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j < n) {
            if constexpr (V == 4) w[j] = reinterpret_cast<const uint32_t *>(p)[j];
            else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[j] << (16 * (j & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool kVec, typename T>
__device__ __forceinline__ void put(T *p, const uint4 &u, int vec, int n) {
    constexpr int V = Of<T>::V;
    if (kVec || (vec && n == V)) {
        *reinterpret_cast<uint4 *>(p) = u;
        return;
    }
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j < n) {
            if constexpr (V == 4) reinterpret_cast<uint32_t *>(p)[j] = w[j];
            else reinterpret_cast<uint16_t *>(p)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        }
}

// A thread's items one after the other, the last one first if kDown; those to come are on their way to shared memory of its own, kDeep of them.  next() gives an item, done() says
// that it has been used.  (Backward of 112 x 112 x 96, 32 images: with items fetched to registers, four at a time, 91 us instead of 75; forward of 224 x 224 x 64 the same 117.)
template <int kDeep>
struct Ahead {
    int head = 0, tail = 0;
    __device__ __forceinline__ int in() { return head++ & (kDeep - 1); }
    __device__ __forceinline__ int out() { return tail++ & (kDeep - 1); }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    static __device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 1) : "memory"); }
};
constexpr int kDeepX = 8, kDeepDy = 4;
constexpr int kRing = kThreads * kDeepX * 16;                // bytes; backward, items of up to 32 bytes: as many
static_assert(kDeepX * 16 == kDeepDy * 32, "");

// Where V channels of a column are in the 8-bit form, and the four bytes of their block's exponent.
__device__ __forceinline__ int64_t codes_at(const Norm &q, int64_t col, int ch) {
    const int c = ch & 127;
    return (int64_t)(ch >> 7) * q.groups8 * 1024 + col * 128 + ((((c >> 4) ^ (int)col) & 7) << 4) + (c & 15);
}
__device__ __forceinline__ int64_t scale_at(const Norm &q, int64_t col, int ch) {
    return (int64_t)q.scale_off + ((int64_t)(ch >> 7) * q.chunks8 + (col >> 7)) * kScales8 + (col & 31) * 16 + (col >> 5 & 3) * 4;
}
// The values of V channels (0 behind the last channel) to 8 bits; the 128 / V threads of a block are neighbours in a warp and all call this.
template <int V>
__device__ __forceinline__ void hold(const Norm &q, uint8_t *to, const uint64_t (&pairs)[V / 2], int64_t col, int ch) {
    float f[V], top = 0.f;
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        const float2 v = f32x2_halves(pairs[j / 2]);
        f[j] = v.x; f[j + 1] = v.y;
        top = max_nan(top, max_nan(fabsf(v.x), fabsf(v.y)));
    }
    if (!(top < INFINITY)) {                                             // what is not finite becomes NaN and leaves the scale alone
        top = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (fabsf(f[j]) < INFINITY) top = fmaxf(top, fabsf(f[j]));
            else f[j] = NAN;
        }
    }
    uint32_t bits = __float_as_uint(top);
    const uint32_t peers = V == 4 ? 0xFFFFFFFFu : 0xFFFFu << (threadIdx.x & 16);
#pragma unroll
    for (int d = 64 / V; d; d >>= 1) bits = max(bits, __shfl_xor_sync(peers, bits, d));
    const uint32_t e = (uint32_t)max((int)((bits + (0x7FFFFFu - 0x600000u)) >> 23) - 8, 1);
    const float down = power_of(254u - e);
    uint32_t codes[V / 4];
#pragma unroll
    for (int j = 0; j < V; j += 4)
        codes[j / 4] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[j] * down, f[j + 1] * down), __NV_SATFINITE, __NV_E4M3) |
                       (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[j + 2] * down, f[j + 3] * down), __NV_SATFINITE, __NV_E4M3) << 16;
    uint8_t *at = to + codes_at(q, col, ch);
    if constexpr (V == 8) *reinterpret_cast<uint2 *>(at) = make_uint2(codes[0], codes[1]);
    else *reinterpret_cast<uint32_t *>(at) = codes[0];
    if ((ch & 127) == 0) *reinterpret_cast<uint32_t *>(to + scale_at(q, col, ch)) = e * 0x01010101u;
}

// (a product instead of a division of some twenty instructions)
__device__ __forceinline__ int group_of(const Norm &q, int channel) {
    return q.cpg_magic ? (int)__umulhi((uint32_t)channel, q.cpg_magic) : channel / q.cpg;
}

// A CTA's place: sample, first channel, channels, groups that it meets, pixels.
struct Place {
    int n, slice, rank, c0, width, g0, ng, px0, px1;
    __device__ __forceinline__ Place(const Norm &q, uint32_t cta) {
        const uint32_t u = cta / (uint32_t)q.ranks;
        rank = (int)(cta - u * (uint32_t)q.ranks);
        n = (int)(u / (uint32_t)q.slices);
        slice = (int)(u - (uint32_t)n * (uint32_t)q.slices);
        c0 = slice * q.width; width = min(q.width, q.channels - c0);
        g0 = group_of(q, c0); ng = group_of(q, c0 + width - 1) + 1 - g0;
        px0 = min(rank * q.per, q.pixels); px1 = min(px0 + q.per, q.pixels);
    }
};
// A thread's place in it: its pixel lane, channels, items and first row.
template <typename T>
struct Mine {
    int lane, v, ch, n, items;
    int64_t row0;
    __device__ __forceinline__ Mine(const Norm &q, const Place &at) {
        constexpr int V = Of<T>::V;
        lane = (int)((uint32_t)threadIdx.x / (uint32_t)q.cv); v = (int)threadIdx.x - lane * q.cv;
        ch = at.c0 + v * V;
        n = lane < q.lanes ? max(0, min(V, at.c0 + at.width - ch)) : 0;
        const bool last = at.rank + 1 == q.ranks;
        items = lane < q.lanes ? (last ? q.some_last : q.some) + (lane < (last ? q.more_last : q.more)) : 0;
        row0 = (int64_t)at.n * q.pixels + at.px0 + lane;
    }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// How many neighbouring lanes share a group when `groups` of them are gone through (a power of two), and a sum over them.
__device__ __forceinline__ int sharers(int groups) {
    int k = 32;
    while (k > 1 && groups * k > kThreads) k >>= 1;
    return k;
}
__device__ __forceinline__ float shared_sum(float v, int k) {
    for (int d = k >> 1; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// A group's channels inside the slice, from its first one on.
struct Span { int lo, hi; };
__device__ __forceinline__ Span span_of(const Norm &q, const Place &at, int g) {
    return {max(at.c0, (at.g0 + g) * q.cpg) - at.c0, min(at.c0 + at.width, (at.g0 + g + 1) * q.cpg) - at.c0};
}
// Large calls: where the CTA's pair of group g goes.
__device__ __forceinline__ float2 *partial_at(const Norm &q, const Place &at, int g) {
    const int64_t group = at.g0 + g;
    return q.partial + (((int64_t)at.n * q.groups + group) * q.ranks + at.rank) * q.parts + (at.slice - (int)(group * q.cpg / q.width));
}
// combine(group, k, lane, count, read, weight) for `ng` groups of sample n from g0 on, by k neighbouring lanes each (all lanes of a warp call it together, the last groups
// more than once); read(i) is the i-th CTA's pair of the group, weight(i) the number of values that it stands for.
template <typename R, typename F>
__device__ __forceinline__ void of_groups(int ng, R reader, F combine) {
    const int k = sharers(ng), lane = threadIdx.x & (k - 1);
    for (int g0 = 0; g0 < ng; g0 += kThreads / k) {
        const int g = min(g0 + (int)threadIdx.x / k, ng - 1);
        reader(g, [&](int count, auto read, auto weight) { combine(g, k, lane, count, read, weight); });
    }
    __syncwarp();
}
// Small calls, in a cluster: `own` [ng] in the CTAs' shared memory.
template <typename F>
__device__ __forceinline__ void of_cluster(const Norm &q, const Place &at, const float2 *own, F combine) {
    cluster_arrive();
    cluster_wait();
    of_groups(at.ng, [&](int g, auto call) {
        const uint32_t mine = smem_at(own + g);
        call(q.ranks,
             [&](int i) {
                 const uint32_t a = peer_address(mine, (uint32_t)i);
                 return make_float2(__uint_as_float(lds32_peer(a)), __uint_as_float(lds32_peer(a + 4)));
             },
             [&](int i) { return (float)(min((i + 1) * q.per, q.pixels) - i * q.per) * (float)q.cpg; });
    }, combine);
    cluster_arrive();                                        // (its wait is at the kernel's end: no CTA leaves while others read from it)
    __syncthreads();
}
// Large calls: out of `partial`.
template <typename F>
__device__ __forceinline__ void of_memory(const Norm &q, const Place &at, F combine) {
    const float full = (float)q.per * (float)q.cpg, rest = (float)(q.pixels - (q.ranks - 1) * q.per) * (float)q.cpg;
    of_groups(at.ng, [&](int g, auto call) {
        const int64_t group = at.g0 + g, from = group * q.cpg, to = from + q.cpg;
        const float2 *row = q.partial + ((int64_t)at.n * q.groups + group) * q.ranks * q.parts;
        if (q.parts == 1) {
            call(q.ranks, [&](int i) { return row[i]; }, [&](int i) { return i + 1 < q.ranks ? full : rest; });
            return;
        }
        const int s0 = (int)(from / q.width), parts = (int)((to - 1) / q.width) + 1 - s0;
        call(q.ranks * parts,
             [&](int i) { const int r = i / parts; return row[r * q.parts + i - r * parts]; },
             [&](int i) {
                 const int r = i / parts;
                 const int64_t s = s0 + i - r * parts;
                 return (r + 1 < q.ranks ? full : rest) / (float)q.cpg * (float)(min(to, (s + 1) * q.width) - max(from, s * q.width));
             });
    }, combine);
    __syncthreads();
}

// How a call is cut (norm_forward.cu).
struct Plan {
    bool cluster;                        // a small call
    int width, slices, ranks, per, cv, parts;
    int resident, fixed_smem;            // items a thread keeps, bytes in front of them
    int64_t tiles;
};
template <auto kernel, size_t kSmem>
cudaError_t allow() {                                                        // (once a kernel and device)
    static std::atomic<uint64_t> ready{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device < 64 && ready.load(std::memory_order_relaxed) >> device & 1) return cudaSuccess;
    e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && device < 64) ready.fetch_or(1ull << device, std::memory_order_relaxed);
    return e;
}
template <auto small, auto sum, auto finish>
cudaError_t run(const Plan &p, const Norm &q, int item, cudaStream_t st) {
    if (p.tiles > 0x7FFFFFFFll) return cudaErrorInvalidValue;
    const size_t smem = p.fixed_smem + (size_t)p.resident * kThreads * item;
    if (p.cluster) {
        const cudaError_t e = allow<small, kMaxSmem>();
        return e != cudaSuccess ? e : launch_clusters(small, (unsigned)p.tiles, kThreads, smem, st, (unsigned)q.ranks, q);
    }
    cudaError_t e = allow<sum, kRing>();
    if (e == cudaSuccess) e = allow<finish, kRing + (kThreads * 8 + 2) * 8>();
    if (e == cudaSuccess) e = launch_chained(sum, (unsigned)p.tiles, kThreads, kRing, st, q);
    return e != cudaSuccess ? e : launch_chained(finish, (unsigned)p.tiles, kThreads, smem, st, q);
}

// The backward pass of each type (norm_backward_*.cu; all of its variants together take some two minutes to compile).
cudaError_t backward_bf16(const Plan &p, const Norm &q, bool one, bool vec, bool from8, cudaStream_t st);
cudaError_t backward_fp16(const Plan &p, const Norm &q, bool one, bool vec, bool from8, cudaStream_t st);
cudaError_t backward_fp32(const Plan &p, const Norm &q, bool one, bool vec, bool from8, cudaStream_t st);

}  // namespace norm
}  // namespace crisp
