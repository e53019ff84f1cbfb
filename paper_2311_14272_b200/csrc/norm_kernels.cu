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
//   large ones    two kernels of as many CTAs as fit, each with its part of the pixels.  The second goes over them backwards: what the first read last is still in L2
//
// A thread holds V = 16 bytes' worth of consecutive channels and goes over pixels, two channels an instruction: per pair p = a x + b (a = gamma rstd, b = beta - mean a),
// dx = a e + B x + C.  Forward sums are about the thread's first value, so that a mean far from zero costs no digits; then mean = sum n_i mean_i / n and
// M2 = sum M2_i + n_i (mean_i - mean)^2 over threads and over CTAs, always in the same order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "block8.h"
#include "block8.cuh"
#include "mask_common.cuh"

namespace crisp {

using namespace block8;

namespace {

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
    int whole8;                          // slices are whole blocks of 128 channels
    int act, vec, vec_dy, vec_out;       // vec: addresses and pitches allow 16 bytes at once
    int stream;                          // the results are not kept in L2 at the cost of what is still to be read
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
__device__ __forceinline__ void put(T *p, const uint4 &u, int vec, int n, int stream) {
    constexpr int V = Of<T>::V;
    if (kVec || (vec && n == V)) {
        if (stream) __stcs(reinterpret_cast<uint4 *>(p), u);
        else *reinterpret_cast<uint4 *>(p) = u;
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
// that it has been used.  (Bound by how much is on its way: with four items at a time in registers 224 x 224 x 64, 32 images, took 117 us, whatever was in L2.)
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

// ---------------------------------------------------------------------------------------------------------------- forward

// The thread's items of x out of memory, or (Kept) out of what it has kept.
template <typename T, bool kVec, bool kDown>
struct StreamX : Ahead<kDeepX> {
    uint4 *slots;
    const T *p;
    int64_t step;
    int left, n, vec;
    __device__ __forceinline__ StreamX(const Norm &q, const Mine<T> &me, uint4 *smem) : slots(smem + threadIdx.x), n(me.n), vec(q.vec) {
        step = (int64_t)q.lanes * q.ldx;
        left = n > 0 ? me.items : 0;
        p = reinterpret_cast<const T *>(q.x) + me.row0 * q.ldx + me.ch;
        if (kDown) { p += (me.items - 1) * step; step = -step; }
        if constexpr (kVec)
            for (int i = 0; i < kDeepX; ++i) done();
    }
    __device__ __forceinline__ uint4 next() {
        if constexpr (kVec) {
            arrived();
            return slots[out() * kThreads];
        } else {
            const uint4 u = fetch<false>(p, vec, n);
            p += step;
            return u;
        }
    }
    __device__ __forceinline__ void done() {
        if constexpr (kVec) {
            if (left > 0) { copy_async<16>(slots + in() * kThreads, p); p += step; --left; }
            commit();
        }
    }
};
struct KeptX {
    const uint4 *slot;
    __device__ __forceinline__ uint4 next() { const uint4 u = *slot; slot += kThreads; return u; }
    __device__ __forceinline__ void done() {}
};

// Pairs (mean, M2) of the CTA's groups to give(g, pair).
template <typename T, bool kOne, bool kOver, typename I, typename F>
__device__ __forceinline__ void sum_x(const Norm &q, const Place &at, const Mine<T> &me, float2 *threads, I &items, F give) {
    constexpr int V = Of<T>::V, P = V / 2;
    uint64_t away[kOne ? 1 : P], s1[P], s2[P];               // away: less the thread's first values (kOne: its very first)
#pragma unroll
    for (int j = 0; j < P; ++j) s1[j] = s2[j] = 0;
#pragma unroll
    for (int j = 0; j < (kOne ? 1 : P); ++j) away[j] = 0;
    if (me.n > 0 && me.items > 0) {
        uint64_t f[P];
        uint4 u = items.next();
        Of<T>::open(u, f);
#pragma unroll
        for (int j = 0; j < (kOne ? 1 : P); ++j) { const float2 v = f32x2_halves(f[j]); away[j] = f32x2(-v.x, kOne ? -v.x : -v.y); }
#pragma unroll 2
        for (int i = 0;;) {
            Of<T>::open(u, f);
#pragma unroll
            for (int j = 0; j < P; ++j) { const uint64_t d = add2(f[j], away[kOne ? 0 : j]); s1[j] = add2(s1[j], d); s2[j] = fma2(d, d, s2[j]); }
            items.done();
            if (++i >= me.items) break;
            u = items.next();
        }
    }
    if constexpr (kOver) __syncthreads();                    // (what follows lies over what the threads had on its way)
    const float count = (float)me.items;
    if constexpr (kOne) {                                    // (mean, M2) of the thread
        const float one = f32x2_sum(P == 4 ? add2(add2(s1[0], s1[1]), add2(s1[P - 2], s1[P - 1])) : add2(s1[0], s1[1]));
        const float two = f32x2_sum(P == 4 ? add2(add2(s2[0], s2[1]), add2(s2[P - 2], s2[P - 1])) : add2(s2[0], s2[1]));
        const float d = me.items ? one / (count * V) : 0.f;
        threads[threadIdx.x] = make_float2(d - f32x2_halves(away[0]).x, max_nan(0.f, fmaf(-one, d, two)));
    } else {                                                 // of each channel
        const float over = me.items ? 1.f / count : 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float2 a = f32x2_halves(away[j / 2]), b = f32x2_halves(s1[j / 2]), c = f32x2_halves(s2[j / 2]);
            const float first = j & 1 ? -a.y : -a.x, one = j & 1 ? b.y : b.x, two = j & 1 ? c.y : c.x, d = one * over;
            threads[threadIdx.x * V + j] = make_float2(first + d, max_nan(0.f, fmaf(-one, d, two)));
        }
    }
    __syncthreads();
    const int pixels = at.px1 - at.px0, k = sharers(at.ng), lane = threadIdx.x & (k - 1);
    const bool is_last = at.rank + 1 == q.ranks;
    const int some = is_last ? q.some_last : q.some, one_more = is_last ? q.more_last : q.more;
    for (int g0 = 0; g0 < at.ng; g0 += kThreads / k) {
        const int g = g0 + threadIdx.x / k;
        const Span in = span_of(q, at, min(g, at.ng - 1));
        const int wide = in.hi - in.lo, across = kOne ? (wide + V - 1) / V : wide, entries = across * q.lanes;       // entries of a group: `across` a lane
        const float total = (float)pixels * (float)wide;
        const bool as_all = wide == q.cpg;
        const auto entry = [&](int i, float *weight) {
            // (a product instead of a division: exact for i below 2^16, which entries are)
            const int l = across == 1 ? i : as_all ? (int)__umulhi((uint32_t)i, q.across_magic) : i / across, a = i - l * across;
            const float here = (float)(l < one_more ? some + 1 : some);
            *weight = kOne ? here * V : here;
            return threads[kOne ? l * q.cv + in.lo / V + a : l * q.cv * V + in.lo + a];
        };
        // (about the first entry's mean, for the same reason as above)
        const float base = threads[kOne ? in.lo / V : in.lo].x;
        float w, sum = 0.f, rest = 0.f;
        for (int i = lane; i < entries; i += k) { const float2 e = entry(i, &w); sum += w > 0.f ? w * (e.x - base) : 0.f; }
        const float m = base + (total > 0.f ? shared_sum(sum, k) / total : 0.f);
        for (int i = lane; i < entries; i += k) { const float2 e = entry(i, &w); rest += w > 0.f ? e.y + w * (e.x - m) * (e.x - m) : 0.f; }
        rest = shared_sum(rest, k);
        if (lane == 0 && g < at.ng) give(g, make_float2(m, rest));
    }
}
// Mean and rstd out of the CTAs' pairs, to the k lanes; in 64 bits about the first one's mean, so that one pass does.
template <typename R, typename W>
__device__ __forceinline__ float2 combine_x(const Norm &q, int k, int lane, int count, R read, W weight) {
    const float base = read(0).x;
    double sum = 0.0, rest = 0.0;
#pragma unroll 8
    for (int i = lane; i < count; i += k) {
        const float2 e = read(i);
        const double w = weight(i), d = (double)e.x - (double)base;
        sum += w * d;
        rest += e.y + w * d * d;
    }
    for (int d = k >> 1; d; d >>= 1) { sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d); rest += __shfl_xor_sync(0xFFFFFFFFu, rest, d); }
    const double all = (double)q.pixels * (double)q.cpg, off = sum / all;
    return make_float2((float)((double)base + off), 1.f / sqrtf((float)((rest - sum * off) / all) + q.eps));
}

template <int kAct, typename T>
__device__ __forceinline__ uint64_t activate(uint64_t p) {   // (NaN stays)
    const float2 v = f32x2_halves(p);
    if constexpr (kAct == kRelu) return f32x2(max_nan(v.x, 0.f), max_nan(v.y, 0.f));
    if constexpr (kAct == kRelu6) {
        float a = max_nan(v.x, 0.f), b = max_nan(v.y, 0.f);
        return f32x2(a > 6.f ? 6.f : a, b > 6.f ? 6.f : b);
    }
    if constexpr (kAct == kSilu) return mul2(p, Of<T>::sigmoid2(p));
    return p;
}

// y, and the 8-bit forms, of the CTA's pixels (kDown: the last one first); known(g): the statistics of the sample's group g.
template <typename T, bool kVec, bool kHold, bool kDown, typename I, typename F>
__device__ __forceinline__ void finish_y(const Norm &q, const Mine<T> &me, I &items, F known) {
    constexpr int V = Of<T>::V, P = V / 2;
    // (threads behind the last channel write the zeros that its block ends with; not of a block in which there is none)
    if (me.lane >= q.lanes || !(me.n > 0 || (kHold && (me.ch & ~127) < q.channels))) return;
    uint64_t a[P], b[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
        float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = me.ch + 2 * j + i;
            if ((kVec && !kHold) || 2 * j + i < me.n) {
                const float2 k = known(group_of(q, c));
                s[i] = k.y * (q.gamma ? q.gamma[c] : 1.f);
                t[i] = fmaf(-k.x, s[i], q.beta ? q.beta[c] : 0.f);
            }
        }
        a[j] = f32x2(s[0], s[1]); b[j] = f32x2(t[0], t[1]);
    }
    T *y = reinterpret_cast<T *>(q.out) + me.row0 * q.ld_out + me.ch;
    const int64_t step_y = (int64_t)q.lanes * q.ld_out;
    const auto finish = [&](auto act) {
        const int64_t skip = kDown ? me.items - 1 : 0, move = kDown ? -step_y : step_y;
        int64_t col = me.row0 + skip * q.lanes;
        y += skip * step_y;
#pragma unroll 2
        for (int i = 0; i < me.items; ++i) {
            uint64_t f[P];
            Of<T>::open(!kHold || me.n > 0 ? items.next() : make_uint4(0, 0, 0, 0), f);
            if constexpr (kHold) if (q.x8) hold<V>(q, q.x8, f, col, me.ch);
#pragma unroll
            for (int j = 0; j < P; ++j) f[j] = activate<decltype(act)::value, T>(fma2(f[j], a[j], b[j]));      // (0 behind the last channel: a = b = 0)
            if constexpr (kHold) if (q.y8) hold<V>(q, q.y8, f, col, me.ch);
            items.done();
            if (!kHold || (q.out && me.n > 0)) put<kVec && !kHold>(y, Of<T>::close(f), q.vec_out, me.n, q.stream);
            y += move;
            col += kDown ? -q.lanes : q.lanes;
        }
    };
    switch (q.act) {
        case kRelu: finish(std::integral_constant<int, kRelu>()); break;
        case kRelu6: finish(std::integral_constant<int, kRelu6>()); break;
        case kSilu: finish(std::integral_constant<int, kSilu>()); break;
        default: finish(std::integral_constant<int, kNone>());
    }
}

// kOne: a thread's channels are of one group.  kVec: every thread's V channels are there, at multiples of 16 bytes.  kHold: an 8-bit form is written.
template <typename T, bool kOne, bool kVec, bool kHold>
__global__ void __launch_bounds__(kThreads, kForwardCtas)
norm_kernel(const __grid_constant__ Norm q) {
    constexpr int V = Of<T>::V;
    extern __shared__ __align__(16) uint8_t smem[];
    wait_for_prerequisites();
    const int most = q.width / q.cpg + 2;                                                // groups that a slice meets, at most
    float2 *groups = reinterpret_cast<float2 *>(smem), *known = groups + most;           // of this CTA, of all
    float2 *threads = known + most;                                                      // [kThreads] or [kThreads][V]
    uint4 *kept = reinterpret_cast<uint4 *>(smem + ((2 * most * 8 + kThreads * (kOne ? 1 : V) * 8 + 15) & ~15)) + threadIdx.x;
    const Place at(q, blockIdx.x);
    const Mine<T> me(q, at);
    if (me.n > 0) {
        const T *x = reinterpret_cast<const T *>(q.x) + me.row0 * q.ldx + me.ch;
        const int64_t step = (int64_t)q.lanes * q.ldx;
        if (kVec || (q.vec && me.n == V)) {
            for (int i = 0; i < me.items; ++i) copy_async<16>(kept + i * kThreads, x + i * step);
            copies_done();
        } else {
            for (int i = 0; i < me.items; ++i) kept[i * kThreads] = fetch<false>(x + i * step, q.vec, me.n);
        }
    }
    KeptX again{kept}, items{kept};
    sum_x<T, kOne, false>(q, at, me, threads, items, [&](int g, float2 pair) { groups[g] = pair; });
    __syncthreads();
    of_cluster(q, at, groups, [&](int g, int k, int lane, int count, auto read, auto weight) {
        const float2 s = combine_x(q, k, lane, count, read, weight);
        if (lane == 0) {
            known[g] = s;
            if (at.rank == 0) *reinterpret_cast<float2 *>(q.stats + 2 * ((int64_t)at.n * q.groups + at.g0 + g)) = s;
        }
    });
    finish_y<T, kVec, kHold, false>(q, me, again, [&](int g) { return known[g - at.g0]; });
    __syncwarp();
    cluster_wait();
}

// The two of a large call.
template <typename T, bool kOne, bool kVec>
__global__ void __launch_bounds__(kThreads, kForwardCtas)
norm_sum_kernel(const __grid_constant__ Norm q) {
    extern __shared__ __align__(16) uint8_t smem[];
    wait_for_prerequisites();
    const Place at(q, blockIdx.x);
    const Mine<T> me(q, at);
    StreamX<T, kVec, false> items(q, me, reinterpret_cast<uint4 *>(smem));
    sum_x<T, kOne, true>(q, at, me, reinterpret_cast<float2 *>(smem), items, [&](int g, float2 pair) { *partial_at(q, at, g) = pair; });
}
template <typename T, bool kVec, bool kHold>
__global__ void __launch_bounds__(kThreads, kForwardCtas)
norm_finish_kernel(const __grid_constant__ Norm q) {
    extern __shared__ __align__(16) uint8_t smem[];
    float2 *known = reinterpret_cast<float2 *>(smem + kRing);
    wait_for_prerequisites();
    const Place at(q, gridDim.x - 1 - blockIdx.x);
    const Mine<T> me(q, at);
    StreamX<T, kVec, true> items(q, me, reinterpret_cast<uint4 *>(smem));
    of_memory(q, at, [&](int g, int k, int lane, int count, auto read, auto weight) {
        const float2 s = combine_x(q, k, lane, count, read, weight);
        if (lane == 0) {
            known[g] = s;
            if (at.rank == 0 && (at.g0 + g) * q.cpg >= at.c0) *reinterpret_cast<float2 *>(q.stats + 2 * ((int64_t)at.n * q.groups + at.g0 + g)) = s;
        }
    });
    finish_y<T, kVec, kHold, true>(q, me, items, [&](int g) { return known[g - at.g0]; });
}

// --------------------------------------------------------------------------------------------------------------- backward

template <int V>
__device__ __forceinline__ void decode(uint32_t lo, uint32_t hi, uint32_t e, uint64_t (&f)[V / 2]) {
    const uint64_t up = both(power_of(e));
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((j < 2 ? lo : hi) >> (16 * (j & 1))), __NV_E4M3)));
        f[j] = mul2(f32x2(v.x, v.y), up);
    }
}

// A thread's coefficients of p = a x + b, and how near to a border of relu or relu6 p may be off.
template <int P>
struct Affine {
    uint64_t a[P], b[P];
    float near;
};
// Which side of the borders p lies on, from the formula in 64 bits: -1, 1 or 7.
__device__ __noinline__ float side_of(const Norm &q, int64_t stat, int c, float x) {
    const double exact = ((double)x - (double)q.stats[2 * stat]) * (double)q.stats[2 * stat + 1] * (q.gamma ? (double)q.gamma[c] : 1.0) + (q.beta ? (double)q.beta[c] : 0.0);
    return exact > 0.0 ? (exact >= 6.0 ? 7.f : 1.f) : -1.f;
}
// e = dy act'(p).  Where p is within its roundings of a border, its side is taken from 64 bits, so that it is the formula's: one element on the wrong side would be
// wrong by all of its dy.
template <int kAct, typename T, int P>
__device__ __forceinline__ void slope(const Norm &q, int n, int ch, const Affine<P> &k, const uint64_t (&x)[P], uint64_t (&dy)[P]) {
    if constexpr (kAct == kNone) return;
    if constexpr (kAct == kSilu) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const uint64_t p = fma2(x[j], k.a[j], k.b[j]);
            const uint64_t s = Of<T>::sigmoid2(p), rest = fma2(s, both(-1.f), both(1.f));
            dy[j] = mul2(dy[j], mul2(s, fma2(p, rest, both(1.f))));
        }
    } else {
        float p[2 * P], least = INFINITY;                     // (three values a minimum)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float2 v = f32x2_halves(fma2(x[j], k.a[j], k.b[j]));
            p[2 * j] = v.x; p[2 * j + 1] = v.y;
            least = fminf(fminf(fabsf(v.x), fabsf(v.y)), least);
            if constexpr (kAct == kRelu6) least = fminf(fminf(fabsf(v.x - 6.f), fabsf(v.y - 6.f)), least);
        }
        if (least < k.near) {
#pragma unroll
            for (int j = 0; j < 2 * P; ++j) {
                if (ch + j >= q.channels) break;
                if (fabsf(p[j]) < k.near || (kAct == kRelu6 && fabsf(p[j] - 6.f) < k.near)) {
                    const float2 v = f32x2_halves(x[j / 2]);
                    p[j] = side_of(q, (int64_t)n * q.groups + (ch + j) / q.cpg, ch + j, j & 1 ? v.y : v.x);
                    if (kAct == kRelu && p[j] > 1.f) p[j] = 1.f;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float2 d = f32x2_halves(dy[j]);
            const bool lo = p[2 * j] > 0.f && (kAct == kRelu || p[2 * j] < 6.f), hi = p[2 * j + 1] > 0.f && (kAct == kRelu || p[2 * j + 1] < 6.f);
            dy[j] = f32x2(lo ? d.x : 0.f, hi ? d.y : 0.f);
        }
    }
}

template <typename T, bool kOne>
__device__ __forceinline__ void affine_of(const Norm &q, const Place &at, const Mine<T> &me, Affine<Of<T>::V / 2> *k, float (&mean)[kOne ? 1 : Of<T>::V],
                                          float (&rstd)[kOne ? 1 : Of<T>::V]) {
    constexpr int V = Of<T>::V;
    k->near = 0.f;
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        float a[2] = {0.f, 0.f}, b[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = me.ch + j + i, m = kOne ? 0 : j + i;
            if (!kOne || j + i == 0) mean[m] = rstd[m] = 0.f;
            if (j + i >= me.n) continue;
            if (!kOne || j + i == 0) {
                const float2 s = *reinterpret_cast<const float2 *>(q.stats + 2 * ((int64_t)at.n * q.groups + group_of(q, c)));
                mean[m] = s.x; rstd[m] = s.y;
            }
            const float beta = q.beta ? q.beta[c] : 0.f;
            a[i] = rstd[m] * (q.gamma ? q.gamma[c] : 1.f);
            b[i] = fmaf(-mean[m], a[i], beta);
            // a and b are off by u of a x, of mean a and of b, p by one more of its own (u = 2^-24); at a border |a x| <= |b| + 6
            k->near = fmaxf(k->near, (fabsf(beta) + 2.f * fabsf(mean[m] * a[i]) + 2.f * fabsf(b[i]) + 16.f) * 0x1p-22f);
        }
        k->a[j / 2] = f32x2(a[0], a[1]); k->b[j / 2] = f32x2(b[0], b[1]);
    }
}

struct Item { uint4 dy, x; };                                // x: 16 bytes, or codes and exponent

template <typename T, bool k8, bool kVec>
struct Reader {
    static constexpr int V = Of<T>::V;
    const Norm &q;
    const Mine<T> &me;
    const T *x, *dy;
    int64_t step_x, step_dy;
    // Where a thread keeps an item's codes: in the order that they have in memory (swizzled by the column) where its block's threads are all there, so that a copy of half a warp goes
    // to one line as it comes from one (else 53 wavefronts an item, not 14: backward of 56 x 56 x 256 from 8 bits, 32 images, 58 us).
    __device__ __forceinline__ int place(int64_t col) const {
        const int c = me.ch & 127;
        return q.whole8 ? (int)(threadIdx.x & ~(128 / V - 1)) * V + ((((c >> 4) ^ (int)col) & 7) << 4) + (c & 15) : (int)threadIdx.x * V;
    }
    __device__ __forceinline__ Reader(const Norm &q_, const Mine<T> &me_)
        : q(q_), me(me_), x(reinterpret_cast<const T *>(q_.x) + me_.row0 * q_.ldx + me_.ch), dy(reinterpret_cast<const T *>(q_.dy) + me_.row0 * q_.ld_dy + me_.ch),
          step_x((int64_t)q_.lanes * q_.ldx), step_dy((int64_t)q_.lanes * q_.ld_dy) {}
    __device__ __forceinline__ Item operator()(int i) const {
        Item r;
        r.dy = fetch<kVec>(dy + i * step_dy, q.vec_dy, me.n);
        if constexpr (k8) {
            const int64_t col = me.row0 + (int64_t)i * q.lanes;
            const uint8_t *p = q.from8 + codes_at(q, col, me.ch);
            if constexpr (V == 8) { const uint2 c = *reinterpret_cast<const uint2 *>(p); r.x.x = c.x; r.x.y = c.y; }
            else { r.x.x = *reinterpret_cast<const uint32_t *>(p); r.x.y = 0; }
            r.x.z = *(q.from8 + scale_at(q, col, me.ch));
            r.x.w = 0;
        } else {
            r.x = fetch<kVec>(x + i * step_x, q.vec, me.n);
        }
        return r;
    }
    static __device__ __forceinline__ void open(const Item &r, uint64_t (&d)[V / 2], uint64_t (&f)[V / 2]) {
        Of<T>::open(r.dy, d);
        if constexpr (k8) decode<V>(r.x.x, r.x.y, r.x.z & 0xFFu, f);
        else Of<T>::open(r.x, f);
    }
};
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case kRelu: f(std::integral_constant<int, kRelu>()); break;
        case kRelu6: f(std::integral_constant<int, kRelu6>()); break;
        case kSilu: f(std::integral_constant<int, kSilu>()); break;
        default: f(std::integral_constant<int, kNone>());
    }
}

// Sums of e and e h of the CTA's channels to q.sums, and of its groups (times gamma) to give(g, pair).
template <typename T, bool kOne, bool k8, bool kVec, bool kOver, typename K, typename F>
__device__ __forceinline__ void sum_e(const Norm &q, const Place &at, const Mine<T> &me, float2 *channels, K &items, F give) {
    constexpr int V = Of<T>::V, P = V / 2, M = kOne ? 1 : V;
    Affine<P> k;
    float mean[M], rstd[M];
    affine_of<T, kOne>(q, at, me, &k, mean, rstd);
    uint64_t r[kOne ? 1 : P], s[kOne ? 1 : P], db[P], dg[P]; // h = r x + s
#pragma unroll
    for (int j = 0; j < (kOne ? 1 : P); ++j) {
        const float r0 = rstd[kOne ? 0 : 2 * j], r1 = rstd[kOne ? 0 : 2 * j + 1];
        r[j] = f32x2(r0, r1); s[j] = f32x2(-mean[kOne ? 0 : 2 * j] * r0, -mean[kOne ? 0 : 2 * j + 1] * r1);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) db[j] = dg[j] = 0;
    if (me.n > 0)
        with_act(q.act, [&](auto act) {
#pragma unroll 1
            for (int i = 0; i < me.items; ++i) {
                uint64_t d[P], x[P];
                Reader<T, k8, kVec>::open(items.next(), d, x);
                slope<decltype(act)::value, T, P>(q, at.n, me.ch, k, x, d);
#pragma unroll
                for (int j = 0; j < P; ++j) { db[j] = add2(db[j], d[j]); dg[j] = fma2(d[j], fma2(x[j], r[kOne ? 0 : j], s[kOne ? 0 : j]), dg[j]); }
                items.done();
            }
        });
    if constexpr (kOver) __syncthreads();
    const int row = q.cv * V;
    if (me.lane < q.lanes) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float2 b = f32x2_halves(db[j]), g = f32x2_halves(dg[j]);
            channels[me.lane * row + me.v * V + 2 * j] = make_float2(b.x, g.x);
            channels[me.lane * row + me.v * V + 2 * j + 1] = make_float2(b.y, g.y);
        }
    }
    __syncthreads();
    // of each channel over the lanes: for gamma and beta, and to the first lane's place, times gamma, for the group
    float *sums = q.sums + ((int64_t)at.n * q.ranks + at.rank) * 2 * q.channels;
    for (int c = threadIdx.x; c < at.width; c += kThreads) {
        float2 t = make_float2(0.f, 0.f);
        for (int l = 0; l < q.lanes; ++l) { const float2 u = channels[l * row + c]; t.x += u.x; t.y += u.y; }
        sums[at.c0 + c] = t.x;
        sums[q.channels + at.c0 + c] = t.y;
        const float w = q.gamma ? q.gamma[at.c0 + c] : 1.f;
        channels[c] = make_float2(w * t.x, w * t.y);
    }
    __syncthreads();
    const int k2 = sharers(at.ng), lane = threadIdx.x & (k2 - 1);
    for (int g0 = 0; g0 < at.ng; g0 += kThreads / k2) {
        const int g = g0 + threadIdx.x / k2;
        const Span in = span_of(q, at, min(g, at.ng - 1));
        float2 t = make_float2(0.f, 0.f);
        for (int c = in.lo + lane; c < in.hi; c += k2) { const float2 u = channels[c]; t.x += u.x; t.y += u.y; }
        t.x = shared_sum(t.x, k2); t.y = shared_sum(t.y, k2);
        if (lane == 0 && g < at.ng) give(g, t);
    }
}
template <typename R>
__device__ __forceinline__ float2 combine_e(const Norm &q, int k, int lane, int count, R read) {
    float2 t = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int i = lane; i < count; i += k) { const float2 u = read(i); t.x += u.x; t.y += u.y; }
    const float all = (float)q.pixels * (float)q.cpg;
    return make_float2(shared_sum(t.x, k) / all, shared_sum(t.y, k) / all);
}

// dx of the CTA's pixels (kDown: the last one first); known(g): m1 and m2 of the sample's group g.  dx = rstd (gamma e - m1 - h m2) = a e + B x + C.
template <typename T, bool kOne, bool k8, bool kVec, bool kDown, typename K, typename F>
__device__ __forceinline__ void finish_dx(const Norm &q, const Place &at, const Mine<T> &me, K &items, F known) {
    constexpr int V = Of<T>::V, P = V / 2, M = kOne ? 1 : V;
    if (me.n <= 0) return;
    Affine<P> k;
    float mean[M], rstd[M];
    affine_of<T, kOne>(q, at, me, &k, mean, rstd);
    uint64_t B[kOne ? 1 : P], C[kOne ? 1 : P];
#pragma unroll
    for (int j = 0; j < (kOne ? 1 : P); ++j) {
        float b[2], c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = kOne ? 0 : 2 * j + i;
            const float2 g = m < me.n ? known(group_of(q, me.ch + m)) : make_float2(0.f, 0.f);
            b[i] = -rstd[m] * rstd[m] * g.y;
            c[i] = -fmaf(b[i], mean[m], rstd[m] * g.x);
        }
        B[j] = f32x2(b[0], b[1]); C[j] = f32x2(c[0], c[1]);
    }
    T *dx = reinterpret_cast<T *>(q.out) + me.row0 * q.ld_out + me.ch;
    const int64_t step_out = (int64_t)q.lanes * q.ld_out;
    with_act(q.act, [&](auto act) {
        const int64_t move = kDown ? -step_out : step_out;
        if (kDown) dx += (me.items - 1) * step_out;
#pragma unroll 1
        for (int i = 0; i < me.items; ++i, dx += move) {
            uint64_t d[P], x[P];
            Reader<T, k8, kVec>::open(items.next(), d, x);
            slope<decltype(act)::value, T, P>(q, at.n, me.ch, k, x, d);
#pragma unroll
            for (int j = 0; j < P; ++j) d[j] = fma2(d[j], k.a[j], fma2(x[j], B[kOne ? 0 : j], C[kOne ? 0 : j]));
            items.done();
            put<kVec>(dx, Of<T>::close(d), q.vec_out, me.n, q.stream);
        }
    });
}

// Where a thread's items are kept: dy, then x; or its codes and the block's exponent.
template <typename T, bool k8, bool kVec>
struct Kept {
    static constexpr int V = Of<T>::V;
    uint4 *dy, *x;
    uint32_t *codes, *e;
    int at = 0;
    __device__ __forceinline__ Item next() { return (*this)(at++); }
    __device__ __forceinline__ void done() {}
    __device__ __forceinline__ Kept(const Norm &q, uint8_t *base)
        : dy(reinterpret_cast<uint4 *>(base) + threadIdx.x), x(dy + q.resident * kThreads),
          codes(reinterpret_cast<uint32_t *>(base + (size_t)q.resident * kThreads * 16) + threadIdx.x * (V / 4)),
          e(reinterpret_cast<uint32_t *>(base + (size_t)q.resident * kThreads * (16 + V)) + threadIdx.x) {}
    __device__ __forceinline__ Item operator()(int i) const {
        Item r;
        r.dy = dy[i * kThreads];
        if constexpr (k8) {
            const uint32_t *c = codes + i * kThreads * (V / 4);
            r.x = make_uint4(c[0], V == 8 ? c[V / 4 - 1] : 0u, e[i * kThreads], 0u);
        } else {
            r.x = x[i * kThreads];
        }
        return r;
    }
    __device__ __forceinline__ void fill(const Norm &q, const Mine<T> &me) const {
        if (me.n <= 0) return;
        const Reader<T, k8, kVec> read(q, me);
        if (kVec || (q.vec_dy && (k8 || q.vec) && me.n == V)) {
            for (int i = 0; i < me.items; ++i) {
                copy_async<16>(dy + i * kThreads, read.dy + i * read.step_dy);
                if constexpr (k8) {
                    const int64_t col = me.row0 + (int64_t)i * q.lanes;
                    copy_async<V>(codes + i * kThreads * (V / 4), q.from8 + codes_at(q, col, me.ch));
                    copy_async<4>(e + i * kThreads, q.from8 + scale_at(q, col, me.ch));
                } else {
                    copy_async<16>(x + i * kThreads, read.x + i * read.step_x);
                }
            }
            copies_done();
        } else {
            for (int i = 0; i < me.items; ++i) {
                const Item r = read(i);
                dy[i * kThreads] = r.dy;
                if constexpr (k8) {
                    uint32_t *c = codes + i * kThreads * (V / 4);
                    c[0] = r.x.x;
                    if constexpr (V == 8) c[1] = r.x.y;
                    e[i * kThreads] = r.x.z;
                } else {
                    x[i * kThreads] = r.x;
                }
            }
        }
    }
};

template <typename T, bool kOne, bool k8, bool kVec>
__global__ void __launch_bounds__(kThreads, kBackwardCtas)
norm_back_kernel(const __grid_constant__ Norm q) {
    constexpr int V = Of<T>::V;
    extern __shared__ __align__(16) uint8_t smem[];
    wait_for_prerequisites();
    const int most = q.width / q.cpg + 2;
    float2 *groups = reinterpret_cast<float2 *>(smem), *known = groups + most;
    float2 *channels = known + most;                                         // [lanes][cv * V]: sums of e and of e h
    const Kept<T, k8, kVec> kept(q, smem + ((2 * most * 8 + kThreads * V * 8 + 15) & ~15));
    const Place at(q, blockIdx.x);
    const Mine<T> me(q, at);
    kept.fill(q, me);
    auto items = kept, again = kept;
    sum_e<T, kOne, k8, kVec, false>(q, at, me, channels, items, [&](int g, float2 pair) { groups[g] = pair; });
    __syncthreads();
    of_cluster(q, at, groups, [&](int g, int k, int lane, int count, auto read, auto) {
        const float2 m = combine_e(q, k, lane, count, read);
        if (lane == 0) known[g] = m;
    });
    finish_dx<T, kOne, k8, kVec, false>(q, at, me, again, [&](int g) { return known[g - at.g0]; });
    __syncwarp();
    cluster_wait();
}

// The thread's items out of memory.
template <typename T, bool k8, bool kVec, bool kDown>
struct StreamDy : Ahead<kDeepDy> {
    static constexpr int V = Of<T>::V;
    Reader<T, k8, kVec> read;
    uint4 *dy, *x;
    uint8_t *codes;
    uint32_t *e;
    int64_t col;                                             // of the item that next() gives
    int to_come, at;                                         // items that are not on their way yet, and the next of them (or, not kVec, the next one)
    __device__ __forceinline__ StreamDy(const Norm &q, const Mine<T> &me, uint8_t *smem)
        : read(q, me), dy(reinterpret_cast<uint4 *>(smem) + threadIdx.x), x(dy + kDeepDy * kThreads),
          codes(smem + kDeepDy * kThreads * 16), e(reinterpret_cast<uint32_t *>(smem + kDeepDy * kThreads * (16 + V)) + threadIdx.x) {
        to_come = me.n > 0 ? me.items : 0;
        at = kDown ? me.items - 1 : 0;
        col = me.row0 + (int64_t)at * q.lanes;
        if constexpr (kVec)
            for (int i = 0; i < kDeepDy; ++i) done();
    }
    __device__ __forceinline__ Item next() {
        if constexpr (kVec) {
            arrived();
            const int s = out() * kThreads;
            Item r;
            r.dy = dy[s];
            if constexpr (k8) {
                const uint32_t *c = reinterpret_cast<const uint32_t *>(codes + s * V + read.place(col));
                if constexpr (V == 8) { const uint2 two = *reinterpret_cast<const uint2 *>(c); r.x = make_uint4(two.x, two.y, e[s], 0u); }
                else r.x = make_uint4(c[0], 0u, e[s], 0u);
                col += kDown ? -read.q.lanes : read.q.lanes;
            } else {
                r.x = x[s];
            }
            return r;
        } else {
            const Item r = read(at);
            at += kDown ? -1 : 1;
            return r;
        }
    }
    __device__ __forceinline__ void done() {
        if constexpr (kVec) {
            if (to_come > 0) {
                const int s = in() * kThreads;
                copy_async<16>(dy + s, read.dy + at * read.step_dy);
                if constexpr (k8) {
                    const int64_t there = read.me.row0 + (int64_t)at * read.q.lanes;
                    copy_async<V>(codes + s * V + read.place(there), read.q.from8 + codes_at(read.q, there, read.me.ch));
                    copy_async<4>(e + s, read.q.from8 + scale_at(read.q, there, read.me.ch));
                } else {
                    copy_async<16>(x + s, read.x + at * read.step_x);
                }
                at += kDown ? -1 : 1;
                --to_come;
            }
            commit();
        }
    }
};

template <typename T, bool kOne, bool k8, bool kVec>
__global__ void __launch_bounds__(kThreads, kBackwardCtas)
norm_back_sum_kernel(const __grid_constant__ Norm q) {
    extern __shared__ __align__(16) uint8_t smem[];
    wait_for_prerequisites();
    const Place at(q, blockIdx.x);
    const Mine<T> me(q, at);
    StreamDy<T, k8, kVec, false> items(q, me, smem);
    sum_e<T, kOne, k8, kVec, true>(q, at, me, reinterpret_cast<float2 *>(smem), items, [&](int g, float2 pair) { *partial_at(q, at, g) = pair; });
}
template <typename T, bool kOne, bool k8, bool kVec>
__global__ void __launch_bounds__(kThreads, kBackwardCtas)
norm_back_finish_kernel(const __grid_constant__ Norm q) {
    extern __shared__ __align__(16) uint8_t smem[];
    float2 *known = reinterpret_cast<float2 *>(smem + kRing);
    wait_for_prerequisites();
    const Place at(q, gridDim.x - 1 - blockIdx.x);
    const Mine<T> me(q, at);
    StreamDy<T, k8, kVec, true> items(q, me, smem);
    of_memory(q, at, [&](int g, int k, int lane, int count, auto read, auto) {
        const float2 m = combine_e(q, k, lane, count, read);
        if (lane == 0) known[g] = m;
    });
    finish_dx<T, kOne, k8, kVec, true>(q, at, me, items, [&](int g) { return known[g - at.g0]; });
}

// dbeta and dgamma: the sums of all CTAs' [rows][2][channels], a warp's lanes on 32 neighbouring ones, in one order.
__global__ void __launch_bounds__(1024)
sum_rows_kernel(const float *sums, int64_t rows, int channels, float *dgamma, float *dbeta) {
    __shared__ float part[32][33];
    wait_for_prerequisites();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < 2 * (int64_t)channels) {
#pragma unroll 8
        for (int64_t r = warp; r < rows; r += 32) s += sums[r * 2 * channels + c];
    }
    part[warp][lane] = s;
    __syncthreads();
    s = warp_sum(part[lane][warp]);                                          // (column `warp` of the 32)
    const int64_t mine = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && mine < 2 * (int64_t)channels) {
        if (mine < channels) { if (dbeta) dbeta[mine] = s; }
        else if (dgamma) dgamma[mine - channels] = s;
    }
}

// ------------------------------------------------------------------------------------------------------------------- host

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// How a call is cut.
struct Plan {
    bool cluster;                        // a small call
    int width, slices, ranks, per, cv, parts;
    int resident, fixed_smem;            // items a thread keeps, bytes in front of them
    int64_t tiles;
};
constexpr int kSms = 148;
constexpr int64_t kSmallBytes = 12 << 20;
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

Plan plan_of(const crisp_group_norm_t &d, bool back, bool from8, bool eight) {
    Plan p{};
    const int size = d.dtype == 1 ? 4 : 2, V = 16 / size, C = d.channels, cpg = C / d.groups;
    const int most = kThreads * V, align = eight ? 128 : V;                  // channels that a CTA's threads hold side by side; multiples that slices are of
    const int item = back ? (from8 ? 16 + V + 4 : 32) : 16;
    const int64_t batch = std::max<int64_t>(1, d.batch), bytes = batch * d.pixels * C * item / V;
    int g = cpg, h = align;
    while (h) { const int t = g % h; g = h; h = t; }
    const int unit = (int)std::min<int64_t>((int64_t)(cpg / g) * align, C);  // the narrowest slice of whole groups
    const bool whole = (unit + align - 1) / align * align <= most;
    const auto slice = [&](int width) {
        p.width = std::min(width, C);
        p.slices = (int)ceil_div(C, p.width);
        p.cv = (int)(eight ? ceil_div(p.width, 128) * (128 / V) : ceil_div(p.width, V));
        p.fixed_smem = (2 * (p.width / cpg + 2) * 8 + kThreads * (cpg % V == 0 && C % V == 0 && !back ? 1 : V) * 8 + 15) & ~15;
    };
    const auto rank = [&](int64_t ranks) {
        p.per = (int)ceil_div(d.pixels, std::max<int64_t>(1, std::min<int64_t>(ranks, d.pixels)));
        p.ranks = (int)ceil_div(d.pixels, p.per);
        p.resident = (int)ceil_div(p.per, kThreads / p.cv);
    };
    const auto wanted = [&] { return p.fixed_smem + (size_t)p.resident * kThreads * item; };
    if (whole && bytes <= kSmallBytes) {
        int width = unit;
        while (width < C && width * size < 128 && width + unit <= most) width += unit;
        slice(width);
        // enough CTAs, but two items a thread before a slice is cut further
        rank(std::min<int64_t>(std::min<int64_t>(kMaxCluster, ceil_div(2 * kSms, batch * p.slices)), ceil_div(d.pixels, 2 * (kThreads / p.cv))));
        while (wanted() > kMaxSmem / 2 && p.ranks < kMaxCluster) rank(std::min(kMaxCluster, p.ranks * 2));
        p.cluster = wanted() <= kMaxSmem && p.ranks <= kMaxCluster;
        p.parts = 1;
    }
    if (!p.cluster) {
        slice((int)std::min<int64_t>(ceil_div(C, align) * align, most));
        p.parts = p.slices == 1 ? 1 : (cpg + p.width - 2) / p.width + 1;
        // as many CTAs as run at once; or, where the slices do not go into that, as many as that is filled some times over.  (Every CTA of the second kernel adds the pairs of
        // its sample's: 128 of them at most.)
        const int64_t slices = batch * p.slices, grid = kSms * (back ? kBackwardCtas : kForwardCtas), once = grid / slices;
        const int64_t ranks = once * slices * 20 >= grid * 17 ? once : ceil_div(4 * grid, slices);
        rank(std::min<int64_t>(std::min<int64_t>(ranks, 128), ceil_div(d.pixels, 4 * (kThreads / p.cv))));
        p.resident = 0;
        p.fixed_smem = kRing + (p.width / cpg + 2) * 8;
    }
    p.tiles = batch * p.slices * p.ranks;
    return p;
}

// Workspace: the sums of gamma's and beta's gradients; for large calls the CTAs' pairs.
struct Space { size_t partial, total; };
Space space_of(const crisp_group_norm_t &d, const Plan &p, bool back) {
    Space s{};
    size_t at = 0;
    if (back) at += align_up((size_t)d.batch * p.ranks * 2 * d.channels * sizeof(float));
    s.partial = at;
    if (!p.cluster) at += align_up((size_t)d.batch * d.groups * p.ranks * p.parts * sizeof(float2));
    s.total = at;
    return s;
}

crisp_status_t check(const crisp_group_norm_t *d) {
    if (!d || d->activation < 0 || d->activation > 3 || d->dtype < 0 || d->dtype > 2 || !(d->eps >= 0.0) || !std::isfinite(d->eps)) return CRISP_INVALID_ARG;
    if (d->batch < 0 || d->pixels <= 0 || d->channels <= 0 || d->groups <= 0 || d->channels % d->groups) return CRISP_BAD_SHAPE;
    if (d->pixels > 0x7FFFFFFFll - 65536 || d->batch > 0x7FFFFFFFll / 65536 || d->channels > kMaxBlocksPerRowTile * 128 ||
        (double)d->batch * (double)d->pixels * (double)d->channels > 0x1p44)
        return CRISP_UNSUPPORTED;
    return CRISP_OK;
}

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
template <typename T, bool kOne, bool kVec, bool kHold>
cudaError_t forward(const Plan &p, const Norm &q, cudaStream_t st) {
    return run<norm_kernel<T, kOne, kVec, kHold>, norm_sum_kernel<T, kOne, kVec>, norm_finish_kernel<T, kVec, kHold>>(p, q, 16, st);
}
template <typename T>
cudaError_t forward(const Plan &p, const Norm &q, bool one, bool vec, bool hold, cudaStream_t st) {
    if (one) {
        if (vec) return hold ? forward<T, true, true, true>(p, q, st) : forward<T, true, true, false>(p, q, st);
        return hold ? forward<T, true, false, true>(p, q, st) : forward<T, true, false, false>(p, q, st);
    }
    if (vec) return hold ? forward<T, false, true, true>(p, q, st) : forward<T, false, true, false>(p, q, st);
    return hold ? forward<T, false, false, true>(p, q, st) : forward<T, false, false, false>(p, q, st);
}
template <typename T, bool kOne, bool k8, bool kVec>
cudaError_t backward(const Plan &p, const Norm &q, cudaStream_t st) {
    return run<norm_back_kernel<T, kOne, k8, kVec>, norm_back_sum_kernel<T, kOne, k8, kVec>, norm_back_finish_kernel<T, kOne, k8, kVec>>(
        p, q, k8 ? 16 + Of<T>::V + 4 : 32, st);
}
template <typename T>
cudaError_t backward(const Plan &p, const Norm &q, bool one, bool vec, bool from8, cudaStream_t st) {
    if (!vec) return from8 ? backward<T, false, true, false>(p, q, st) : backward<T, false, false, false>(p, q, st);
    if (one) return from8 ? backward<T, true, true, true>(p, q, st) : backward<T, true, false, true>(p, q, st);
    return from8 ? backward<T, false, true, true>(p, q, st) : backward<T, false, false, true>(p, q, st);
}

int vec_of(const void *p, int64_t ld, int size) { return aligned_to(p, 16) && ld * size % 16 == 0; }

Norm norm_of(const crisp_group_norm_t &d, const Plan &p, const Space &s, void *workspace) {
    Norm q{};
    uint8_t *w = reinterpret_cast<uint8_t *>(workspace);
    q.sums = reinterpret_cast<float *>(w);
    q.partial = reinterpret_cast<float2 *>(w + s.partial);
    q.pixels = (int)d.pixels; q.channels = d.channels; q.groups = d.groups; q.cpg = d.channels / d.groups;
    q.width = p.width; q.slices = p.slices; q.ranks = p.ranks; q.per = p.per; q.parts = p.parts; q.cv = p.cv;
    q.lanes = kThreads / p.cv;
    const int last = q.pixels - (p.ranks - 1) * p.per;
    q.some = p.per / q.lanes; q.more = p.per % q.lanes; q.some_last = last / q.lanes; q.more_last = last % q.lanes;
    q.resident = p.resident;
    q.whole8 = d.channels % 128 == 0 && p.width % 128 == 0;
    if (q.cpg > 1 && (double)d.channels * q.cpg < 4294967296.0) q.cpg_magic = (uint32_t)((((uint64_t)1 << 32) + q.cpg - 1) / q.cpg);
    q.stream = !p.cluster && (double)d.batch * d.pixels * d.channels * (d.dtype == 1 ? 4 : 2) > 64e6;
    q.act = d.activation;
    q.eps = (float)d.eps;
    const Act8 a = act8(d.channels, d.batch * d.pixels);
    q.groups8 = a.groups; q.chunks8 = a.chunks; q.scale_off = a.scale_off;
    return q;
}

}  // namespace

}  // namespace crisp

extern "C" {

using namespace crisp;

crisp_status_t crisp_group_norm_sizes(const crisp_group_norm_t *desc, int32_t backward, size_t *workspace_bytes) {
    const crisp_status_t bad = check(desc);
    if (bad != CRISP_OK) return bad;
    if (!workspace_bytes || (backward != 0 && backward != 1)) return CRISP_INVALID_ARG;
    *workspace_bytes = 0;
    for (int eight = 0; eight < 2; ++eight) {
        const Plan p = plan_of(*desc, backward != 0, backward && eight, !backward && eight);
        const Space s = space_of(*desc, p, backward != 0);
        *workspace_bytes = std::max(*workspace_bytes, s.total);
    }
    return CRISP_OK;
}

crisp_status_t crisp_group_norm(const crisp_group_norm_t *desc, const void *d_x, int64_t ldx, const float *d_gamma, const float *d_beta, void *d_y, int64_t ldy,
                                float *d_stats, void *d_x8, void *d_y8, void *d_workspace, void *stream) {
    const crisp_status_t bad = check(desc);
    if (bad != CRISP_OK) return bad;
    const crisp_group_norm_t &d = *desc;
    if (d.batch == 0) return CRISP_OK;
    const int size = d.dtype == 1 ? 4 : 2;
    if (!d_x || !d_stats || (!d_y && !d_y8) || !aligned_to(d_x, size) || !aligned_to(d_y, size) || !aligned_to(d_gamma, 4) || !aligned_to(d_beta, 4) ||
        !aligned_to(d_stats, 8) || !aligned_to(d_x8, kAlign) || !aligned_to(d_y8, kAlign) || !aligned_to(d_workspace, kAlign))
        return CRISP_INVALID_ARG;
    if (ldx < d.channels || (d_y && ldy < d.channels)) return CRISP_BAD_SHAPE;
    const bool eight = d_x8 || d_y8;
    size_t bytes = 0;
    if (eight && crisp_quantize8_sizes(d.channels, d.batch * d.pixels, &bytes) != CRISP_OK) return CRISP_UNSUPPORTED;
    const Plan p = plan_of(d, false, false, eight);
    const Space s = space_of(d, p, false);
    if (s.total && !d_workspace) return CRISP_INVALID_ARG;
    Norm q = norm_of(d, p, s, d_workspace);
    q.x = d_x; q.ldx = ldx; q.out = d_y; q.ld_out = ldy; q.gamma = d_gamma; q.beta = d_beta; q.stats = d_stats;
    q.x8 = reinterpret_cast<uint8_t *>(d_x8); q.y8 = reinterpret_cast<uint8_t *>(d_y8);
    q.vec = vec_of(d_x, ldx, size); q.vec_out = vec_of(d_y, ldy, size);
    const int V = 16 / size;
    const bool one = q.cpg % V == 0, vec = d.channels % V == 0 && q.vec && q.vec_out;
    const uint32_t across = (uint32_t)(one ? q.cpg / V : q.cpg);
    q.across_magic = (uint32_t)((((uint64_t)1 << 32) + across - 1) / across);
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == 1 ? forward<float>(p, q, one, vec, eight, st)
                        : d.dtype == 0 ? forward<__nv_bfloat16>(p, q, one, vec, eight, st) : forward<__half>(p, q, one, vec, eight, st);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_group_norm_backward(const crisp_group_norm_t *desc, const void *d_dy, int64_t ld_dy, const void *d_x, int64_t ldx, const void *d_x8,
                                         const float *d_stats, const float *d_gamma, const float *d_beta, void *d_dx, int64_t ld_dx, float *d_dgamma,
                                         float *d_dbeta, void *d_workspace, void *stream) {
    const crisp_status_t bad = check(desc);
    if (bad != CRISP_OK) return bad;
    const crisp_group_norm_t &d = *desc;
    const int size = d.dtype == 1 ? 4 : 2;
    if (!aligned_to(d_dgamma, 4) || !aligned_to(d_dbeta, 4)) return CRISP_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (d.batch == 0) {
        const size_t bytes = (size_t)d.channels * sizeof(float);
        if (d_dgamma && cudaMemsetAsync(d_dgamma, 0, bytes, st) != cudaSuccess) return CRISP_CUDA_ERROR;
        if (d_dbeta && cudaMemsetAsync(d_dbeta, 0, bytes, st) != cudaSuccess) return CRISP_CUDA_ERROR;
        return CRISP_OK;
    }
    if (!d_dy || !d_dx || !d_stats || !d_workspace || (d_x == nullptr) == (d_x8 == nullptr) || !aligned_to(d_dy, size) || !aligned_to(d_dx, size) ||
        !aligned_to(d_x, size) || !aligned_to(d_x8, kAlign) || !aligned_to(d_stats, 8) || !aligned_to(d_gamma, 4) || !aligned_to(d_beta, 4) ||
        !aligned_to(d_workspace, kAlign))
        return CRISP_INVALID_ARG;
    if (ld_dy < d.channels || ld_dx < d.channels || (d_x && ldx < d.channels)) return CRISP_BAD_SHAPE;
    size_t bytes = 0;
    if (d_x8 && crisp_quantize8_sizes(d.channels, d.batch * d.pixels, &bytes) != CRISP_OK) return CRISP_UNSUPPORTED;
    const Plan p = plan_of(d, true, d_x8 != nullptr, false);
    const Space s = space_of(d, p, true);
    Norm q = norm_of(d, p, s, d_workspace);
    q.x = d_x; q.ldx = ldx; q.from8 = reinterpret_cast<const uint8_t *>(d_x8); q.dy = d_dy; q.ld_dy = ld_dy; q.out = d_dx; q.ld_out = ld_dx;
    q.gamma = d_gamma; q.beta = d_beta; q.stats = const_cast<float *>(d_stats);
    q.vec = vec_of(d_x, ldx, size); q.vec_dy = vec_of(d_dy, ld_dy, size); q.vec_out = vec_of(d_dx, ld_dx, size);
    const int V = 16 / size;
    const bool one = q.cpg % V == 0, vec = d.channels % V == 0 && (d_x8 || q.vec) && q.vec_dy && q.vec_out, from8 = d_x8 != nullptr;
    cudaError_t e = d.dtype == 1 ? backward<float>(p, q, one, vec, from8, st)
                  : d.dtype == 0 ? backward<__nv_bfloat16>(p, q, one, vec, from8, st) : backward<__half>(p, q, one, vec, from8, st);
    if (e == cudaSuccess && (d_dgamma || d_dbeta))
        e = launch_chained(sum_rows_kernel, (unsigned)((2 * (int64_t)d.channels + 31) / 32), 1024, 0, st, q.sums, (int64_t)(d.batch * p.ranks), d.channels, d_dgamma,
                           d_dbeta);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

}  // extern "C"
