// Group norm with an activation over channels-last activations, forward and backward.
//
//   of a sample's group (pixels x C / G channels):  mean, rstd = 1 / sqrt(var + eps)
//   h = (x - mean) rstd      y = act(p), p = gamma h + beta
//   backward:  e = dy act'(p)   dbeta = sum e   dgamma = sum e h   dx = rstd (gamma e - m1 - h m2),  m1, m2 = the group's means of gamma e, gamma e h
//
// Bound by memory: each value is needed twice, and what counts is that it comes from DRAM once.  A cluster of CTAs takes one sample's slice of whole groups; every
// thread keeps the values that it has read in shared memory of its own (no barrier: it reads what it wrote) until the cluster's sums are there, and reads again what
// does not fit.  Where one cluster's share of the SMs would be too few (one large image), and for groups of more channels than a slice holds, the same code runs as two
// kernels with the partial sums in between.
//
// A thread holds V = 16 bytes' worth of consecutive channels and goes over pixels.  Sums: each thread's values about its first one, so that a mean far from zero costs no
// digits; then mean = sum n_i mean_i / n and M2 = sum M2_i + n_i (mean_i - mean)^2 over threads and over CTAs, always in the same order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "block8.h"
#include "block8.cuh"

namespace crisp {

using namespace block8;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxCluster = 16;
constexpr size_t kMaxSmem = 232448 - 1024;

enum Act { kNone = 0, kRelu = 1, kRelu6 = 2, kSilu = 3 };
enum Mode { kWhole = 0, kSums = 1, kApply = 2 };          // one kernel with clusters, or the first and the second of two

struct Norm {
    const void *x, *dy;                  // dy: backward
    void *out;                           // y (or nullptr), dx
    const uint8_t *from8;                // backward: x in 8 bits (x: nullptr)
    uint8_t *x8, *y8;                    // forward: 8-bit forms to write, or nullptr
    const float *gamma, *beta;           // or nullptr: 1, 0
    float *stats;                        // [batch, groups, 2]
    float2 *partial;                     // two kernels: [batch, groups, p_ranks, parts]
    float *sums;                         // backward: [batch * ranks][2][channels]
    int64_t ldx, ld_dy, ld_out;
    int64_t cols8, groups8, chunks8;     // 8-bit form: columns (pixels of all samples), their groups of 8 and of 128
    size_t scale_off;
    int pixels, channels, groups, cpg;   // cpg: channels a group
    int width, slices;                   // channels a slice (kWhole: whole groups), slices a sample
    int ranks, per;                      // CTAs of a sample's slice, pixels of one
    int p_width, p_ranks, p_per, parts;  // the same of the kernel that fills `partial`, and the most slices that a group lies in there
    int cv, lanes;                       // threads a pixel, pixels at a time
    int resident;                        // items (V channels of a pixel) that a thread keeps
    int act, vec, vec_dy, vec_out;       // vec: addresses and pitches allow 16 bytes at once
    float eps;
};

template <typename T>
struct Of;
template <>
struct Of<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void open(const uint4 &u, float (&f)[4]) {
        f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 close(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float sigmoid(float p) { return 1.f / (1.f + expf(-p)); }
};
template <>
struct Of<__nv_bfloat16> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void open(const uint4 &u, float (&f)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 v = floats(w[i]); f[2 * i] = v.x; f[2 * i + 1] = v.y; }
    }
    static __device__ __forceinline__ uint4 close(const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t *>(&b); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // (some 2^-21 of the value, far below the result's last place)
    static __device__ __forceinline__ float sigmoid(float p) { return __fdividef(1.f, 1.f + __expf(-p)); }
};
template <>
struct Of<__half> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void open(const uint4 &u, float (&f)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[i])); f[2 * i] = v.x; f[2 * i + 1] = v.y; }
    }
    static __device__ __forceinline__ uint4 close(const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __half2 b = __floats2half2_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t *>(&b); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float sigmoid(float p) { return __fdividef(1.f, 1.f + __expf(-p)); }
};

__device__ __forceinline__ uint32_t smem_at(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
template <int kBytes>
__device__ __forceinline__ void copy_async(void *to, const void *from) {
    if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(to)), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_at(to)), "l"(from), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// V channels of one pixel, `n` of them there (the others 0).
template <typename T>
__device__ __forceinline__ uint4 fetch(const T *p, int vec, int n) {
    constexpr int V = Of<T>::V;
    if (vec && n == V) return *reinterpret_cast<const uint4 *>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j < n) {
            if constexpr (V == 4) w[j] = reinterpret_cast<const uint32_t *>(p)[j];
            else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[j] << (16 * (j & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void put(T *p, const uint4 &u, int vec, int n) {
    constexpr int V = Of<T>::V;
    if (vec && n == V) { *reinterpret_cast<uint4 *>(p) = u; return; }
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j < n) {
            if constexpr (V == 4) reinterpret_cast<uint32_t *>(p)[j] = w[j];
            else reinterpret_cast<uint16_t *>(p)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        }
}

// Where V channels of a column are in the 8-bit form, and the four bytes of their block's exponent.
__device__ __forceinline__ int64_t codes_at(const Norm &q, int64_t col, int ch) {
    const int kb = ch >> 7, c = ch & 127, r = (int)(col & 7);
    return ((int64_t)kb * q.groups8 + (col >> 3)) * 1024 + r * 128 + (((c >> 4) ^ r) << 4) + (c & 15);
}
__device__ __forceinline__ int64_t scale_at(const Norm &q, int64_t col, int ch) {
    return (int64_t)q.scale_off + ((int64_t)(ch >> 7) * q.chunks8 + (col >> 7)) * kScales8 + (col & 31) * 16 + (col >> 5 & 3) * 4;
}
// The values f of V channels (0 behind the last channel) to 8 bits; the 128 / V threads of a block are neighbours in a warp and all call this.
template <int V>
__device__ __forceinline__ void hold(const Norm &q, uint8_t *to, const float (&f)[V], int64_t col, int ch) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, fabsf(f[j]) < INFINITY ? fabsf(f[j]) : 0.f);         // what is not finite leaves the scale alone
    uint32_t bits = __float_as_uint(top);
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t peers = V == 4 ? 0xFFFFFFFFu : 0xFFFFu << (lane & 16);
#pragma unroll
    for (int d = 64 / V; d; d >>= 1) bits = max(bits, __shfl_xor_sync(peers, bits, d));
    const uint32_t e = (uint32_t)max((int)((bits + (0x7FFFFFu - 0x600000u)) >> 23) - 8, 1);
    const float down = power_of(254u - e);
    uint32_t codes[V / 4];
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        float s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fabsf(f[j + i]) < INFINITY ? f[j + i] * down : NAN;
        codes[j / 4] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(s[0], s[1]), __NV_SATFINITE, __NV_E4M3) |
                       (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(s[2], s[3]), __NV_SATFINITE, __NV_E4M3) << 16;
    }
    uint8_t *at = to + codes_at(q, col, ch);
    if constexpr (V == 8) *reinterpret_cast<uint2 *>(at) = make_uint2(codes[0], codes[1]);
    else *reinterpret_cast<uint32_t *>(at) = codes[0];
    if ((ch & 127) == 0) *reinterpret_cast<uint32_t *>(to + scale_at(q, col, ch)) = e * 0x01010101u;
}

template <int kAct, typename T>
__device__ __forceinline__ float activate(float p) {
    if constexpr (kAct == kRelu) return p < 0.f ? 0.f : p;                     // (NaN stays)
    if constexpr (kAct == kRelu6) return p < 0.f ? 0.f : p > 6.f ? 6.f : p;
    if constexpr (kAct == kSilu) return p * Of<T>::sigmoid(p);
    return p;
}

// A CTA's place: sample, first channel, channels, groups, pixels.
struct Place {
    int n, slice, rank, c0, width, g0, ng, px0, px1;
    __device__ __forceinline__ Place(const Norm &q) {
        const uint32_t u = blockIdx.x / (uint32_t)q.ranks;
        rank = (int)(blockIdx.x - u * (uint32_t)q.ranks);
        n = (int)(u / (uint32_t)q.slices);
        slice = (int)(u - (uint32_t)n * (uint32_t)q.slices);
        c0 = slice * q.width; width = min(q.width, q.channels - c0);
        g0 = c0 / q.cpg; ng = (c0 + width - 1) / q.cpg + 1 - g0;
        px0 = min(rank * q.per, q.pixels); px1 = min(px0 + q.per, q.pixels);
    }
};
__device__ __forceinline__ int items_of(int pixels, int lane, int lanes) { return pixels > lane ? (pixels - lane + lanes - 1) / lanes : 0; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// A group's channels inside the slice, from its first one on.
struct Span { int lo, hi; };
__device__ __forceinline__ Span span_of(const Norm &q, const Place &at, int g) {
    return {max(at.c0, (at.g0 + g) * q.cpg) - at.c0, min(at.c0 + at.width, (at.g0 + g + 1) * q.cpg) - at.c0};
}
// kSums: where the CTA's pair of group g goes.
__device__ __forceinline__ float2 *partial_at(const Norm &q, const Place &at, int g) {
    const int64_t group = at.g0 + g;
    return q.partial + (((int64_t)at.n * q.groups + group) * q.p_ranks + at.rank) * q.parts + (at.slice - (int)(group * q.cpg / q.p_width));
}
// A pair of each group of the slice, of all CTAs: kWhole: `own` [ng] in their shared memory; kApply: `partial`.  combine(g, count, lane, read, weight) is called by one
// warp a group; read(i) is the i-th pair and weight(i) the number of values that it stands for.
template <int kMode, typename F>
__device__ __forceinline__ void of_all(const Norm &q, const Place &at, const float2 *own, F combine) {
    const int lane = threadIdx.x & 31;
    if constexpr (kMode == kWhole) {
        cluster_arrive();
        cluster_wait();
    }
    for (int g = threadIdx.x >> 5; g < at.ng; g += kThreads / 32) {
        if constexpr (kMode == kWhole) {
            const uint32_t mine = smem_at(own + g);
            combine(g, q.ranks, lane,
                    [&](int i) {
                        const uint32_t a = peer_address(mine, (uint32_t)i);
                        return make_float2(__uint_as_float(lds32_peer(a)), __uint_as_float(lds32_peer(a + 4)));
                    },
                    [&](int i) { const int first = min(i * q.per, q.pixels); return (float)(min(first + q.per, q.pixels) - first) * (float)q.cpg; });
        } else {
            const int64_t group = at.g0 + g;
            const int from = (int)(group * q.cpg), to = from + q.cpg, s0 = from / q.p_width, parts = (to - 1) / q.p_width + 1 - s0;
            const float2 *row = q.partial + ((int64_t)at.n * q.groups + group) * q.p_ranks * q.parts;
            combine(g, q.p_ranks * parts, lane,
                    [&](int i) { const int r = i / parts; return row[r * q.parts + i - r * parts]; },
                    [&](int i) {
                        const int r = i / parts, s = s0 + i - r * parts, first = min(r * q.p_per, q.pixels);
                        return (float)(min(first + q.p_per, q.pixels) - first) * (float)(min(to, (s + 1) * q.p_width) - max(from, s * q.p_width));
                    });
        }
    }
    __syncwarp();
    if constexpr (kMode == kWhole) cluster_arrive();         // (its wait is at the kernel's end: no CTA leaves while others read from it)
    __syncthreads();
}

// ---------------------------------------------------------------------------------------------------------------- forward

// kOne: a thread's channels are of one group.
template <typename T, bool kOne, int kMode>
__global__ void __launch_bounds__(kThreads, 3)
norm_kernel(const __grid_constant__ Norm q) {
    constexpr int V = Of<T>::V;
    extern __shared__ __align__(16) uint8_t smem[];
    wait_for_prerequisites();
    const Place at(q);
    const int lane = threadIdx.x / q.cv, v = threadIdx.x - lane * q.cv;
    const int ch = at.c0 + v * V, n = lane < q.lanes ? max(0, min(V, at.c0 + at.width - ch)) : 0;
    const int items = lane < q.lanes ? items_of(at.px1 - at.px0, lane, q.lanes) : 0;
    const int64_t row0 = (int64_t)at.n * q.pixels + at.px0 + lane;
    const T *x = reinterpret_cast<const T *>(q.x) + row0 * q.ldx + ch;
    const int64_t step = (int64_t)q.lanes * q.ldx;
    float2 *groups = reinterpret_cast<float2 *>(smem);                       // [ng] of this CTA, then [ng] of all
    float2 *threads = groups + 2 * at.ng;                                    // [kThreads] or [kThreads][V]
    uint4 *kept = reinterpret_cast<uint4 *>(smem + ((2 * at.ng * 8 + kThreads * (kOne ? 1 : V) * 8 + 15) & ~15)) + threadIdx.x;
    const int resident = kMode == kWhole ? min(items, q.resident) : 0;

    if constexpr (kMode != kApply) {
        if (n > 0) {
            if (q.vec && n == V) {
                for (int i = 0; i < resident; ++i) copy_async<16>(kept + i * kThreads, x + i * step);
                copies_done();
            } else {
                for (int i = 0; i < resident; ++i) kept[i * kThreads] = fetch(x + i * step, q.vec, n);
            }
        }
        float pivot[V], s1[V], s2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) pivot[j] = s1[j] = s2[j] = 0.f;
        if (n > 0 && items > 0) Of<T>::open(resident ? kept[0] : fetch(x, q.vec, n), pivot);
        const auto add = [&](const uint4 &u) {
            float f[V];
            Of<T>::open(u, f);
#pragma unroll
            for (int j = 0; j < V; ++j) { const float d = f[j] - pivot[j]; s1[j] += d; s2[j] = fmaf(d, d, s2[j]); }
        };
        if (n > 0) {
            for (int i = 0; i < resident; ++i) add(kept[i * kThreads]);
            int i = resident;
            for (; i + 4 <= items; i += 4) {
                uint4 u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) u[k] = fetch(x + (i + k) * step, q.vec, n);
#pragma unroll
                for (int k = 0; k < 4; ++k) add(u[k]);
            }
            for (; i < items; ++i) add(fetch(x + i * step, q.vec, n));
        }
        // (mean, M2) of each channel, and of the thread
        const float count = (float)items, over = items ? 1.f / count : 0.f;
        float mean[V], m2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = s1[j] * over;
            mean[j] = pivot[j] + d;
            m2[j] = fmaxf(0.f, fmaf(-s1[j], d, s2[j]));
            if (!(s2[j] < INFINITY)) m2[j] = NAN;                            // (fmaxf would lose it)
        }
        if constexpr (kOne) {
            float all = 0.f, rest = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < n) all += mean[j] - mean[0];
            const float m = mean[0] + (n ? all / (float)n : 0.f);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < n) rest += m2[j] + count * (mean[j] - m) * (mean[j] - m);
            threads[threadIdx.x] = make_float2(m, rest);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) threads[threadIdx.x * V + j] = make_float2(mean[j], m2[j]);
        }
        __syncthreads();
        for (int g = threadIdx.x >> 5; g < at.ng; g += kThreads / 32) {
            const Span in = span_of(q, at, g);
            const int wide = in.hi - in.lo, across = kOne ? (wide + V - 1) / V : wide;       // entries of a group and lane
            const float total = (float)(at.px1 - at.px0) * (float)wide;
            const int entries = across * q.lanes;
            const auto entry = [&](int i, float *weight) {
                const int l = i / across, a = i - l * across;
                const float here = (float)items_of(at.px1 - at.px0, l, q.lanes);
                if constexpr (kOne) {
                    *weight = here * (float)min(V, wide - a * V);
                    return threads[l * q.cv + in.lo / V + a];
                } else {
                    const int c = in.lo + a;
                    *weight = here;
                    return threads[l * q.cv * V + c];
                }
            };
            // (about the first entry's mean, for the same reason as above)
            const float base = threads[kOne ? in.lo / V : in.lo].x;
            float w, sum = 0.f;
            for (int i = threadIdx.x & 31; i < entries; i += 32) { const float2 e = entry(i, &w); sum += w > 0.f ? w * (e.x - base) : 0.f; }
            const float m = base + (total > 0.f ? warp_sum(sum) / total : 0.f);
            float rest = 0.f;
            for (int i = threadIdx.x & 31; i < entries; i += 32) { const float2 e = entry(i, &w); rest += w > 0.f ? e.y + w * (e.x - m) * (e.x - m) : 0.f; }
            rest = warp_sum(rest);
            if ((threadIdx.x & 31) == 0) {
                if constexpr (kMode == kSums) *partial_at(q, at, g) = make_float2(m, rest);
                else groups[g] = make_float2(m, rest);
            }
        }
        if constexpr (kMode == kSums) return;
        __syncthreads();
    }
    float2 *known = groups + at.ng;
    of_all<kMode>(q, at, groups, [&](int g, int count, int l, auto read, auto weight) {
        const float all = (float)q.pixels * (float)q.cpg, base = read(0).x;
        float sum = 0.f, rest = 0.f;
        for (int i = l; i < count; i += 32) { const float w = weight(i); sum += w > 0.f ? w * (read(i).x - base) : 0.f; }
        const float m = base + warp_sum(sum) / all;
        for (int i = l; i < count; i += 32) { const float2 e = read(i); const float w = weight(i); rest += w > 0.f ? e.y + w * (e.x - m) * (e.x - m) : 0.f; }
        rest = warp_sum(rest);
        if (l == 0) {
            const float2 s = make_float2(m, 1.f / sqrtf(rest / all + q.eps));
            known[g] = s;
            if (at.rank == 0 && (at.g0 + g) * q.cpg >= at.c0) *reinterpret_cast<float2 *>(q.stats + 2 * ((int64_t)at.n * q.groups + at.g0 + g)) = s;
        }
    });
    const bool holds = q.x8 || q.y8;
    // (threads behind the last channel write the zeros that its block ends with; not of a block in which there is none)
    if (lane < q.lanes && (n > 0 || (holds && (ch & ~127) < q.channels))) {
        constexpr int M = kOne ? 1 : V;
        float mean[M], a[V], b[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            a[j] = b[j] = 0.f;
            if (j == 0 || !kOne) mean[kOne ? 0 : j] = 0.f;
            if (j >= n) continue;
            const float2 s = known[(ch + j) / q.cpg - at.g0];
            if (j == 0 || !kOne) mean[kOne ? 0 : j] = s.x;
            a[j] = s.y * (q.gamma ? q.gamma[ch + j] : 1.f);
            b[j] = q.beta ? q.beta[ch + j] : 0.f;
        }
        T *y = reinterpret_cast<T *>(q.out) + row0 * q.ld_out + ch;
        const int64_t step_y = (int64_t)q.lanes * q.ld_out;
        const auto finish = [&](int i, const uint4 &u) {
            float f[V], r[V];
            Of<T>::open(u, f);
            if (q.x8) hold<V>(q, q.x8, f, row0 + (int64_t)i * q.lanes, ch);
            const auto all = [&](auto act) {
#pragma unroll
                for (int j = 0; j < V; ++j) r[j] = activate<decltype(act)::value, T>(fmaf(f[j] - mean[kOne ? 0 : j], a[j], b[j]));
            };
            switch (q.act) {
                case kRelu: all(std::integral_constant<int, kRelu>()); break;
                case kRelu6: all(std::integral_constant<int, kRelu6>()); break;
                case kSilu: all(std::integral_constant<int, kSilu>()); break;
                default: all(std::integral_constant<int, kNone>());
            }
            if (holds && n < V) {
#pragma unroll
                for (int j = 0; j < V; ++j) r[j] = j < n ? r[j] : 0.f;
            }
            if (q.y8) hold<V>(q, q.y8, r, row0 + (int64_t)i * q.lanes, ch);
            if (q.out) put(y + i * step_y, Of<T>::close(r), q.vec_out, n);
        };
        const uint4 none = make_uint4(0, 0, 0, 0);
        for (int i = 0; i < resident; ++i) finish(i, n ? kept[i * kThreads] : none);
        int i = resident;
        for (; i + 4 <= items; i += 4) {
            uint4 u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = n ? fetch(x + (i + k) * step, q.vec, n) : none;
#pragma unroll
            for (int k = 0; k < 4; ++k) finish(i + k, u[k]);
        }
        for (; i < items; ++i) finish(i, n ? fetch(x + i * step, q.vec, n) : none);
    }
    __syncwarp();
    if constexpr (kMode == kWhole) cluster_wait();
}

// --------------------------------------------------------------------------------------------------------------- backward

template <int V>
__device__ __forceinline__ void decode(const uint32_t (&codes)[V / 4], uint32_t e, float (&f)[V]) {
    const float up = power_of(e);
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes[j / 4] >> (8 * (j & 2))), __NV_E4M3)));
        f[j] = v.x * up; f[j + 1] = v.y * up;
    }
}

// e = dy act'(p).  Where p is within its rounding of a border of relu or relu6, it is taken again in 64 bits, so that which side it lies on is the formula's: one
// element on the wrong side would be wrong by all of its dy.
template <int kAct, typename T>
__device__ __forceinline__ float slope(float dy, float x, float mean, float rstd, float gamma, float beta, float h) {
    if constexpr (kAct == kNone) return dy;
    float p = fmaf(h, gamma, beta);
    if constexpr (kAct == kSilu) {
        const float s = Of<T>::sigmoid(p);
        return dy * (s * fmaf(p, 1.f - s, 1.f));
    } else {
        const float near = (fabsf(beta) + 8.f) * 0x1p-20f;                   // h, p: four roundings of values up to |beta| + 6 around the borders
        if (fabsf(p) < near || (kAct == kRelu6 && fabsf(p - 6.f) < near)) {
            const double exact = ((double)x - (double)mean) * (double)rstd * (double)gamma + (double)beta;
            p = exact > 0.0 ? (kAct == kRelu6 && exact >= 6.0 ? 7.f : 1.f) : -1.f;
        }
        if constexpr (kAct == kRelu) return p <= 0.f ? 0.f : dy;
        return p <= 0.f || p >= 6.f ? 0.f : dy;
    }
}

template <typename T, bool kOne, bool k8, int kMode>
__global__ void __launch_bounds__(kThreads, 2)
norm_back_kernel(const __grid_constant__ Norm q) {
    constexpr int V = Of<T>::V, M = kOne ? 1 : V;
    extern __shared__ __align__(16) uint8_t smem[];
    wait_for_prerequisites();
    const Place at(q);
    const int lane = threadIdx.x / q.cv, v = threadIdx.x - lane * q.cv;
    const int ch = at.c0 + v * V, n = lane < q.lanes ? max(0, min(V, at.c0 + at.width - ch)) : 0;
    const int items = n > 0 ? items_of(at.px1 - at.px0, lane, q.lanes) : 0;
    const int64_t row0 = (int64_t)at.n * q.pixels + at.px0 + lane;
    const T *x = reinterpret_cast<const T *>(q.x) + row0 * q.ldx + ch, *dy = reinterpret_cast<const T *>(q.dy) + row0 * q.ld_dy + ch;
    const int64_t step_x = (int64_t)q.lanes * q.ldx, step_dy = (int64_t)q.lanes * q.ld_dy;
    float2 *groups = reinterpret_cast<float2 *>(smem);
    float2 *channels = groups + 2 * at.ng;                                   // [lanes][cv * V]: sums of e and of e h
    uint8_t *kept = smem + ((2 * at.ng * 8 + kThreads * V * 8 + 15) & ~15);
    // a thread's items: dy, then x; or its codes and the block's exponent
    uint4 *kept_dy = reinterpret_cast<uint4 *>(kept) + threadIdx.x, *kept_x = kept_dy + q.resident * kThreads;
    uint32_t *kept_codes = reinterpret_cast<uint32_t *>(kept + (size_t)q.resident * kThreads * 16) + threadIdx.x * (V / 4);
    uint32_t *kept_e = reinterpret_cast<uint32_t *>(kept + (size_t)q.resident * kThreads * (16 + V)) + threadIdx.x;
    const int resident = kMode == kWhole ? min(items, q.resident) : 0;

    float mean[M], rstd[M], gamma[V], beta[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        gamma[j] = beta[j] = 0.f;
        if (!kOne || j == 0) mean[kOne ? 0 : j] = rstd[kOne ? 0 : j] = 0.f;
        if (j >= n) continue;
        if (!kOne || j == 0) {
            const float2 s = *reinterpret_cast<const float2 *>(q.stats + 2 * ((int64_t)at.n * q.groups + (ch + j) / q.cpg));
            mean[kOne ? 0 : j] = s.x; rstd[kOne ? 0 : j] = s.y;
        }
        gamma[j] = q.gamma ? q.gamma[ch + j] : 1.f;
        beta[j] = q.beta ? q.beta[ch + j] : 0.f;
    }
    struct Item { uint4 dy, x; };                                            // x: 16 bytes, or codes and exponent
    const auto from_memory = [&](int i) {
        Item r;
        r.dy = fetch(dy + i * step_dy, q.vec_dy, n);
        if constexpr (k8) {
            const int64_t col = row0 + (int64_t)i * q.lanes;
            const uint8_t *p = q.from8 + codes_at(q, col, ch);
            if constexpr (V == 8) { const uint2 c = *reinterpret_cast<const uint2 *>(p); r.x.x = c.x; r.x.y = c.y; }
            else { r.x.x = *reinterpret_cast<const uint32_t *>(p); r.x.y = 0; }
            r.x.z = *reinterpret_cast<const uint32_t *>(q.from8 + scale_at(q, col, ch));
            r.x.w = 0;
        } else {
            r.x = fetch(x + i * step_x, q.vec, n);
        }
        return r;
    };
    const auto from_kept = [&](int i) {
        Item r;
        r.dy = kept_dy[i * kThreads];
        if constexpr (k8) {
            const uint32_t *c = kept_codes + i * kThreads * (V / 4);
            r.x = make_uint4(c[0], V == 8 ? c[V / 4 - 1] : 0u, kept_e[i * kThreads], 0u);
        } else {
            r.x = kept_x[i * kThreads];
        }
        return r;
    };
    const auto keep = [&](int i, const Item &r) {
        kept_dy[i * kThreads] = r.dy;
        if constexpr (k8) {
            uint32_t *c = kept_codes + i * kThreads * (V / 4);
            c[0] = r.x.x;
            if constexpr (V == 8) c[1] = r.x.y;
            kept_e[i * kThreads] = r.x.z;
        } else {
            kept_x[i * kThreads] = r.x;
        }
    };
    // calls f(e, h) with V values of each
    const auto terms = [&](const Item &r, auto f) {
        float d[V], xs[V], h[V];
        Of<T>::open(r.dy, d);
        if constexpr (k8) {
            uint32_t c[V / 4];
            c[0] = r.x.x;
            if constexpr (V == 8) c[1] = r.x.y;
            decode<V>(c, r.x.z & 0xFFu, xs);
        } else {
            Of<T>::open(r.x, xs);
        }
        const auto all = [&](auto act) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float m = mean[kOne ? 0 : j], s = rstd[kOne ? 0 : j];
                h[j] = (xs[j] - m) * s;
                d[j] = slope<decltype(act)::value, T>(d[j], xs[j], m, s, gamma[j], beta[j], h[j]);
            }
        };
        switch (q.act) {
            case kRelu: all(std::integral_constant<int, kRelu>()); break;
            case kRelu6: all(std::integral_constant<int, kRelu6>()); break;
            case kSilu: all(std::integral_constant<int, kSilu>()); break;
            default: all(std::integral_constant<int, kNone>());
        }
        f(d, h);
    };
    if constexpr (kMode != kApply) {
        if (q.vec_dy && (k8 || q.vec) && n == V) {
            for (int i = 0; i < resident; ++i) {
                copy_async<16>(kept_dy + i * kThreads, dy + i * step_dy);
                if constexpr (k8) {
                    const int64_t col = row0 + (int64_t)i * q.lanes;
                    copy_async<V>(kept_codes + i * kThreads * (V / 4), q.from8 + codes_at(q, col, ch));
                    copy_async<4>(kept_e + i * kThreads, q.from8 + scale_at(q, col, ch));
                } else {
                    copy_async<16>(kept_x + i * kThreads, x + i * step_x);
                }
            }
            copies_done();
        } else {
            for (int i = 0; i < resident; ++i) keep(i, from_memory(i));
        }
        float db[V], dg[V];
#pragma unroll
        for (int j = 0; j < V; ++j) db[j] = dg[j] = 0.f;
        const auto add = [&](const float (&e)[V], const float (&h)[V]) {
#pragma unroll
            for (int j = 0; j < V; ++j) { db[j] += e[j]; dg[j] = fmaf(e[j], h[j], dg[j]); }
        };
        for (int i = 0; i < resident; ++i) terms(from_kept(i), add);
        int i = resident;
        for (; i + 2 <= items; i += 2) {
            const Item a = from_memory(i), b = from_memory(i + 1);
            terms(a, add);
            terms(b, add);
        }
        if (i < items) terms(from_memory(i), add);
        const int row = q.cv * V;
        if (lane < q.lanes) {
#pragma unroll
            for (int j = 0; j < V; ++j) channels[lane * row + v * V + j] = make_float2(db[j], dg[j]);
        }
        __syncthreads();
        // of each channel over the lanes: for gamma and beta, and back to the first lane's place times gamma for the group
        float *sums = q.sums + ((int64_t)at.n * q.ranks + at.rank) * 2 * q.channels;
        for (int c = threadIdx.x; c < at.width; c += kThreads) {
            float2 s = make_float2(0.f, 0.f);
            for (int l = 0; l < q.lanes; ++l) { const float2 t = channels[l * row + c]; s.x += t.x; s.y += t.y; }
            sums[at.c0 + c] = s.x;
            sums[q.channels + at.c0 + c] = s.y;
            const float w = q.gamma ? q.gamma[at.c0 + c] : 1.f;
            channels[c] = make_float2(w * s.x, w * s.y);
        }
        __syncthreads();
        for (int g = threadIdx.x >> 5; g < at.ng; g += kThreads / 32) {
            float2 s = make_float2(0.f, 0.f);
            const Span in = span_of(q, at, g);
            for (int c = in.lo + (threadIdx.x & 31); c < in.hi; c += 32) { const float2 t = channels[c]; s.x += t.x; s.y += t.y; }
            s.x = warp_sum(s.x); s.y = warp_sum(s.y);
            if ((threadIdx.x & 31) == 0) {
                if constexpr (kMode == kSums) *partial_at(q, at, g) = s;
                else groups[g] = s;
            }
        }
        if constexpr (kMode == kSums) return;
        __syncthreads();
    }
    float2 *known = groups + at.ng;
    of_all<kMode>(q, at, groups, [&](int g, int count, int l, auto read, auto) {
        float2 s = make_float2(0.f, 0.f);
        for (int i = l; i < count; i += 32) { const float2 t = read(i); s.x += t.x; s.y += t.y; }
        s.x = warp_sum(s.x); s.y = warp_sum(s.y);
        const float all = (float)q.pixels * (float)q.cpg;
        if (l == 0) known[g] = make_float2(s.x / all, s.y / all);
    });
    if (items > 0) {
        float2 m[M];
#pragma unroll
        for (int j = 0; j < M; ++j) m[j] = j < n ? known[(ch + j) / q.cpg - at.g0] : make_float2(0.f, 0.f);
        T *dx = reinterpret_cast<T *>(q.out) + row0 * q.ld_out + ch;
        const int64_t step_out = (int64_t)q.lanes * q.ld_out;
        const auto finish = [&](int i, const Item &r) {
            terms(r, [&](const float (&e)[V], const float (&h)[V]) {
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 g = m[kOne ? 0 : j];
                    o[j] = rstd[kOne ? 0 : j] * (fmaf(gamma[j], e[j], -g.x) - h[j] * g.y);
                }
                put(dx + i * step_out, Of<T>::close(o), q.vec_out, n);
            });
        };
        for (int i = 0; i < resident; ++i) finish(i, from_kept(i));
        int i = resident;
        for (; i + 2 <= items; i += 2) {
            const Item a = from_memory(i), b = from_memory(i + 1);
            finish(i, a);
            finish(i + 1, b);
        }
        if (i < items) finish(i, from_memory(i));
    }
    __syncwarp();
    if constexpr (kMode == kWhole) cluster_wait();
}

// dbeta and dgamma: the sums of all CTAs' [rows][2][channels], a warp's lanes on 32 neighbouring ones, in one order.
__global__ void __launch_bounds__(1024)
sum_rows_kernel(const float *sums, int64_t rows, int channels, float *dgamma, float *dbeta) {
    __shared__ float part[32][33];
    wait_for_prerequisites();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < 2 * (int64_t)channels)
        for (int64_t r = warp; r < rows; r += 32) s += sums[r * 2 * channels + c];
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

// How a call is cut: a kernel with clusters, or two without.
struct Cut { int width, slices, ranks, per, cv; };
struct Plan {
    bool whole;
    Cut sums, apply;                     // (whole: `sums` is the one kernel's)
    int resident, parts;
    int threads_smem, groups_smem;       // bytes in front of what the threads keep
};
constexpr int kSms = 148;
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

Cut cut_of(const crisp_group_norm_t &d, int V, int width, bool eight, int64_t most_ranks, int64_t ctas) {
    Cut c{};
    c.width = width;
    c.slices = ceil_div(d.channels, width);
    c.cv = eight ? ceil_div(width, 128) * (128 / V) : ceil_div(width, V);
    const int lanes = kThreads / c.cv;
    // enough CTAs, but two items a thread before a slice is cut further
    int64_t ranks = std::min(most_ranks, std::max<int64_t>(1, ctas / std::max<int64_t>(1, d.batch * c.slices)));
    ranks = std::max<int64_t>(1, std::min<int64_t>(ranks, ceil_div(d.pixels, 2 * lanes)));
    c.per = ceil_div(d.pixels, ranks);
    c.ranks = (int)ranks;
    return c;
}

Plan plan_of(const crisp_group_norm_t &d, bool back, bool from8, bool eight) {
    Plan p{};
    const int size = d.dtype == 1 ? 4 : 2, V = 16 / size, C = d.channels, cpg = C / d.groups;
    const int most = kThreads * V, align = eight ? 128 : V;                  // channels that a CTA's threads hold side by side; multiples that slices are of
    int g = cpg, h = align;
    while (h) { const int t = g % h; g = h; h = t; }
    const int64_t lcm = (int64_t)(cpg / g) * align;
    const int unit = (int)std::min<int64_t>(lcm, C);                         // the narrowest slice of whole groups
    const int item = back ? (from8 ? 16 + V + 4 : 32) : 16;
    p.threads_smem = kThreads * (cpg % V == 0 && !back ? 1 : V) * 8;
    if ((unit + align - 1) / align * align <= most) {
        int width = unit;
        while (width < C && width * size < 128 && width + unit <= most) width += unit;
        width = std::min(width, C);
        p.sums = cut_of(d, V, width, eight, kMaxCluster, 3 * kSms);
        const int lanes = kThreads / p.sums.cv;
        const auto fixed = [&] { return (size_t)((2 * (ceil_div(p.sums.width, cpg) + 1) * 8 + p.threads_smem + 15) & ~15); };
        const auto wanted = [&] { return fixed() + (size_t)ceil_div(p.sums.per, lanes) * kThreads * item; };
        while (wanted() > kMaxSmem / 3 && p.sums.ranks < kMaxCluster) {
            p.sums.ranks = std::min(kMaxCluster, p.sums.ranks * 2);
            p.sums.per = ceil_div(d.pixels, p.sums.ranks);
        }
        p.whole = d.batch * p.sums.slices * p.sums.ranks >= kSms / 2 || d.pixels * C * d.batch <= (1 << 20);
        const size_t room = wanted() <= kMaxSmem / 3 ? kMaxSmem / 3 : wanted() <= kMaxSmem / 2 ? kMaxSmem / 2 : kMaxSmem;
        p.resident = std::min(ceil_div(p.sums.per, lanes), (int)((room - fixed()) / (kThreads * item)));
    }
    if (!p.whole) {
        int width = align;
        while (width < C && width * size < 512 && width + align <= most) width += align;
        width = std::min(width, C);
        p.sums = p.apply = cut_of(d, V, width, eight, 1 << 16, 6 * kSms);
        p.resident = 0;
    }
    p.parts = p.whole ? 1 : (cpg + p.sums.width - 2) / p.sums.width + 1;
    p.groups_smem = 2 * (ceil_div(p.sums.width, cpg) + 1) * 8;
    return p;
}
size_t smem_of(const Plan &p, int item) { return (size_t)((p.groups_smem + p.threads_smem + 15) & ~15) + (size_t)p.resident * kThreads * item; }

// Workspace: the sums of gamma's and beta's gradients, then the two kernels' partial sums.
struct Space { size_t sums, partial; };
Space space_of(const crisp_group_norm_t &d, const Plan &p, bool back) {
    Space s{};
    if (back) s.sums = align_up((size_t)d.batch * p.sums.ranks * 2 * d.channels * sizeof(float));
    if (!p.whole) s.partial = align_up((size_t)d.batch * d.groups * p.sums.ranks * p.parts * sizeof(float2));
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

template <auto kernel>
cudaError_t launch(const Norm &q, int64_t batch, size_t smem, unsigned cluster, cudaStream_t st) {
    const int64_t grid = batch * q.slices * q.ranks;
    if (grid > 0x7FFFFFFFll) return cudaErrorInvalidValue;
    static std::atomic<uint64_t> ready{0};                                    // (one a kernel: by device)
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= 64 || !(ready.load(std::memory_order_relaxed) >> device & 1)) {
        e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (device < 64) ready.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    return launch_clusters(kernel, (unsigned)grid, kThreads, smem, st, cluster, q);
}

void set_cut(Norm *q, const Cut &c) {
    q->width = c.width; q->slices = c.slices; q->ranks = c.ranks; q->per = c.per; q->cv = c.cv;
    q->lanes = kThreads / c.cv;
}

template <typename T, bool kOne>
cudaError_t forward(const crisp_group_norm_t &d, const Plan &p, Norm q, cudaStream_t st) {
    set_cut(&q, p.sums);
    if (p.whole) return launch<norm_kernel<T, kOne, kWhole>>(q, d.batch, smem_of(p, 16), (unsigned)q.ranks, st);
    const cudaError_t e = launch<norm_kernel<T, kOne, kSums>>(q, d.batch, smem_of(p, 16), 1, st);
    if (e != cudaSuccess) return e;
    set_cut(&q, p.apply);
    return launch<norm_kernel<T, kOne, kApply>>(q, d.batch, smem_of(p, 16), 1, st);
}
template <typename T, bool kOne, bool k8>
cudaError_t backward(const crisp_group_norm_t &d, const Plan &p, Norm q, cudaStream_t st) {
    const int item = k8 ? 16 + Of<T>::V + 4 : 32;
    set_cut(&q, p.sums);
    if (p.whole) return launch<norm_back_kernel<T, kOne, k8, kWhole>>(q, d.batch, smem_of(p, item), (unsigned)q.ranks, st);
    const cudaError_t e = launch<norm_back_kernel<T, kOne, k8, kSums>>(q, d.batch, smem_of(p, item), 1, st);
    if (e != cudaSuccess) return e;
    set_cut(&q, p.apply);
    return launch<norm_back_kernel<T, kOne, k8, kApply>>(q, d.batch, smem_of(p, item), 1, st);
}

int vec_of(const void *p, int64_t ld, int size) { return aligned_to(p, 16) && ld * size % 16 == 0; }

Norm norm_of(const crisp_group_norm_t &d, const Plan &p, const Space &s, void *workspace) {
    Norm q{};
    q.sums = reinterpret_cast<float *>(workspace);
    q.partial = reinterpret_cast<float2 *>(reinterpret_cast<uint8_t *>(workspace) + s.sums);
    q.pixels = (int)d.pixels; q.channels = d.channels; q.groups = d.groups; q.cpg = d.channels / d.groups;
    q.p_width = p.sums.width; q.p_ranks = p.sums.ranks; q.p_per = p.sums.per; q.parts = p.parts;
    q.resident = p.resident;
    q.act = d.activation;
    q.eps = (float)d.eps;
    const Act8 a = act8(d.channels, d.batch * d.pixels);
    q.cols8 = d.batch * d.pixels; q.groups8 = a.groups; q.chunks8 = a.chunks; q.scale_off = a.scale_off;
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
        *workspace_bytes = std::max(*workspace_bytes, s.sums + s.partial);
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
    if (s.partial && !d_workspace) return CRISP_INVALID_ARG;
    Norm q = norm_of(d, p, s, d_workspace);
    q.x = d_x; q.ldx = ldx; q.out = d_y; q.ld_out = ldy; q.gamma = d_gamma; q.beta = d_beta; q.stats = d_stats;
    q.x8 = reinterpret_cast<uint8_t *>(d_x8); q.y8 = reinterpret_cast<uint8_t *>(d_y8);
    q.vec = vec_of(d_x, ldx, size); q.vec_out = vec_of(d_y, ldy, size);
    const bool one = q.cpg % (16 / size) == 0;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == 1 ? (one ? forward<float, true>(d, p, q, st) : forward<float, false>(d, p, q, st))
                        : d.dtype == 0 ? (one ? forward<__nv_bfloat16, true>(d, p, q, st) : forward<__nv_bfloat16, false>(d, p, q, st))
                                       : (one ? forward<__half, true>(d, p, q, st) : forward<__half, false>(d, p, q, st));
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
    const bool one = q.cpg % (16 / size) == 0;
    cudaError_t e;
#define CRISP_BACK(T) (one ? (d_x8 ? backward<T, true, true>(d, p, q, st) : backward<T, true, false>(d, p, q, st)) \
                           : (d_x8 ? backward<T, false, true>(d, p, q, st) : backward<T, false, false>(d, p, q, st)))
    if (d.dtype == 1) e = CRISP_BACK(float);
    else if (d.dtype == 0) e = CRISP_BACK(__nv_bfloat16);
    else e = CRISP_BACK(__half);
#undef CRISP_BACK
    if (e == cudaSuccess && (d_dgamma || d_dbeta))
        e = launch_chained(sum_rows_kernel, (unsigned)((2 * (int64_t)d.channels + 31) / 32), 1024, 0, st, q.sums, (int64_t)(d.batch * p.sums.ranks), d.channels, d_dgamma,
                           d_dbeta);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

}  // extern "C"
