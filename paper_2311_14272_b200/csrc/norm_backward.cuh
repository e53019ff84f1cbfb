// Group norm with an activation: the backward pass (norm.cuh has the formulas and what bounds them).
#pragma once

#include "norm.cuh"

namespace crisp {
namespace norm {

namespace {

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

// A thread's coefficients of p = a (x - mean) + b, and how near to a border of relu or relu6 p may be off.
template <int P, bool kOne>
struct Affine {
    uint64_t away[kOne ? 1 : P], a[P], b[P];                 // away: less the means
    float near;
};
// Which side of the borders p lies on, from the formula in 64 bits: -1, 1 or 7.
__device__ __noinline__ float side_of(const Norm &q, int64_t stat, int c, float x) {
    const double exact = ((double)x - (double)q.stats[2 * stat]) * (double)q.stats[2 * stat + 1] * (q.gamma ? (double)q.gamma[c] : 1.0) + (q.beta ? (double)q.beta[c] : 0.0);
    return exact > 0.0 ? (exact >= 6.0 ? 7.f : 1.f) : -1.f;
}
// e = dy act'(p), d = x - mean.  Where p is within its roundings of a border, its side is taken from 64 bits, so that it is the formula's: one element on the wrong side would be
// wrong by all of its dy.  again(x): x once more.
template <int kAct, typename T, int P, bool kOne, typename F>
__device__ __forceinline__ void slope(const Norm &q, int n, int ch, const Affine<P, kOne> &k, const uint64_t (&d)[P], uint64_t (&dy)[P], F again) {
    if constexpr (kAct == kNone) return;
    if constexpr (kAct == kSilu) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const uint64_t p = fma2(d[j], k.a[j], k.b[j]);
            const uint64_t s = Of<T>::sigmoid2(p), rest = fma2(s, both(-1.f), both(1.f));
            dy[j] = mul2(dy[j], mul2(s, fma2(p, rest, both(1.f))));
        }
    } else {
        float p[2 * P], least = INFINITY;                     // (three values a minimum)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float2 v = f32x2_halves(fma2(d[j], k.a[j], k.b[j]));
            p[2 * j] = v.x; p[2 * j + 1] = v.y;
            least = fminf(fminf(fabsf(v.x), fabsf(v.y)), least);
            if constexpr (kAct == kRelu6) least = fminf(fminf(fabsf(v.x - 6.f), fabsf(v.y - 6.f)), least);
        }
        if (least < k.near) {
            uint64_t x[P];
            again(x);
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
__device__ __forceinline__ void affine_of(const Norm &q, const Place &at, const Mine<T> &me, Affine<Of<T>::V / 2, kOne> *k, float (&rstd)[kOne ? 1 : Of<T>::V]) {
    constexpr int V = Of<T>::V;
    k->near = 0.f;
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        float mean[2] = {0.f, 0.f}, a[2] = {0.f, 0.f}, b[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = me.ch + j + i, m = kOne ? 0 : j + i;
            if (!kOne || j + i == 0) rstd[m] = 0.f;
            if (j + i >= me.n) continue;
            if (!kOne || j + i == 0) {
                const float2 s = *reinterpret_cast<const float2 *>(q.stats + 2 * ((int64_t)at.n * q.groups + group_of(q, c)));
                mean[i] = s.x; rstd[m] = s.y;
            }
            a[i] = rstd[m] * (q.gamma ? q.gamma[c] : 1.f);
            b[i] = q.beta ? q.beta[c] : 0.f;
            // a and x - mean are each off by u (2^-24), p by one more of its own; at a border |a (x - mean)| <= |b| + 6
            k->near = fmaxf(k->near, (fabsf(b[i]) + 8.f) * 0x1p-22f);
        }
        if constexpr (kOne) { if (j == 0) k->away[0] = both(-mean[0]); }
        else k->away[j / 2] = f32x2(-mean[0], -mean[1]);
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
    // to one line as it comes from one (else 53 wavefronts an item, not 14; the time of 56 x 56 x 256 from 8 bits, 32 images, is 58 us either way).  The items that come to
    // one place of the ring lie a multiple of eight columns apart then, so that the bytes are the thread's own there.
    __device__ __forceinline__ int place(int64_t col) const {
        const int c = me.ch & 127;
        return q.as_stored ? (int)(threadIdx.x & ~(128 / V - 1)) * V + ((((c >> 4) ^ (int)col) & 7) << 4) + (c & 15) : (int)threadIdx.x * V;
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
        open_x(r, f);
    }
    static __device__ __forceinline__ void open_x(const Item &r, uint64_t (&f)[V / 2]) {
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
    Affine<P, kOne> k;
    float rstd[M];
    affine_of<T, kOne>(q, at, me, &k, rstd);
    uint64_t db[P], dg[P];                                   // dg: of e (x - mean)
#pragma unroll
    for (int j = 0; j < P; ++j) db[j] = dg[j] = 0;
    if (me.n > 0)
        with_act(q.act, [&](auto act) {
#pragma unroll 1
            for (int i = 0; i < me.items; ++i) {
                uint64_t e[P], d[P];
                const Item item = items.next();
                Reader<T, k8, kVec>::open(item, e, d);
#pragma unroll
                for (int j = 0; j < P; ++j) d[j] = add2(d[j], k.away[kOne ? 0 : j]);
                slope<decltype(act)::value, T, P, kOne>(q, at.n, me.ch, k, d, e, [&](uint64_t (&x)[P]) { Reader<T, k8, kVec>::open_x(item, x); });
#pragma unroll
                for (int j = 0; j < P; ++j) { db[j] = add2(db[j], e[j]); dg[j] = fma2(e[j], d[j], dg[j]); }
                items.done();
            }
        });
    if constexpr (kOver) __syncthreads();
    const int row = q.cv * V;
    if (me.lane < q.lanes) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float2 b = f32x2_halves(db[j]), g = f32x2_halves(dg[j]);
            channels[me.lane * row + me.v * V + 2 * j] = make_float2(b.x, g.x * rstd[kOne ? 0 : 2 * j]);
            channels[me.lane * row + me.v * V + 2 * j + 1] = make_float2(b.y, g.y * rstd[kOne ? 0 : 2 * j + 1]);
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

// dx of the CTA's pixels (kDown: the last one first); known(g): m1 and m2 of the sample's group g.  dx = rstd (gamma e - m1 - h m2) = a e + B (x - mean) + C.
template <typename T, bool kOne, bool k8, bool kVec, bool kDown, typename K, typename F>
__device__ __forceinline__ void finish_dx(const Norm &q, const Place &at, const Mine<T> &me, K &items, F known) {
    constexpr int V = Of<T>::V, P = V / 2, M = kOne ? 1 : V;
    if (me.n <= 0) return;
    Affine<P, kOne> k;
    float rstd[M];
    affine_of<T, kOne>(q, at, me, &k, rstd);
    uint64_t B[kOne ? 1 : P], C[kOne ? 1 : P];
#pragma unroll
    for (int j = 0; j < (kOne ? 1 : P); ++j) {
        float b[2], c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = kOne ? 0 : 2 * j + i;
            const float2 g = m < me.n ? known(group_of(q, me.ch + m)) : make_float2(0.f, 0.f);
            b[i] = -rstd[m] * rstd[m] * g.y;
            c[i] = -rstd[m] * g.x;
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
            uint64_t e[P], d[P];
            const Item item = items.next();
            Reader<T, k8, kVec>::open(item, e, d);
#pragma unroll
            for (int j = 0; j < P; ++j) d[j] = add2(d[j], k.away[kOne ? 0 : j]);
            slope<decltype(act)::value, T, P, kOne>(q, at.n, me.ch, k, d, e, [&](uint64_t (&x)[P]) { Reader<T, k8, kVec>::open_x(item, x); });
#pragma unroll
            for (int j = 0; j < P; ++j) e[j] = fma2(e[j], k.a[j], fma2(d[j], B[kOne ? 0 : j], C[kOne ? 0 : j]));
            items.done();
            put<kVec>(dx, Of<T>::close(e), q.vec_out, me.n);
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

}  // namespace

}  // namespace norm
}  // namespace crisp
