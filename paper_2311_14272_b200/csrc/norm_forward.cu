// Group norm with an activation: the forward pass, how calls are cut, and the C entries (norm.cuh has the formulas and what bounds them).
#include "norm.cuh"

namespace crisp {
namespace norm {

namespace {

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

__device__ __forceinline__ uint64_t minus(uint64_t a) { return mul2(a, f32x2(-1.f, -1.f)); }
// A thread's sums of `count` items (values less a point, and their squares) about the mean so far; over = 1 / count.  Done after 1, 4, 16 ... items: those that follow, three times as many, add
// 3 count d^2 for the distance d of their mean from that one, of which 3/4 count d^2 is theirs to add, so that no more than four times a sum is added and taken away again (eight times in a first
// item of eight channels), wherever the values lie that are far from the others.  (About the first value all along: a first one of 1000, and 240 others of size one, left 1e-4 of the variance wrong.)
template <int V, bool kOne>
__device__ __forceinline__ void about_mean(int count, float over, uint64_t (&away)[kOne ? 1 : V / 2], uint64_t (&s1)[V / 2], uint64_t (&s2)[V / 2]) {
    constexpr int P = V / 2;
    if constexpr (kOne) {
        const float one = f32x2_sum(P == 4 ? add2(add2(s1[0], s1[1]), add2(s1[P - 2], s1[P - 1])) : add2(s1[0], s1[1]));
        const float two = f32x2_sum(P == 4 ? add2(add2(s2[0], s2[1]), add2(s2[P - 2], s2[P - 1])) : add2(s2[0], s2[1]));
        const float old = f32x2_halves(away[0]).x, n = (float)count * V, point = fmaf(one, -over / V, old), by = old - point, rest = fmaf(-n, by, one);
        away[0] = both(point);
#pragma unroll
        for (int j = 0; j < P; ++j) s1[j] = s2[j] = 0;
        s1[0] = f32x2(rest, 0.f);
        s2[0] = f32x2(fmaf(-by, one + rest, two), 0.f);      // sum (v - by)^2 = sum v^2 - by (sum v + sum (v - by))
    } else {
        const uint64_t n = both(-(float)count), less = both(-over);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const uint64_t old = away[j], by = add2(old, minus(away[j] = fma2(s1[j], less, old))), one = s1[j];
            s1[j] = fma2(n, by, one);
            s2[j] = fma2(minus(by), add2(one, s1[j]), s2[j]);
        }
    }
}
// Pairs (mean, M2) of the CTA's groups to give(g, pair).
template <typename T, bool kOne, bool kOver, typename I, typename F>
__device__ __forceinline__ void sum_x(const Norm &q, const Place &at, const Mine<T> &me, float2 *threads, I &items, F give) {
    constexpr int V = Of<T>::V, P = V / 2;
    uint64_t away[kOne ? 1 : P], s1[P], s2[P];               // away: less the point that sums are about (kOne: one for all)
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
        float over = 1.f;
        for (int i = 0, until = 1;; until *= 4, over *= 0.25f) {
            const int end = min(until, me.items);
#pragma unroll 2
            for (;;) {
                Of<T>::open(u, f);
#pragma unroll
                for (int j = 0; j < P; ++j) { const uint64_t d = add2(f[j], away[kOne ? 0 : j]); s1[j] = add2(s1[j], d); s2[j] = fma2(d, d, s2[j]); }
                items.done();
                if (++i >= end) break;
                u = items.next();
            }
            if (i >= me.items) break;
            about_mean<V, kOne>(i, over, away, s1, s2);
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
    return make_float2((float)((double)base + off), 1.f / sqrtf(max_nan(0.f, (float)((rest - sum * off) / all)) + q.eps));
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
    uint64_t away[P], a[P], b[P];                            // p = a (x - mean) + beta
#pragma unroll
    for (int j = 0; j < P; ++j) {
        float m[2] = {0.f, 0.f}, s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = me.ch + 2 * j + i;
            if ((kVec && !kHold) || 2 * j + i < me.n) {
                const float2 k = known(group_of(q, c));
                m[i] = -k.x;
                s[i] = k.y * (q.gamma ? q.gamma[c] : 1.f);
                t[i] = q.beta ? q.beta[c] : 0.f;
            }
        }
        away[j] = f32x2(m[0], m[1]); a[j] = f32x2(s[0], s[1]); b[j] = f32x2(t[0], t[1]);
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
            for (int j = 0; j < P; ++j) f[j] = activate<decltype(act)::value, T>(fma2(add2(f[j], away[j]), a[j], b[j]));      // (0 behind the last channel)
            if constexpr (kHold) if (q.y8) hold<V>(q, q.y8, f, col, me.ch);
            items.done();
            if (!kHold || (q.out && me.n > 0)) put<kVec && !kHold>(y, Of<T>::close(f), q.vec_out, me.n);
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

constexpr int kSms = 148;
// Small calls: those that read at most so much (dy, too); above that either form can be ahead, by the shape.  Device times of one kernel with clusters and of two, us: forward 1 x 28 x 28 x 512 (0.8 MB) 7.4 and 8.3, 8 images (6.4 MB)
// 7.9 and 12.0, 32 images (25.7 MB) 11.4 and 15.9, 48 images 18.3 and 19.5, 16 x 112 x 112 x 96 (38.5 MB) 34.9 and 22.0; backward 8 x 14 x 14 x 512 (3.2 MB) 9.1 and 12.2, 8 x 28 x 28 x 256
// (6.4 MB) 11.4 and 13.8, 4 x 56 x 56 x 256 (12.8 MB) 20.2 and 15.6, 24 x 28 x 28 x 512 (38.5 MB) 28.9 and 22.2.
constexpr int64_t kSmallForward = 28 << 20, kSmallBackward = 8 << 20;
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
    if (whole && bytes <= (back ? kSmallBackward : kSmallForward)) {
        // slices of 128 bytes a pixel and more, where there are CTAs enough, and of about the same width
        int64_t width = unit;
        while (width < C && width + unit <= most && (width * size < 128 || (2 * width <= most && batch * ceil_div(C, 2 * width) >= 2 * kSms))) width += unit;
        const int64_t slices = ceil_div(C, width);
        width = ceil_div(ceil_div(C, slices), unit) * unit;
        slice((int)std::min<int64_t>(width, C));
        // a power of two of CTAs (other clusters leave SMs of a GPC empty), no more in all than run at once, two items a thread before a slice is cut further
        const int64_t at_once = 2 * kSms / (batch * p.slices), worth = ceil_div(d.pixels, 2 * (kThreads / p.cv));
        int64_t ranks = 1;
        while (2 * ranks <= kMaxCluster && 2 * ranks <= at_once && ranks < worth) ranks *= 2;
        rank(ranks);
        while (wanted() > kMaxSmem / 2 && p.ranks < kMaxCluster) rank(std::min<int64_t>(kMaxCluster, 2 * (int64_t)p.ranks));
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
    if (d->pixels > 0x7FFFFFFFll - 65536 || d->batch > 0x7FFFFFFFll || d->channels > kMaxBlocksPerRowTile * 128 ||
        (double)d->batch * (double)d->pixels * (double)d->channels > 0x1p44)
        return CRISP_UNSUPPORTED;
    return CRISP_OK;
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
    // (an odd number of pixel lanes would have a place of the ring change its order, and a thread write where a neighbour has yet to read)
    q.as_stored = d.channels % 128 == 0 && p.width % 128 == 0 && kDeepDy * q.lanes % 8 == 0;
    if (q.cpg > 1 && (double)d.channels * q.cpg < 4294967296.0) q.cpg_magic = (uint32_t)((((uint64_t)1 << 32) + q.cpg - 1) / q.cpg);
    q.act = d.activation;
    q.eps = (float)d.eps;
    const Act8 a = act8(d.channels, d.batch * d.pixels);
    q.groups8 = a.groups; q.chunks8 = a.chunks; q.scale_off = a.scale_off;
    return q;
}

}  // namespace

}  // namespace norm
}  // namespace crisp

extern "C" {

using namespace crisp;
using namespace crisp::norm;

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
    cudaError_t e = d.dtype == 1 ? backward_fp32(p, q, one, vec, from8, st)
                  : d.dtype == 0 ? backward_bf16(p, q, one, vec, from8, st) : backward_fp16(p, q, one, vec, from8, st);
    if (e == cudaSuccess && (d_dgamma || d_dbeta))
        e = launch_chained(sum_rows_kernel, (unsigned)((2 * (int64_t)d.channels + 31) / 32), 1024, 0, st, q.sums, (int64_t)(d.batch * p.ranks), d.channels, d_dgamma,
                           d_dbeta);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

}  // extern "C"
