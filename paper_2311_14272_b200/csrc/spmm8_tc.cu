// The 8-bit product on the tensor cores: Y = act(W X + bias) with e4m3 operands and a power-of-two scale for each block of 128 (block8.h has the layout).
//
//   Y[r, c] = sum over the kept blocks b of r's row tile of 2^(Ew + Ex[b, c]) sum_k qw[r, k] qx[k, c]
//
// tcgen05.mma.kind::mxf8f6f4.block_scale takes a scale for every row of A and column of B and each 32 of K; here the four K steps of a block share theirs, so that the
// accumulator in tensor memory holds the scaled sum and nothing is rescaled outside.  A CTA multiplies a tile of 128 rows (one row tile of the layer, whose kept
// blocks it walks) and up to 256 columns.  Per kept block a pipeline stage holds 16.5 KB of weights with their scales (one tiled copy of the weight buffer), the codes
// of the columns (a contiguous piece of the activation buffer, one copy) and their scales.  Roles as in the bf16 kernel: a thread that fetches weights, one that
// fetches activations, one that issues scale copies and MMAs, and warps that drain accumulators.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cstring>
#include <memory>
#include <new>

#include "block8.cuh"
#include "block8.h"
#include "tc_common.cuh"

namespace crisp {

using namespace tc;
using namespace block8;

struct Plan8 {                               // launch plan for one activation buffer and number of columns
    const void *act;
    int64_t ncols;
    int box;                                 // columns a copy brings
    int chunks;                              // and chunks of 128 scales
    CUtensorMap map_x, map_s;
};

}  // namespace crisp

struct crisp_handle8_s {
    crisp::Geometry g;
    uint8_t *buf;
    crisp::Epilogue epilogue;
    int tile_cols, split;                    // tuning: columns a tile and CTAs that share one, -1 for pairs (0 = chosen by the library)
    unsigned long long wait_limit_cycles;
    int skip_fill;
    CUtensorMap map_a;
    bool maps;                               // map_a is there (a layer without kept blocks has none)
    std::mutex plan_lock;                    // of what follows
    crisp::Settled settled;                  // whether the next product may read the weights early
    crisp::Plan8 plan;
    crisp_launch_info_t last;
};

namespace crisp {

namespace {

struct Params8 {
    const int32_t *blk_col;
    int32_t *status;
    const uint16_t *x;                       // columns that are quantised here
    int64_t ldx;
    int k, x_layout, x_vec;
    void *y;
    const float *bias;
    int64_t ldy, ncols;
    int64_t groups, chunks;                  // of the activation buffer
    int rows, nrt, kkeep, num_tiles;
    int all;                                 // every block is kept: block e of the walk is block e
    int y_layout, f32, relu, vec_ok, stages, early;
    unsigned long long wait_limit;
    int skip_fill;
};

constexpr int kQuantisers = 8;

template <int N>
struct Tile8 {
    // Chunks of 128 columns' scales that a tile can touch: tiles begin at multiples of N, so that 64-column ones and those of 192 may begin in the middle of
    // one.  (The MMA takes the scales of B from an even column of tensor memory: a tile that began at an odd multiple of 32 raised a misaligned address.)
    static_assert(N % 64 == 0 || N <= 32, "wider tiles begin at multiples of 64");
    static constexpr int kChunks = N <= 128 ? 1 : 2;
    static constexpr int kAcc = N <= 192 ? 2 : 1;
    static constexpr int kScaleCols = 4 + 4 * kChunks;                // tensor memory columns of one set of scales
    static constexpr uint32_t kX = 17 * 1024;                         // codes of the columns in a stage, behind the weights
    static constexpr uint32_t kS = kX + N * 128;                      // their scales
    static constexpr uint32_t kStage = (kS + kChunks * kScales8 + 1023) / 1024 * 1024;
    static constexpr uint32_t kBytes = kEntry8 + N * 128 + kChunks * kScales8;
    static constexpr int kEpi = N >= 128 ? 8 : 4;                     // draining warps
    static constexpr int kUsed = kAcc * N + 2 * kScaleCols;
    static constexpr int kTmemCols = kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
    static constexpr uint32_t kStaging = 4096;                        // bytes a draining warp: 32 x 32 results of up to four bytes
    static_assert(kUsed <= 512, "tensor memory is 512 columns");
};

__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
// Instruction descriptor: e4m3 x e4m3, both K-major, E8M0 scales, M = 128.
__host__ __device__ constexpr uint32_t make_idesc8(int n) { return (1u << 23) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }

__device__ __forceinline__ float activation(float v, int relu) { return relu && v < 0.f ? 0.f : v; }         // (a NaN stays)

// One draining warp's 32 rows x 32 columns (lane = row, x[i] = column i), through its staging tile, so that the lanes write whole sectors.
template <bool kF32>
__device__ __forceinline__ void store_chunk8(const Params8 &p, uint8_t *stage, int lane, const float (&x)[32], int row0, int64_t col0) {
    constexpr int kSize = kF32 ? 4 : 2, kLine = 32 * kSize;          // bytes of a staged line: a row of Y's 32 elements
    constexpr int kVecs = kLine / 16;                                // 16-byte pieces of a line
    const int64_t cols = min((int64_t)32, p.ncols - col0);
    const int rows = min(32, p.rows - row0);
    __syncwarp();
    if (p.y_layout == 0) {
        // a lane has a line; its pieces are swizzled so that eight lanes' writes touch different banks
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            uint4 v;
            if constexpr (kF32) v = make_uint4(__float_as_uint(x[4 * j]), __float_as_uint(x[4 * j + 1]), __float_as_uint(x[4 * j + 2]), __float_as_uint(x[4 * j + 3]));
            else v = make_uint4(pack_bf16(x[8 * j], x[8 * j + 1]), pack_bf16(x[8 * j + 2], x[8 * j + 3]), pack_bf16(x[8 * j + 4], x[8 * j + 5]), pack_bf16(x[8 * j + 6], x[8 * j + 7]));
            *reinterpret_cast<uint4 *>(stage + lane * kLine + ((j ^ (kF32 ? lane & 7 : lane >> 1 & 3)) << 4)) = v;
        }
    } else {
        // a line is a column; the lanes write an element of it each
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if constexpr (kF32) *reinterpret_cast<float *>(stage + i * kLine + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4) = x[i];
            else *reinterpret_cast<__nv_bfloat16 *>(stage + i * kLine + (((lane >> 3) ^ (i >> 1 & 3)) << 4) + (lane & 7) * 2) = __float2bfloat16_rn(x[i]);
        }
    }
    __syncwarp();
    const int lines = p.y_layout == 0 ? rows : (int)cols, width = p.y_layout == 0 ? (int)cols : rows;
    uint8_t *y = reinterpret_cast<uint8_t *>(p.y) + (p.y_layout == 0 ? (int64_t)row0 * p.ldy + col0 : col0 * p.ldy + row0) * kSize;
    const int64_t pitch = p.ldy * kSize;
    if (p.vec_ok && width == 32) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = j * 32 + lane, line = i / kVecs, piece = i % kVecs;
            if (line < lines)
                *reinterpret_cast<uint4 *>(y + line * pitch + piece * 16) =
                    *reinterpret_cast<const uint4 *>(stage + line * kLine + ((piece ^ (kF32 ? line & 7 : line >> 1 & 3)) << 4));
        }
    } else {
        const auto staged = [&](int line, int e) -> const uint8_t * {
            return stage + line * kLine + (((e * kSize >> 4) ^ (kF32 ? line & 7 : line >> 1 & 3)) << 4) + (e * kSize & 15);
        };
        if (width < 32 || lines < 32) {                      // (a line a pass, the lanes side by side)
#pragma unroll 4
            for (int line = 0; line < lines; ++line)
                if (lane < width) {
                    if constexpr (kF32) *reinterpret_cast<float *>(y + line * pitch + lane * 4) = *reinterpret_cast<const float *>(staged(line, lane));
                    else *reinterpret_cast<uint16_t *>(y + line * pitch + lane * 2) = *reinterpret_cast<const uint16_t *>(staged(line, lane));
                }
        } else if constexpr (kF32) {
#pragma unroll 8
            for (int line = 0; line < 32; ++line) *reinterpret_cast<float *>(y + line * pitch + lane * 4) = *reinterpret_cast<const float *>(staged(line, lane));
        } else {
            // Two lines a pass, in pairs of elements that begin at a multiple of four bytes; of a line that does not begin at one an element at each end is left, which the
            // lanes store for all lines together.  (4096 x 3874 of one block: questions in the loop 33.6 us, now 21.5; pieces of 16 bytes 14.6.)
            const int half = lane >> 4, i = lane & 15;
            uint8_t *to = y + half * pitch;                   // (lines of one half begin alike)
            const int odd = (int)(reinterpret_cast<uintptr_t>(to) >> 1 & 1), e = 2 * i + odd;
            const bool pair = e < 31;
            to += e * 2;
#pragma unroll
            for (int it = 0; it < 16; ++it) {
                const uint32_t lo = *reinterpret_cast<const uint16_t *>(staged(2 * it + half, e)), hi = *reinterpret_cast<const uint16_t *>(staged(2 * it + half, (e + 1) & 31));
                if (pair) *reinterpret_cast<uint32_t *>(to) = lo | hi << 16;
                to += 2 * pitch;
            }
            uint16_t *line = reinterpret_cast<uint16_t *>(y + lane * pitch);
            if (reinterpret_cast<uintptr_t>(line) & 2u) {
                line[0] = *reinterpret_cast<const uint16_t *>(staged(lane, 0));
                line[31] = *reinterpret_cast<const uint16_t *>(staged(lane, 31));
            }
        }
    }
}

// Eight values of a column that the fused product quantises: k from `at` on.
__device__ __forceinline__ uint4 fetch8(const Params8 &p, int64_t col, int at) {
    uint32_t v[4] = {};
    if (p.x_layout == 1) {
        const uint16_t *x = p.x + col * p.ldx + at;
        if (p.x_vec && at + 8 <= p.k) return *reinterpret_cast<const uint4 *>(x);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at + j < p.k) v[j / 2] |= (uint32_t)x[j] << (16 * (j & 1));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at + j < p.k) v[j / 2] |= (uint32_t)p.x[(at + j) * p.ldx + col] << (16 * (j & 1));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// kSplit: the CTAs of a cluster share one tile, each walks a part of its blocks, and they add up their accumulators through distributed shared memory, in the
// order of their ranks.
// kFused: X is not in an activation buffer.  Eight warps fetch and quantise it on the way into the pipeline's stages, a whole stage (a k-block of all columns) each,
// so that the loads of eight stages are under way at once; each row tile's CTAs do that anew, which a few columns are worth (one launch less).
template <int N, bool kSplit, bool kFused>
__global__ void __launch_bounds__(32 * (2 + Tile8<N>::kEpi + (kFused ? kQuantisers : 2)), 1)
spmm8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_s,
             const __grid_constant__ Params8 p, int split) {
    using T = Tile8<N>;
    constexpr int kEpi = T::kEpi;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t ring = smem_u32(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t staging = ring + p.stages * T::kStage, ctrl = staging + kEpi * T::kStaging;
    uint8_t *ctrl_gen = smem_raw + (ctrl - ring);
    // barriers: full[s] and empty[s] (s < 12), accumulators full and empty
    const uint32_t bar_full = ctrl, bar_empty = ctrl + 96, bar_tfull = ctrl + 192, bar_tempty = ctrl + 208;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 224);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(ctrl_gen + 228);
    const bool aligned = (ring & 1023u) == 0;            // (swizzled operands need it; checked, not assumed)
    if (warp == 1) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), T::kTmemCols);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        if (p.kkeep > 0) prefetch_tensormap(&map_a);      // (else there are none)
        if (p.kkeep > 0 && !kFused) { prefetch_tensormap(&map_x); prefetch_tensormap(&map_s); }
        for (int s = 0; s < p.stages; ++s) { mbar_init(bar_full + 8 * s, kFused ? 2 : 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int a = 0; a < T::kAcc; ++a) { mbar_init(bar_tfull + 8 * a, 1); mbar_init(bar_tempty + 8 * a, kEpi); }
        *abort_flag = aligned ? 0 : 1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (p.early: the weights are there.  The kernel in front is the one that quantised X, which began when all before it had finished, or settled.h says so)
    if (!p.early) wait_for_prerequisites();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (p.early && warp != 0) wait_for_prerequisites();
    const int rank = kSplit ? (int)cluster_rank() : 0;
    const int tile0 = kSplit ? (int)blockIdx.x / split : (int)blockIdx.x, tile_step = kSplit ? p.num_tiles : (int)gridDim.x;
    // this CTA's part of a tile's blocks
    const int first = kSplit ? (int)((int64_t)p.kkeep * rank / split) : 0;
    const int len = (kSplit ? (int)((int64_t)p.kkeep * (rank + 1) / split) : p.kkeep) - first;

    // The threads that issue copies and MMAs are bound by their own instructions.  Their warps run the loops as a whole, so that addresses and descriptors stay in uniform
    // registers, where the instructions take them from, and an elected thread issues.  (Loops of one thread: 4096 x 4096, 512 columns 17.8 us instead of 12.9, 8192 columns 127 instead of
    // 116; a block of 64 columns 0.33 us instead of 0.2.)
    if (warp == 0) {
        // -------------------------------------------------- weights, and the byte count of a stage
        const bool leader = elect_one();
        uint32_t dst = ring, full = bar_full, empty = bar_empty, ph = 0;
        int s = 0, fill = 0;
        bool ok = true;
        for (int t = tile0; t < p.num_tiles && ok; t += tile_step) {
            int row = ((t % p.nrt) * p.kkeep + first) * (int)(kEntry8 / 256);
            for (int e = 0; e < len; ++e) {
                if (!wait_warp<true>(empty, ph ^ 1u, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                if (leader) {
                    mbar_expect_tx(full, kFused ? kEntry8 : T::kBytes);
                    if (fill != p.skip_fill) tma_load_2d(dst, &map_a, 0, row, full);
                }
                ++fill;
                row += kEntry8 / 256;
                dst += T::kStage; full += 8; empty += 8;
                if (++s == p.stages) { s = 0; dst = ring; full = bar_full; empty = bar_empty; ph ^= 1u; }
            }
        }
        wait_for_prerequisites();                        // (it may have had nothing to wait for; the other warps have waited)
    } else if (warp >= 2 + kEpi) {
        if constexpr (kFused) {
            // ---------------------------------------------- X: half a warp a column, eight values a lane
            constexpr int kPasses = N / 2, kAtOnce = kPasses < 8 ? kPasses : 8;
            const int half = lane >> 4, l16 = lane & 15;
            int s = warp - (2 + kEpi), e = s, t = tile0;         // this warp's next stage and entry
            uint32_t ph = 0;
            while (s >= p.stages) { s -= p.stages; ph ^= 1u; }
            bool ok = true;
            for (; t < p.num_tiles && ok; t += tile_step) {
                const int64_t c0 = (int64_t)(t / p.nrt) * N;
                const int cols = (int)min((int64_t)N, p.ncols - c0);
                const int32_t *list = p.blk_col + (int64_t)(t % p.nrt) * p.kkeep + first;
                for (; e < len; e += kQuantisers) {
                    const int at = (p.all ? first + e : __ldcg(list + e)) * 128 + l16 * 8;
                    uint8_t *stage = smem_raw + s * T::kStage;
                    bool waited = false;
#pragma unroll 1
                    for (int g = 0; g < kPasses && 2 * g < cols; g += kAtOnce) {
                        uint4 v[kAtOnce];
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            const int c = 2 * (g + i) + half;
                            v[i] = c < cols && at < p.k ? fetch8(p, c0 + c, at) : make_uint4(0, 0, 0, 0);
                        }
                        if (!waited) {
                            int go = 0;
                            if (lane == 0) go = mbar_wait(bar_empty + 8 * s, ph ^ 1u, abort_flag, p.wait_limit);
                            ok = __shfl_sync(0xFFFFFFFFu, go, 0) != 0;
                            waited = true;
                            if (!ok) break;
                        }
                        // (the passes side by side: their shuffles would otherwise wait for one another; two passes' largest values travel in a word)
                        uint32_t top[kAtOnce], word[kAtOnce / 2], any = 0;
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            top[i] = larger(larger(larger(larger(0, v[i].x), v[i].y), v[i].z), v[i].w);
                            any = __vmaxu2(any, top[i]);
                        }
                        if (__any_sync(0xFFFFFFFFu, larger_of(any) >= 0x7F80u)) {
#pragma unroll
                            for (int i = 0; i < kAtOnce; ++i) {
                                top[i] = larger(larger(larger(larger(0, finite(v[i].x)), finite(v[i].y)), finite(v[i].z)), finite(v[i].w));
                                v[i] = make_uint4(nan_for_infinity(v[i].x), nan_for_infinity(v[i].y), nan_for_infinity(v[i].z), nan_for_infinity(v[i].w));
                            }
                        }
#pragma unroll
                        for (int i = 0; i < kAtOnce / 2; ++i) word[i] = larger_of(top[2 * i]) | larger_of(top[2 * i + 1]) << 16;
#pragma unroll
                        for (int d = 8; d; d >>= 1)
#pragma unroll
                            for (int i = 0; i < kAtOnce / 2; ++i) word[i] = __vmaxu2(word[i], __shfl_xor_sync(0xFFFFFFFFu, word[i], d));
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            const int c = 2 * (g + i) + half;
                            if (c >= cols) break;
                            const uint32_t exponent = exponent_of(word[i / 2] >> (16 * (i & 1)) & 0xFFFFu);
                            const float down = power_of(254u - exponent);
                            *reinterpret_cast<uint2 *>(stage + T::kX + (c >> 3) * 1024 + (c & 7) * 128 + (((l16 >> 1) ^ (c & 7)) << 4) + (l16 & 1) * 8) =
                                make_uint2(codes2(v[i].x, down) | codes2(v[i].y, down) << 16, codes2(v[i].z, down) | codes2(v[i].w, down) << 16);
                            if (l16 == 0) *reinterpret_cast<uint32_t *>(stage + T::kS + (c & 31) * 16 + (c >> 5) * 4) = exponent * 0x01010101u;
                        }
                    }
                    if (!ok) break;
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_full + 8 * s);
                    s += kQuantisers;
                    while (s >= p.stages) { s -= p.stages; ph ^= 1u; }
                }
                e -= len;                                        // (stages are numbered through the tiles)
            }
        } else {
            // ---------------------------------------------- activations, and in a warp of its own their scales
            const bool leader = elect_one(), codes = warp == 2 + kEpi;
            constexpr int kAhead = 8;
            const uint32_t at = codes ? T::kX : T::kS;
            uint32_t dst = ring + at, full = bar_full, empty = bar_empty, ph = 0;
            int s = 0, fill = 0;
            bool ok = true;
            for (int t = tile0; t < p.num_tiles && ok; t += tile_step) {
                const int rt = t % p.nrt;
                const int64_t c0 = (int64_t)(t / p.nrt) * N;
                // rows of the map of a k-block, and of the tile's first column in it
                const int pitch = (int)(codes ? p.groups * 4 : p.chunks * 2), start = (int)(codes ? (c0 >> 3) * 4 : (c0 >> 7) * 2);
                const int32_t *cols = p.blk_col + (int64_t)rt * p.kkeep + first;
                int next[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) next[u] = u < len ? (p.all ? first + u : __ldcg(cols + u)) : 0;
                for (int e0 = 0; e0 < len && ok; e0 += kAhead) {
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int e = e0 + u;
                        if (e >= len) break;
                        const int row = next[u] * pitch + start;
                        if (e + kAhead < len) next[u] = p.all ? first + e + kAhead : __ldcg(cols + e + kAhead);
                        if (!wait_warp<false>(empty, ph ^ 1u, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                        if (leader && fill != p.skip_fill) {
                            if (codes) tma_load_2d(dst, &map_x, 0, row, full);
                            else tma_load_2d(dst, &map_s, 0, row, full);
                        }
                        ++fill;
                        dst += T::kStage; full += 8; empty += 8;
                        if (++s == p.stages) { s = 0; dst = ring + at; full = bar_full; empty = bar_empty; ph ^= 1u; }
                    }
                }
            }
        }
    } else if (warp == 1) {
        // -------------------------------------------------- scales to tensor memory, MMAs
        constexpr uint32_t idesc = make_idesc8(N);
        const bool leader = elect_one();
        const uint64_t a0 = make_smem_desc(ring, 16, 1024, kLayoutSw128), b0 = make_smem_desc(ring + T::kX, 16, 1024, kLayoutSw128);
        const uint64_t sa0 = make_smem_desc(ring + kTile8, 128, 128, kLayoutNone), sb0 = make_smem_desc(ring + T::kS, 128, 128, kLayoutNone);
        const uint32_t scales = tmem + T::kAcc * N;
        uint32_t off = 0, full = bar_full, empty = bar_empty, ph = 0, acc = 0, acc_ph = 0, set = 0;
        int s = 0;
        for (int t = tile0; t < p.num_tiles; t += tile_step) {
            const int64_t c0 = (int64_t)(t / p.nrt) * N;
            const uint32_t shift = (uint32_t)(c0 & 127) >> 5;                // of the tile's first column in its chunk of scales
            if (!wait_warp<false>(bar_tempty + 8 * acc, acc_ph ^ 1u, leader, abort_flag, p.wait_limit)) break;
            tc_fence_after();
            const uint32_t d = tmem + acc * N;
            bool ok = true;
            for (int e = 0; e < len; ++e) {
                if (!wait_warp<false>(full, ph, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                tc_fence_after();
                const uint32_t sa = scales + set * T::kScaleCols, sb = sa + 4;
                if (leader) {
                    copy_scales(sa, sa0 + off);
#pragma unroll
                    for (int c = 0; c < T::kChunks; ++c) copy_scales(sb + 4 * c, sb0 + off + c * (kScales8 >> 4));
#pragma unroll
                    for (int j = 0; j < 4; ++j) mma_scaled(d, a0 + off + 2 * j, b0 + off + 2 * j, idesc, sa, sb + shift, (uint32_t)(e | j));
                    mma_commit(empty);
                }
                set ^= 1u;
                off += T::kStage >> 4; full += 8; empty += 8;
                if (++s == p.stages) { s = 0; off = 0; full = bar_full; empty = bar_empty; ph ^= 1u; }
            }
            if (!ok) break;
            if (leader) mma_commit(bar_tfull + 8 * acc);
            if (++acc == T::kAcc) { acc = 0; acc_ph ^= 1u; }
        }
    } else {
        // -------------------------------------------------- drain: tensor memory -> registers -> Y (or this CTA's part of a sum)
        const int ew = warp - 2, q = warp & 3, part = ew >> 2;       // a warp may read the lanes of its quarter only
        uint8_t *stage = smem_raw + (staging - ring) + ew * T::kStaging;
        uint32_t acc = 0, acc_ph = 0;
        for (int t = tile0; t < p.num_tiles; t += tile_step) {
            const int row0 = (t % p.nrt) * 128 + 32 * q;
            const int64_t c0 = (int64_t)(t / p.nrt) * N;
            int go = 0;
            if (lane == 0) go = !*abort_flag && mbar_wait(bar_tfull + 8 * acc, acc_ph, abort_flag, p.wait_limit);
            go = __shfl_sync(0xFFFFFFFFu, go, 0);
            if (!go) break;
            tc_fence_after();
            const uint32_t from = tmem + acc * N + ((uint32_t)(32 * q) << 16);
            // the warp's whole share goes to registers first: the accumulator is free for the next tile while these are stored
            constexpr int kMine = N >= 32 ? N / 32 / (kEpi / 4) : 1;         // chunks of 32 columns, next to one another
            uint32_t r[kMine][32];
            if (len) {
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    if constexpr (N == 16) tmem_ld16(from, r[i]);
                    else tmem_ld32(from + 32 * (kMine * part + i), r[i]);
                }
                tmem_ld_wait();
            } else {
#pragma unroll
                for (int i = 0; i < kMine; ++i)
#pragma unroll
                    for (int j = 0; j < 32; ++j) r[i][j] = 0;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_tempty + 8 * acc);
            if (++acc == T::kAcc) { acc = 0; acc_ph ^= 1u; }
            const float bias = !kSplit && p.bias != nullptr && row0 + lane < p.rows ? p.bias[row0 + lane] : 0.f;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int c = 32 * (kMine * part + i);
                if constexpr (kSplit) {
                    // (every stage has been multiplied: the ring is free)
                    float *sum = reinterpret_cast<float *>(smem_raw);
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (N >= 32 || j < N) sum[(c + j) * 128 + 32 * q + lane] = __uint_as_float(r[i][j]);
                } else if (c0 + c < p.ncols && row0 < p.rows) {
                    float x[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = activation(__uint_as_float(r[i][j]) + bias, p.relu);
                    if (p.f32) store_chunk8<true>(p, stage, lane, x, row0, c0 + c);
                    else store_chunk8<false>(p, stage, lane, x, row0, c0 + c);
                }
            }
        }
    }
    __syncwarp();
    if constexpr (kSplit) {
        // (all threads of all CTAs come here, also where a wait has run out)
        cluster_arrive();
        cluster_wait();
        const int row0 = (tile0 % p.nrt) * 128;
        const int64_t c0 = (int64_t)(tile0 / p.nrt) * N;
        const int cols = (int)min((int64_t)N, p.ncols - c0);
        if (warp >= 2 && warp < 2 + kEpi) {
            // Four rows of a column at a time, the ranks' parts fetched together and added up in their order.
            const int me = (warp - 2) * 32 + lane, threads = 32 * kEpi;
            for (int i = rank * threads + me; i < cols * 32; i += split * threads) {
                const int c = i >> 5, r = (i & 31) * 4;
                float4 part[8];
#pragma unroll
                for (int s = 0; s < 8; ++s)
                    if (s < split) part[s] = lds128_peer(peer_address(ring + (c * 128 + r) * 4, s));
                float v[4] = {part[0].x, part[0].y, part[0].z, part[0].w};
#pragma unroll
                for (int s = 1; s < 8; ++s)
                    if (s < split) { v[0] += part[s].x; v[1] += part[s].y; v[2] += part[s].z; v[3] += part[s].w; }
                if (*abort_flag) break;
                uint32_t bits[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = row0 + r + j;
                    v[j] = activation(v[j] + (p.bias != nullptr && row < p.rows ? p.bias[row] : 0.f), p.relu);
                    bits[j] = __float_as_uint(v[j]);
                }
                const int64_t at = p.y_layout == 0 ? (row0 + r) * p.ldy + c0 + c : (c0 + c) * p.ldy + row0 + r;
                if (p.y_layout == 1 && p.vec_ok && row0 + r + 4 <= p.rows) {
                    if (p.f32) *reinterpret_cast<uint4 *>(reinterpret_cast<float *>(p.y) + at) = make_uint4(bits[0], bits[1], bits[2], bits[3]);
                    else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(p.y) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (row0 + r + j >= p.rows) break;
                        const int64_t to = at + j * (p.y_layout == 0 ? p.ldy : 1);
                        if (p.f32) reinterpret_cast<float *>(p.y)[to] = v[j];
                        else reinterpret_cast<__nv_bfloat16 *>(p.y)[to] = __float2bfloat16_rn(v[j]);
                    }
                }
            }
        }
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 1) launch_dependents();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicCAS(p.status, 0, (int)(aligned ? CRISP_TIMEOUT : CRISP_CUDA_ERROR));
        // copies that may still be in flight land before shared memory is released
        const unsigned long long t0 = clock64();
        while ((unsigned long long)(clock64() - t0) < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, T::kTmemCols);
    }
}

// ------------------------------------------------------------------------------------------------ pairs of SMs
//
// Where every block is kept, two row tiles walk the same list, and two CTAs (a cluster) multiply 256 rows by N columns with cta_group::2: each holds its row tile's
// weights and half of the columns, and the tensor cores of both read both halves.  What bounds the single CTA's MMAs is the operands they read from shared memory, 64
// bytes a cycle (128 x N x 32: 4 KB + 32 N bytes; 98, 118, 160 and 191 cycles measured for 64, 128, 192 and 256 columns where the products need 32, 64, 96 and 128); a
// pair reads half of the columns' bytes a CTA, and fetches half of them from L2.
//
// The CTA of rank 0 issues for both.  The copies of both complete on its barriers, which count the bytes of both (what has landed in the peer's shared memory is acquired
// at the scope of the cluster); commits go to both (multicast); accumulators are handed back by the draining warps of both.  These two are seen at the scope of the
// cluster, relaxed: what tcgen05 instructions read and write is ordered by their commits and fences, and nothing else is handed over.  (Accumulators released and acquired, a
// tile takes 0.35 us more; stages announced one by one by a warp of the peer, released at that scope, 4096 x 4096 x 8192 188 us.)
template <int N>
struct Pair8 {
    static constexpr int kChunks = N <= 128 ? 1 : 2;
    static constexpr int kAcc = N <= 192 ? 2 : 1;
    static constexpr int kScaleCols = 4 + 4 * kChunks;
    static constexpr uint32_t kX = 17 * 1024;
    static constexpr uint32_t kS = kX + N / 2 * 128;
    static constexpr uint32_t kStage = (kS + kChunks * kScales8 + 1023) / 1024 * 1024;
    static constexpr uint32_t kBytes = kEntry8 + N / 2 * 128 + kChunks * kScales8;
    static constexpr int kEpi = 8;
    static constexpr uint32_t kStaging = 4096;
    static constexpr uint32_t kFixed = kEpi * kStaging + 256;
    static constexpr int kMost = (int)((kSmemBudget - kFixed) / kStage), kStages = kMost < 12 ? kMost : 12;
    static_assert(kAcc * N + 2 * kScaleCols <= 512, "tensor memory is 512 columns");
    static_assert(N % 64 == 0 && N / 2 * 128 % 1024 == 0, "halves are whole atoms, and scales begin at even columns");
};

__device__ __forceinline__ void copy_scales_pair(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_scaled_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
template <int N>
__global__ void __launch_bounds__(32 * (4 + Pair8<N>::kEpi), 1)
spmm8_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_s,
                  const __grid_constant__ Params8 p, int) {
    using T = Pair8<N>;
    constexpr int kEpi = T::kEpi, kTmemCols = 512;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t ring = smem_u32(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t staging = ring + T::kStages * T::kStage, ctrl = staging + kEpi * T::kStaging;
    uint8_t *ctrl_gen = smem_raw + (ctrl - ring);
    // barriers: (rank 0) full[s] of both, and empty[s], s < 12; accumulators full, and (rank 0) empty
    const uint32_t bar_full = ctrl, bar_empty = ctrl + 96, bar_tfull = ctrl + 192, bar_tempty = ctrl + 208;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 224);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(ctrl_gen + 228);
    const uint32_t rank = cluster_rank(), full0 = peer_address(bar_full, 0);
    const bool aligned = (ring & 1023u) == 0;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t *>(tmem_slot))), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        prefetch_tensormap(&map_a); prefetch_tensormap(&map_x); prefetch_tensormap(&map_s);
        for (int s = 0; s < T::kStages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int a = 0; a < T::kAcc; ++a) { mbar_init(bar_tfull + 8 * a, 1); mbar_init(bar_tempty + 8 * a, 2 * kEpi); }
        *abort_flag = aligned ? 0 : 1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (!p.early) wait_for_prerequisites();
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                        // (the peer's barriers are there, and its tensor memory)
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (p.early && warp != 0) wait_for_prerequisites();
    const int pairs = (p.nrt + 1) >> 1, tile0 = (int)(blockIdx.x >> 1), tile_step = (int)(gridDim.x >> 1), len = p.kkeep;

    if (warp == 0) {
        // -------------------------------------------------- this CTA's weights (an odd number of row tiles: the last one's once more), and (rank 0) both CTAs' byte count
        const bool leader = elect_one();
        uint32_t dst = ring, full = full0, empty = bar_empty, ph = 0;
        int s = 0, fill = 0;
        bool ok = true;
        for (int t = tile0; t < p.num_tiles && ok; t += tile_step) {
            int row = min(2 * (t % pairs) + (int)rank, p.nrt - 1) * len * (int)(kEntry8 / 256);
            for (int e = 0; e < len; ++e) {
                if (!wait_warp<true>(empty, ph ^ 1u, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                mbar_seen_cluster<false>(empty, ph ^ 1u);
                if (leader) {
                    // (the peer's bytes may come first: a phase ends with this arrival at the earliest, and the peer fills a stage anew when the one before has been multiplied)
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, 2 * T::kBytes);
                    if (fill != p.skip_fill) tma_load_2d_pair(dst, &map_a, 0, row, full);
                }
                ++fill;
                row += kEntry8 / 256;
                dst += T::kStage; full += 8; empty += 8;
                if (++s == T::kStages) { s = 0; dst = ring; full = full0; empty = bar_empty; ph ^= 1u; }
            }
        }
        wait_for_prerequisites();
    } else if (warp >= 2 + kEpi) {
        // -------------------------------------------------- this CTA's half of the columns, and the scales of all of them
        const bool leader = elect_one(), codes = warp == 2 + kEpi;
        const uint32_t at = codes ? T::kX : T::kS;
        uint32_t dst = ring + at, full = full0, empty = bar_empty, ph = 0;
        int s = 0, fill = 0;
        bool ok = true;
        const int pitch = (int)(codes ? p.groups * 4 : p.chunks * 2);
        for (int t = tile0; t < p.num_tiles && ok; t += tile_step) {
            const int64_t c0 = (int64_t)(t / pairs) * N;
            int row = (int)(codes ? ((c0 >> 3) + rank * (N / 16)) * 4 : (c0 >> 7) * 2);
            for (int e = 0; e < len; ++e) {
                if (!wait_warp<false>(empty, ph ^ 1u, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                mbar_seen_cluster<false>(empty, ph ^ 1u);
                if (leader && fill != p.skip_fill) {
                    if (codes) tma_load_2d_pair(dst, &map_x, 0, row, full);
                    else tma_load_2d_pair(dst, &map_s, 0, row, full);
                }
                ++fill;
                row += pitch;
                dst += T::kStage; full += 8; empty += 8;
                if (++s == T::kStages) { s = 0; dst = ring + at; full = full0; empty = bar_empty; ph ^= 1u; }
            }
        }
    } else if (warp == 1 && rank == 0) {
        // -------------------------------------------------- scales to tensor memory and MMAs, of both CTAs
        constexpr uint32_t idesc = (1u << 23) | ((uint32_t)(N >> 3) << 17) | (16u << 24);       // as make_idesc8, M = 256
        const bool leader = elect_one();
        const uint64_t a0 = make_smem_desc(ring, 16, 1024, kLayoutSw128), b0 = make_smem_desc(ring + T::kX, 16, 1024, kLayoutSw128);
        const uint64_t sa0 = make_smem_desc(ring + kTile8, 128, 128, kLayoutNone), sb0 = make_smem_desc(ring + T::kS, 128, 128, kLayoutNone);
        const uint32_t scales = tmem + T::kAcc * N;
        uint32_t off = 0, ph = 0, acc = 0, acc_ph = 0, set = 0;
        int s = 0;
        for (int t = tile0; t < p.num_tiles; t += tile_step) {
            const uint32_t shift = (uint32_t)((int64_t)(t / pairs) * N & 127) >> 5;
            if (!wait_warp<false>(bar_tempty + 8 * acc, acc_ph ^ 1u, leader, abort_flag, p.wait_limit)) break;
            mbar_seen_cluster<false>(bar_tempty + 8 * acc, acc_ph ^ 1u);
            tc_fence_after();
            const uint32_t d = tmem + acc * N;
            bool ok = true;
            for (int e = 0; e < len; ++e) {
                if (!wait_warp<false>(bar_full + 8 * s, ph, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                mbar_seen_cluster<true>(bar_full + 8 * s, ph);
                tc_fence_after();
                const uint32_t sa = scales + set * T::kScaleCols, sb = sa + 4;
                if (leader) {
                    copy_scales_pair(sa, sa0 + off);
#pragma unroll
                    for (int c = 0; c < T::kChunks; ++c) copy_scales_pair(sb + 4 * c, sb0 + off + c * (kScales8 >> 4));
#pragma unroll
                    for (int j = 0; j < 4; ++j) mma_scaled_pair(d, a0 + off + 2 * j, b0 + off + 2 * j, idesc, sa, sb + shift, (uint32_t)(e | j));
                    mma_commit_pair(bar_empty + 8 * s);
                }
                set ^= 1u;
                off += T::kStage >> 4;
                if (++s == T::kStages) { s = 0; off = 0; ph ^= 1u; }
            }
            if (!ok) break;
            if (leader) mma_commit_pair(bar_tfull + 8 * acc);
            if (++acc == T::kAcc) { acc = 0; acc_ph ^= 1u; }
        }
    } else if (warp >= 2) {
        // -------------------------------------------------- drain: this CTA's row tile
        const int ew = warp - 2, q = warp & 3, part = ew >> 2;
        uint8_t *stage = smem_raw + (staging - ring) + ew * T::kStaging;
        const uint32_t back = peer_address(bar_tempty, 0);
        uint32_t acc = 0, acc_ph = 0;
        for (int t = tile0; t < p.num_tiles; t += tile_step) {
            const int row0 = (2 * (t % pairs) + (int)rank) * 128 + 32 * q;
            const int64_t c0 = (int64_t)(t / pairs) * N;
            int go = 0;
            if (lane == 0) go = !*abort_flag && mbar_wait(bar_tfull + 8 * acc, acc_ph, abort_flag, p.wait_limit);
            go = __shfl_sync(0xFFFFFFFFu, go, 0);
            if (!go) break;
            mbar_seen_cluster<false>(bar_tfull + 8 * acc, acc_ph);
            tc_fence_after();
            const uint32_t from = tmem + acc * N + ((uint32_t)(32 * q) << 16);
            constexpr int kMine = N / 64;
            uint32_t r[kMine][32];
#pragma unroll
            for (int i = 0; i < kMine; ++i) tmem_ld32(from + 32 * (kMine * part + i), r[i]);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(back + 8 * acc);
            if (++acc == T::kAcc) { acc = 0; acc_ph ^= 1u; }
            const float bias = p.bias != nullptr && row0 + lane < p.rows ? p.bias[row0 + lane] : 0.f;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int c = 32 * (kMine * part + i);
                if (c0 + c >= p.ncols || row0 >= p.rows) break;
                float x[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) x[j] = activation(__uint_as_float(r[i][j]) + bias, p.relu);
                if (p.f32) store_chunk8<true>(p, stage, lane, x, row0, c0 + c);
                else store_chunk8<false>(p, stage, lane, x, row0, c0 + c);
            }
        }
    }
    __syncwarp();
    if (warp == 1) launch_dependents();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicCAS(p.status, 0, (int)(aligned ? CRISP_TIMEOUT : CRISP_CUDA_ERROR));
        const unsigned long long t0 = clock64();             // (copies that may still be in flight land)
        while ((unsigned long long)(clock64() - t0) < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    cluster_arrive();                                        // neither CTA's memory is read by the other any more
    cluster_wait();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

typedef void (*Kernel8)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const Params8, int);

constexpr int kMaxDevices = 64;

struct Variant8 {
    Kernel8 kern;
    int threads, stages;
    uint32_t smem;
    std::atomic<bool> *configured;
};

template <int N, bool kSplit, bool kFused = false>
Variant8 make_variant8() {
    static std::atomic<bool> configured[kMaxDevices];
    using T = Tile8<N>;
    constexpr uint32_t fixed = T::kEpi * T::kStaging + 256;
    constexpr int most = (int)((kSmemBudget - fixed) / T::kStage), stages = most < 12 ? most : 12;
    // (a quantising warp goes from one of its stages to the next without looking at those between: it must not come round to one that has not been multiplied)
    static_assert(!kFused || stages >= kQuantisers, "more quantising warps than stages");
    return Variant8{spmm8_kernel<N, kSplit, kFused>, 32 * (2 + T::kEpi + (kFused ? kQuantisers : 2)), stages, stages * T::kStage + fixed, configured};
}

template <bool kSplit>
Variant8 variant8(int tile) {
    switch (tile) {
        case 16: return make_variant8<16, kSplit>();
        case 32: return make_variant8<32, kSplit>();
        case 64: return make_variant8<64, kSplit>();
        case 128: return make_variant8<128, kSplit>();
        case 192: return make_variant8<192, kSplit>();
        default: return make_variant8<256, kSplit>();
    }
}

template <int N>
Variant8 make_pair_variant8() {
    static std::atomic<bool> configured[kMaxDevices];
    using T = Pair8<N>;
    return Variant8{spmm8_pair_kernel<N>, 32 * (4 + T::kEpi), T::kStages, T::kStages * T::kStage + T::kFixed, configured};
}
Variant8 pair_variant8(int tile) { return tile == 128 ? make_pair_variant8<128>() : tile == 192 ? make_pair_variant8<192>() : make_pair_variant8<256>(); }

// The products that quantise X themselves, in every row tile's CTAs: one launch less for the host, which takes some 8 us for two in a row (4.7 for one), but not always
// less for the device.  In a row from the host and in a graph, us, so and quantised apart: 1024 x 1024, 8 tokens 5.9 and 8.0, in a graph 5.8 and 5.3; 4096 x 4096, half of
// the blocks, 8 tokens 6.8 and 8.0 (6.8 and 6.1), 12 tokens 7.2 and 8.0 (7.2 and 6.3), 16 tokens 7.6 and 8.1 (7.7 and 6.3), 32 tokens 9.5 and 8.2 (9.5 and 7.1); all blocks, 12
// tokens 8.6 and 8.9 (8.8 and 8.5), 16 tokens 9.3 and 8.9; 8192 x 8192, half, where a CTA has 16 blocks, 5 tokens 10.5 and 9.5 (10.5 and 8.8).  Of [k, ncols] a thread
// fetches its values one by one: 4096 x 4096, half, 5 columns 7.6 and 8.7 (7.2 and 8.1), 8 columns 8.4 and 8.4 (8.2 and 7.4).
bool fused8(const Geometry &g, int64_t ncols, int layout) { return ncols <= (layout ? 12 : 5) && (int64_t)g.nrt * g.kkeep <= 1536; }

// How many clusters of s CTAs, one an SM, run at once: fewer than SMs / s, since a cluster lies within one GPC.  (A second wave for two of sixteen clusters of eight
// made 2048 x 2048 with one column 10.2 us instead of 5.7.)
int clusters_at_once(int device, int s, int sms) {
    static std::atomic<int> known[kMaxDevices][9];
    int n = known[device][s].load(std::memory_order_relaxed);
    if (n > 0) return n;
    const Variant8 v = make_variant8<64, true>();
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)s; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(s * (sms / s)));
    cfg.blockDim = dim3((unsigned)v.threads);
    cfg.dynamicSmemBytes = v.smem;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(reinterpret_cast<const void *>(v.kern), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget + 1024) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, reinterpret_cast<const void *>(v.kern), &cfg) != cudaSuccess || n <= 0) {
        (void)cudaGetLastError();
        n = std::max(1, sms / s - (s > 2 ? 2 : 0));
    }
    known[device][s].store(n, std::memory_order_relaxed);
    return n;
}

// Tiles that begin within a chunk of scales do so at an even multiple of 32 columns: the narrow ones are for a single tile.
bool fits8(int tile, int64_t ncols) { return tile >= 64 || ncols <= tile; }

// Columns a tile and CTAs that share one: the pair that takes the least time by a model of it, in us.  A block takes a CTA as long as its copies and MMAs, a tile a
// fixed time beside them, the sum over a cluster one that grows with the columns a CTA has to add up; tiles come in waves of as many as there are SMs.  Measured on
// 4096 x 4096 in a row, all blocks kept: 64 columns a tile 11.7 us for 128 tiles (256 columns) and 206 for 28 waves (8192), 128 columns 12.9 and 128, 192 columns
// 15.2 and 115, 256 columns 19.6 and 116; two, four CTAs a tile: 64 columns 11.6, 9.3, 128 columns 12.6, 9.9, 256 columns 18.9, 11.6.
void choose8(const crisp_handle8_s *h, int64_t ncols, int device, int *tile, int *split, bool *pair) {
    const int sms = sm_count_of(device);
    struct Cost { int cols; double block, tile; };
    static const Cost costs[] = {{16, 0.17, 0.5}, {32, 0.17, 0.5}, {64, 0.20, 0.6}, {128, 0.24, 0.8}, {192, 0.31, 1.0}, {256, 0.43, 1.4}};
    const Geometry &g = h->g;
    double best = 1e300;
    *tile = 64; *split = 1; *pair = false;
    for (const Cost &c : costs) {
        if (!fits8(c.cols, ncols) || (h->tile_cols && fits8(h->tile_cols, ncols) && c.cols != h->tile_cols)) continue;
        const int64_t tiles = (int64_t)g.nrt * ((ncols + c.cols - 1) / c.cols);
        for (int s = 1; s <= 8 && s <= std::max(1, g.kkeep); ++s) {
            if (h->split > 0 ? s != std::min(h->split, std::max(1, g.kkeep)) : s > 1 && (tiles > clusters_at_once(device, s, sms) || 2 * s > g.kkeep)) continue;
            const double waves = (double)((tiles * s + sms - 1) / sms);
            const double t = waves * (c.block * ((g.kkeep + s - 1) / s) + c.tile) + (s > 1 ? 0.9 + c.cols / (48.0 * s) : 0.0);
            if (t < best) { best = t; *tile = c.cols; *split = s; }
        }
    }
    if (g.kkeep < g.nblk || g.nrt < 2 || h->split > 0) return;
    static const Cost pairs[] = {{128, 0.22, 1.0}, {192, 0.26, 1.5}, {256, 0.30, 2.0}};
    if (h->split == -1) best = 1e300;
    for (const Cost &c : pairs) {
        if (h->tile_cols && h->tile_cols != c.cols && h->tile_cols >= 128) continue;
        const int64_t tiles = (int64_t)((g.nrt + 1) / 2) * ((ncols + c.cols - 1) / c.cols);
        const double waves = (double)((tiles + sms / 2 - 1) / (sms / 2)), t = waves * (c.block * g.kkeep + c.tile);
        if (t < best && (h->split == -1 || !h->tile_cols)) { best = t; *tile = c.cols; *split = 1; *pair = true; }
    }
}

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// A buffer as rows of 256 bytes, loaded `rows` at a time, as it lies.
bool make_map_bytes(CUtensorMap *map, const void *base, uint64_t bytes, uint32_t rows) { return make_map_image(map, base, bytes, rows * 256); }

crisp_status_t check_product(crisp_handle8_s *h, const void *d_act, bool fused, int64_t ncols, const void *d_y, int64_t ldy, int32_t y_layout, int32_t y_dtype) {
    if (!h || (!d_act && !fused) || !d_y || (y_layout != 0 && y_layout != 1) || (y_dtype != 0 && y_dtype != 1)) return CRISP_INVALID_ARG;
    if (ncols <= 0 || ldy < (y_layout ? h->g.rows : ncols)) return CRISP_BAD_SHAPE;
    if (!aligned_to(d_act, kAlign) || !aligned_to(d_y, y_dtype ? 4 : 2)) return CRISP_INVALID_ARG;
    // (a buffer's rows of 256 bytes are numbered in 31 bits, and so are tiles)
    const Act8 a = act8(h->g.k, ncols);
    if (a.total / 256 >= (1ull << 31) - 4096 || (int64_t)h->g.nrt * ((ncols + 15) / 16) > 0x7FFFFFFFll) return CRISP_UNSUPPORTED;
    return CRISP_OK;
}

// x: what the product quantises itself (fused8); else nullptr, and d_act holds the codes, which the kernel in front wrote if `behind`.
cudaError_t launch_spmm8(crisp_handle8_s *h, const uint16_t *x, int64_t ldx, int x_layout, const void *d_act, bool behind, int64_t ncols, void *d_y, int64_t ldy,
                         int y_layout, int y_dtype, uint64_t moment, cudaStream_t st) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device < 0 || device >= kMaxDevices) return cudaErrorInvalidDevice;
    const Geometry &g = h->g;
    const auto settle = [&](const crisp_launch_info_t &info) {                   // (under the lock)
        h->last = info;
        if (h->settled.holds(st, moment)) return;
        // (what is captured has not run; one name of a stream stands for another stream in every thread)
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        h->settled.note(st, moment, st != cudaStreamPerThread && cudaStreamIsCapturing(st, &capture) == cudaSuccess && capture == cudaStreamCaptureStatusNone);
    };
    if (x && few8(g, ncols) && !h->tile_cols && !h->split && h->skip_fill < 0) {
        const Image8 I = image8(g);
        FewParams p{h->buf + I.image_off, reinterpret_cast<const int32_t *>(h->buf + I.col_off), x, d_y, h->epilogue.bias, ldx, ldy, g.rows, g.k, g.kkeep,
                    g.kkeep == g.nblk, (int)ncols, x_layout, aligned_to(x, 16) && ldx % 8 == 0, y_layout, y_dtype, h->epilogue.relu, 0};
        {
            std::lock_guard<std::mutex> hold(h->plan_lock);
            p.early = h->settled.holds(st, moment);
        }
        e = launch_product(encodes, p, moment, [&] { return launch_few8(p, g.nrt, device, st); });
        if (e == cudaSuccess) {
            std::lock_guard<std::mutex> hold(h->plan_lock);
            settle(crisp_launch_info_t{CRISP_PATH_DIRECT, 0, 0, 1, 0, 0, g.nrt * 16, 0, 1});
        }
        return e;
    }
    int tile, split;
    bool pair;
    choose8(h, ncols, device, &tile, &split, &pair);
    if (x) { tile = 16; pair = false; }
    const Act8 a = act8(g.k, ncols);
    const Variant8 v = pair ? pair_variant8(tile) : x ? (split > 1 ? make_variant8<16, true, true>() : make_variant8<16, false, true>()) : split > 1 ? variant8<true>(tile) : variant8<false>(tile);
    if (!v.configured[device].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(reinterpret_cast<const void *>(v.kern), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget + 1024);
        if (e != cudaSuccess) return e;
        v.configured[device].store(true, std::memory_order_relaxed);
    }
    Plan8 plan;
    Params8 p{};
    const int box = pair ? tile / 2 : tile, chunks = tile <= 128 ? 1 : 2;
    {
        std::lock_guard<std::mutex> hold(h->plan_lock);
        plan = h->plan;
        p.early = behind || h->settled.holds(st, moment);
    }
    if (g.kkeep > 0 && !x && (plan.act != d_act || plan.ncols != ncols || plan.box != box || plan.chunks != chunks)) {
        e = ensure_context(device);
        if (e != cudaSuccess) return e;
        plan.act = d_act; plan.ncols = ncols; plan.box = box; plan.chunks = chunks;
        if (!make_map_bytes(&plan.map_x, d_act, a.scale_off, box / 2) ||
            !make_map_bytes(&plan.map_s, reinterpret_cast<const uint8_t *>(d_act) + a.scale_off, a.total - a.scale_off, 2 * chunks))
            return cudaErrorInvalidValue;
        std::lock_guard<std::mutex> hold(h->plan_lock);
        h->plan = plan;
    }
    const Image8 I = image8(g);
    p.x = x; p.ldx = ldx; p.x_layout = x_layout; p.k = g.k; p.x_vec = aligned_to(x, 16) && ldx % 8 == 0;
    p.all = g.kkeep == g.nblk;
    p.blk_col = reinterpret_cast<const int32_t *>(h->buf + I.col_off);
    p.status = reinterpret_cast<int32_t *>(h->buf);
    p.y = d_y; p.bias = h->epilogue.bias; p.ldy = ldy; p.ncols = ncols; p.groups = a.groups; p.chunks = a.chunks;
    p.rows = g.rows; p.nrt = g.nrt; p.kkeep = g.kkeep;
    p.num_tiles = (int)((int64_t)(pair ? (g.nrt + 1) / 2 : g.nrt) * ((ncols + tile - 1) / tile));
    p.y_layout = y_layout; p.f32 = y_dtype; p.relu = h->epilogue.relu;
    const int size = y_dtype ? 4 : 2;
    p.vec_ok = aligned_to(d_y, 16) && ldy * size % 16 == 0;
    p.stages = v.stages;
    p.wait_limit = h->wait_limit_cycles ? h->wait_limit_cycles : kWaitLimitCycles;
    p.skip_fill = h->skip_fill;
    const int sms = sm_count_of(device);
    const unsigned grid = (unsigned)(pair ? 2 * std::min(p.num_tiles, sms / 2) : split > 1 ? p.num_tiles * split : std::min(p.num_tiles, sms));
    const auto launch = [&] { return launch_clusters(v.kern, grid, (unsigned)v.threads, v.smem, st, pair ? 2u : (unsigned)split, h->map_a, plan.map_x, plan.map_s, p, split); };
    e = behind ? launch() : launch_product(encodes, p, moment, launch);
    if (e == cudaSuccess) {
        std::lock_guard<std::mutex> hold(h->plan_lock);
        settle(crisp_launch_info_t{CRISP_PATH_DENSE, tile, tile <= 192 ? 2 : 1, pair ? -1 : split, tile >= 128 ? 8 : 4, v.stages, (int32_t)grid, 0, 1});
    }
    return e;
}

}  // namespace

}  // namespace crisp

extern "C" {

using namespace crisp;

crisp_status_t crisp_encode8_sizes(crisp_mask_t mask, size_t *bytes) {
    if (!mask || !bytes) return CRISP_INVALID_ARG;
    if (mask->g.bm != 128 || mask->g.bk != 128) return CRISP_UNSUPPORTED;
    const Image8 I = image8(mask->g);
    if (I.total / 256 >= (1ull << 31)) return CRISP_UNSUPPORTED;
    *bytes = I.total;
    return CRISP_OK;
}

crisp_status_t crisp_encode8(const uint16_t *d_w_bf16, int64_t ld_w, crisp_mask_t mask, void *d_buf, void *stream, crisp_handle8_t *out) {
    if (!out) return CRISP_INVALID_ARG;
    *out = nullptr;
    size_t bytes = 0;
    const crisp_status_t bad = crisp_encode8_sizes(mask, &bytes);
    if (bad != CRISP_OK) return bad;
    if (!d_w_bf16 || !d_buf || !aligned_to(d_w_bf16, 2) || !aligned_to(d_buf, kAlign)) return CRISP_INVALID_ARG;
    const Geometry &g = mask->g;
    if (ld_w < g.k) return CRISP_BAD_SHAPE;
    std::unique_ptr<crisp_handle8_s> h(new (std::nothrow) crisp_handle8_s);
    if (!h) return CRISP_CUDA_ERROR;
    h->g = g;
    h->buf = reinterpret_cast<uint8_t *>(d_buf);
    h->epilogue = Epilogue{nullptr, 0};
    h->tile_cols = h->split = 0;
    h->wait_limit_cycles = 0;
    h->skip_fill = -1;
    std::memset(&h->plan, 0, sizeof h->plan);
    std::memset(&h->map_a, 0, sizeof h->map_a);
    h->last = crisp_launch_info_t{-1, 0, 0, 1, 0, 0, 0, 0, 1};
    h->maps = (int64_t)g.nrt * g.kkeep > 0;
    if (h->maps) {
        int device = 0;
        if (cudaGetDevice(&device) != cudaSuccess || ensure_context(device) != cudaSuccess) return CRISP_CUDA_ERROR;
        const Image8 I = image8(g);
        if (!make_map_image(&h->map_a, h->buf + I.image_off, I.total - I.image_off, kEntry8)) return CRISP_CUDA_ERROR;
    }
    if (launch_encode8(g, d_w_bf16, ld_w, mask->d_blk_col, mask->d_nm_bits, h->buf, (cudaStream_t)stream) != cudaSuccess) return CRISP_CUDA_ERROR;
    *out = h.release();
    return CRISP_OK;
}

crisp_status_t crisp_decode8(crisp_handle8_t h, uint16_t *d_w_dense_bf16, int64_t ld, void *stream) {
    if (!h || !d_w_dense_bf16 || !aligned_to(d_w_dense_bf16, 2)) return CRISP_INVALID_ARG;
    if (ld < h->g.k) return CRISP_BAD_SHAPE;
    return launch_decode8(h->g, h->buf, d_w_dense_bf16, ld, (cudaStream_t)stream) == cudaSuccess ? CRISP_OK : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_quantize8_sizes(int64_t k, int64_t ncols, size_t *bytes) {
    if (!bytes) return CRISP_INVALID_ARG;
    if (k <= 0 || ncols <= 0) return CRISP_BAD_SHAPE;
    if (k > (int64_t)kMaxBlocksPerRowTile * 128 || ncols > ((int64_t)1 << 40)) return CRISP_UNSUPPORTED;
    const Act8 a = act8(k, ncols);
    if (a.total / 256 >= (1ull << 31) - 4096) return CRISP_UNSUPPORTED;
    *bytes = a.total;
    return CRISP_OK;
}

static crisp_status_t check_quantize(const uint16_t *d_x, int64_t ldx, int32_t x_layout, int64_t k, int64_t ncols, const void *d_act, bool fused = false) {
    size_t bytes = 0;
    const crisp_status_t bad = crisp_quantize8_sizes(k, ncols, &bytes);
    if (bad != CRISP_OK) return bad;
    if (!d_x || (!d_act && !fused) || (x_layout != 0 && x_layout != 1) || !aligned_to(d_x, 2) || !aligned_to(d_act, kAlign)) return CRISP_INVALID_ARG;
    return ldx < (x_layout ? k : ncols) ? CRISP_BAD_SHAPE : CRISP_OK;
}

static crisp_status_t quantize(const uint16_t *d_x, int64_t ldx, int32_t x_layout, int64_t k, int64_t ncols, void *d_act, const uint8_t *used, void *stream) {
    const cudaError_t e = launch_quantize8(d_x, ldx, x_layout, k, ncols, reinterpret_cast<uint8_t *>(d_act), used, (cudaStream_t)stream);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_quantize8(const uint16_t *d_x_bf16, int64_t ldx, int32_t x_layout, int64_t k, int64_t ncols, void *d_act, void *stream) {
    const crisp_status_t bad = check_quantize(d_x_bf16, ldx, x_layout, k, ncols, d_act);
    return bad != CRISP_OK ? bad : quantize(d_x_bf16, ldx, x_layout, k, ncols, d_act, nullptr, stream);
}

crisp_status_t crisp_dequantize8(const void *d_act, int32_t y_layout, int64_t k, int64_t ncols, uint16_t *d_y_bf16, int64_t ldy, void *stream) {
    const crisp_status_t bad = check_quantize(d_y_bf16, ldy, y_layout, k, ncols, d_act);
    if (bad != CRISP_OK) return bad;
    const cudaError_t e = launch_dequantize8(reinterpret_cast<const uint8_t *>(d_act), y_layout, k, ncols, d_y_bf16, ldy, (cudaStream_t)stream);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_spmm8_quantized(crisp_handle8_t h, const void *d_act, int64_t ncols, void *d_y, int64_t ldy, int32_t y_layout, int32_t y_dtype,
                                     void *stream) {
    const uint64_t moment = encodes.now();
    const crisp_status_t bad = check_product(h, d_act, false, ncols, d_y, ldy, y_layout, y_dtype);
    if (bad != CRISP_OK) return bad;
    return launch_spmm8(h, nullptr, 0, 0, d_act, false, ncols, d_y, ldy, y_layout, y_dtype, moment, (cudaStream_t)stream) == cudaSuccess ? CRISP_OK : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_spmm8_sizes(crisp_handle8_t h, int64_t ncols, size_t *act_bytes) {
    if (!h || !act_bytes) return CRISP_INVALID_ARG;
    const crisp_status_t bad = crisp_quantize8_sizes(h->g.k, ncols, act_bytes);
    if (bad == CRISP_OK && fused8(h->g, ncols, 0) && fused8(h->g, ncols, 1)) *act_bytes = 0;
    return bad;
}

crisp_status_t crisp_spmm8(crisp_handle8_t h, const uint16_t *d_x_bf16, int64_t ldx, int32_t x_layout, int64_t ncols, void *d_act, void *d_y, int64_t ldy,
                           int32_t y_layout, int32_t y_dtype, void *stream) {
    const uint64_t moment = encodes.now();
    const bool fused = h && fused8(h->g, ncols, x_layout);
    crisp_status_t bad = check_product(h, d_act, fused, ncols, d_y, ldy, y_layout, y_dtype);
    if (bad == CRISP_OK) bad = check_quantize(d_x_bf16, ldx, x_layout, h->g.k, ncols, d_act, fused);
    // (what no row tile keeps is neither read nor quantised)
    const bool some = h && h->g.kkeep > 0 && h->g.kkeep < h->g.nblk;
    if (bad == CRISP_OK && !fused && h->g.kkeep > 0)
        bad = quantize(d_x_bf16, ldx, x_layout, h->g.k, ncols, d_act, some ? h->buf + image8(h->g).used_off : nullptr, stream);
    if (bad != CRISP_OK) return bad;
    const cudaError_t e = launch_spmm8(h, fused ? d_x_bf16 : nullptr, ldx, x_layout, d_act, !fused && h->g.kkeep > 0, ncols, d_y, ldy, y_layout, y_dtype, moment, (cudaStream_t)stream);
    return e == cudaSuccess ? CRISP_OK : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_set_epilogue8(crisp_handle8_t h, const float *d_bias_f32, int32_t relu) {
    if (!h || (relu != 0 && relu != 1) || !aligned_to(d_bias_f32, 4)) return CRISP_INVALID_ARG;
    h->epilogue = Epilogue{d_bias_f32, relu};
    return CRISP_OK;
}

crisp_status_t crisp_last_launch8(crisp_handle8_t h, crisp_launch_info_t *out) {
    if (!h || !out) return CRISP_INVALID_ARG;
    std::lock_guard<std::mutex> hold(h->plan_lock);
    *out = h->last;
    return CRISP_OK;
}

crisp_status_t crisp_device_status8(crisp_handle8_t h, void *stream, int32_t *status_out) {
    if (!h || !status_out) return CRISP_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(status_out, h->buf, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess) return CRISP_CUDA_ERROR;
    return cudaStreamSynchronize(st) == cudaSuccess ? CRISP_OK : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_reset_status8(crisp_handle8_t h, void *stream) {
    if (!h) return CRISP_INVALID_ARG;
    return cudaMemsetAsync(h->buf, 0, sizeof(int32_t), (cudaStream_t)stream) == cudaSuccess ? CRISP_OK : CRISP_CUDA_ERROR;
}

crisp_status_t crisp_set_tuning8(crisp_handle8_t h, int32_t tile_cols, int32_t split, uint64_t wait_limit_cycles, int32_t skip_fill) {
    if (!h || skip_fill < -1 || split < -1 || split > 8) return CRISP_INVALID_ARG;
    if (tile_cols != 0 && tile_cols != 16 && tile_cols != 32 && tile_cols != 64 && tile_cols != 128 && tile_cols != 192 && tile_cols != 256) return CRISP_INVALID_ARG;
    h->tile_cols = tile_cols;
    h->split = split;
    h->wait_limit_cycles = wait_limit_cycles;
    h->skip_fill = skip_fill;
    return CRISP_OK;
}

void crisp_destroy8(crisp_handle8_t h) { delete h; }

}  // extern "C"
