// The weight gradient of a layer from its activations in 8 bits, dW[r, k] = sum over tokens t of dY[t, r] x[t, k], x = code * 2^E.
//
// The sum runs over tokens, and a block's scale belongs to one token: it cannot be taken out of the sum, so the tensor cores' block scaling does not apply.  But a code times a
// power of two is exact in bf16: x goes back to bf16 (a pass over it, in the caller's workspace), and the product is one of bf16 with fp32 accumulators.  Tokens are the
// slow dimension of both operands (dY [tokens, rows], NHWC; x as it was dequantised), and tcgen05 takes them that way round: no transposition.
//
// A CTA takes 128 rows by up to four boxes of 64 columns of dW (a box lies within one filter tap) and a part of the tokens, 64 at a time: a box of output pixels for a
// convolution, whose x is the same box shifted by the tap (TMA fills in the padding).  Under a mask of 128 x 128 blocks the boxes are those of the row tile's kept blocks.
//
// The accumulators in tensor memory lose what is shifted out (measured: 1.1e-9 of the result for each token), so that chains are kept short: after 512 tokens eight warps
// add the accumulator to sums in registers, rounding to nearest, while the next chain runs in the other accumulator.  Parts of the tokens are added by a second kernel, in their order.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "block8.h"
#include "tc_common.cuh"

namespace crisp {

using namespace tc;

namespace {

constexpr int kStep = 64;                                     // tokens a stage
constexpr int kChain = 8;                                     // stages a chain
constexpr int kBoxes = 4;                                     // boxes of 64 columns a tile, at most
constexpr int kDrain = 8;                                     // warps
constexpr int kGradThreads = 128 + 32 * kDrain;
constexpr uint32_t kABytes = 16384, kBoxBytes = 8192, kStage = kABytes + kBoxes * kBoxBytes;
constexpr int kStages = 4;
constexpr size_t kStaging = kDrain * 32 * 17 * 4;             // (16 columns of a warp's rows, where dW is not written in 16-byte pieces)
constexpr size_t kGradSmem = kStages * kStage + 256 + kStaging + 1024;
constexpr int kMaps = 16;                                     // tensor maps of x, at most

struct Grad {
    int rows, channels, kernel_w, pad, linear;
    int cboxes;                                               // boxes of a tap's channels (one tap under a list: of its blocks, whose last box may lie behind the last channel)
    int per, tiles_row, boxes, splits, items;                 // boxes a tile, tiles a row tile, boxes a row tile
    int tw, th, tb, nx, ny;                                   // pixels of a stage; boxes of them along a line, lines along an image
    int wo, ho;                                               // of dY (a linear layer: one line of tokens)
    int narrow, low, width0, height0;                         // columns and lines of taps with a map of their own, and what the first ones' maps show of the images
    int chunks, chunks_split;
    const int32_t *blk_col;                                   // masks of 128 x 128: kept blocks of a row tile (else nullptr)
    int kkeep;
    const uint32_t *nm_bits;                                  // a mask, or nullptr
    int wpr;
    int zero_row, zeros, zero_k, zero_warps;                              // blocks a row tile and in all that are to be looked at for zeros (0: none), columns of dW
    void *dw;
    int64_t ld;
    int f32, accumulate, vec;
    float *partial;                                           // splits > 1: [item][256 columns][128 rows]
    int32_t *status;
    unsigned long long wait_limit;
    int skip_fill;
};

// Box i of a row tile's list: its first column within a tap, and the tap.
struct BoxAt { int tap, c; };
__device__ __forceinline__ BoxAt box_at(const Grad &p, int rt, int i) {
    const int b = p.blk_col ? 2 * p.blk_col[(int64_t)rt * p.kkeep + (i >> 1)] + (i & 1) : i;
    if (p.linear) return {0, b * 64};
    const int tap = b / p.cboxes;
    return {tap, (b - tap * p.cboxes) * 64};
}

// Boxes of pixels run past the output's last column and line, where dY is zeros.  x there has to be zeros, too, and not what the images hold behind the last pixel that a tap covers: 0 times
// NaN would reach a weight in whose sum that pixel is not.  So the taps left of (above) the last ones that end inside the padding have maps that show no more of the images than they cover,
// the first tap width0 x height0 pixels, the next one a column (line) more.
template <int kCount>
struct MapsOfX { CUtensorMap of[kCount]; };

// Box i as it is copied: its map, first column and shift.
struct From { const CUtensorMap *map; int c, dx, dy; };
template <int kCount>
__device__ __forceinline__ From from_of(const Grad &p, const MapsOfX<kCount> &maps, const BoxAt &at) {
    if (p.linear) return {&maps.of[0], at.c, 0, 0};
    const int i = at.tap / p.kernel_w, j = at.tap - i * p.kernel_w;
    if constexpr (kCount == 1) return {&maps.of[0], at.c, j - p.pad, i - p.pad};
    const bool nothing = (j < p.narrow && p.width0 + j <= 0) || (i < p.low && p.height0 + i <= 0);
    return {&maps.of[min(i, p.low) * (p.narrow + 1) + min(j, p.narrow)], nothing ? p.cboxes * 64 : at.c, j - p.pad, i - p.pad};
}

__device__ __forceinline__ uint32_t mask_bits(const Grad &p, int row, int col) {      // 32 columns from `col` on
    const uint32_t *w = p.nm_bits + (int64_t)row * p.wpr;
    const int i = col >> 5;
    return __funnelshift_r(i < p.wpr ? w[i] : 0u, i + 1 < p.wpr ? w[i + 1] : 0u, col & 31);
}

// 16 sums of each of a warp's 32 rows to dW: in 16-byte pieces by the lanes that have them; or, where they do not lie at multiples of that, through the warp's staging rows, so that
// a store covers pieces of two rows (4096 x 4095 in fp32, 16 tokens: 45 us; with an element a lane, each in a row of its own, 103).
constexpr int kStaged = 17;
__device__ __forceinline__ void store16(const Grad &p, float *stage, int row0, int lane, int col, int n, float (&v)[16]) {
    const int row = row0 + lane;
    if (p.nm_bits && row < p.rows) {
        const uint32_t bits = mask_bits(p, row, col);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (!(bits >> j & 1u)) v[j] = 0.f;                // (a choice: what is not finite is gone, too)
    }
    if (!(p.vec && n == 16 && (col & (p.f32 ? 3 : 7)) == 0)) {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 16; ++j) stage[lane * kStaged + j] = v[j];
        __syncwarp();
        const int j = lane & 15;
#pragma unroll 8
        for (int r = lane >> 4; r < 32; r += 2) {
            const int row = row0 + r;
            if (row >= p.rows || j >= n) continue;
            const float x = stage[r * kStaged + j];
            const int64_t at = (int64_t)row * p.ld + col + j;
            if (p.f32) {
                float *to = reinterpret_cast<float *>(p.dw) + at;
                *to = p.accumulate ? *to + x : x;
            } else {
                __nv_bfloat16 *to = reinterpret_cast<__nv_bfloat16 *>(p.dw) + at;
                *to = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*to) + x : x);
            }
        }
        return;
    }
    if (row >= p.rows) return;
    const int64_t at = (int64_t)row * p.ld + col;
    if (p.f32) {
        float *to = reinterpret_cast<float *>(p.dw) + at;
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            float4 q = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            if (p.accumulate) {
                const float4 o = *reinterpret_cast<const float4 *>(to + j);
                q.x += o.x; q.y += o.y; q.z += o.z; q.w += o.w;
            }
            *reinterpret_cast<float4 *>(to + j) = q;
        }
    } else {
        __nv_bfloat16 *to = reinterpret_cast<__nv_bfloat16 *>(p.dw) + at;
#pragma unroll
        for (int j = 0; j < 16; j += 8) {
            uint4 q = make_uint4(0, 0, 0, 0);
            if (p.accumulate) q = *reinterpret_cast<const uint4 *>(to + j);
            const uint32_t o[4] = {q.x, q.y, q.z, q.w};
            uint32_t r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a = v[j + 2 * i], b = v[j + 2 * i + 1];
                if (p.accumulate) { a += __uint_as_float(o[i] << 16); b += __uint_as_float(o[i] & 0xFFFF0000u); }
                r[i] = pack_bf16(a, b);
            }
            *reinterpret_cast<uint4 *>(to + j) = make_uint4(r[0], r[1], r[2], r[3]);
        }
    }
}

__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}

// The first pixel of a chunk.  (The threads that issue copies are bound by their own instructions: they go from chunk to chunk without a division.  4096 x 4096, 8192 tokens,
// in pairs: 280 us with two of them a chunk and single threads that issue, 202 with none and whole warps in step.)
struct Pixels {
    int x, y, z;
    __device__ __forceinline__ Pixels(const Grad &p, int c) {
        const int by = c / p.nx;
        z = by / p.ny;
        x = (c - by * p.nx) * p.tw; y = (by - z * p.ny) * p.th;
        z *= p.tb;
    }
    __device__ __forceinline__ void next(const Grad &p) {
        x += p.tw;
        if (x < p.wo) return;
        x = 0; y += p.th;
        if (y < p.ho) return;
        y = 0; z += p.tb;
    }
};

// Where the CTA is: an item (a tile and a part of the tokens), and a chunk of it.
struct Walk {
    int item, rt, first, n, c, c1;
    __device__ __forceinline__ void enter(const Grad &p, int i) {
        item = i;
        c = c1 = 0;
        if (i >= p.items) return;
        const int tile = i / p.splits, split = i - tile * p.splits;
        rt = tile / p.tiles_row;
        first = (tile - rt * p.tiles_row) * p.per;
        n = min(p.per, p.boxes - first);
        c = split * p.chunks_split;
        c1 = min(c + p.chunks_split, p.chunks);
    }
    __device__ __forceinline__ bool over(const Grad &p) const { return item >= p.items; }
};

// A chain's accumulator to the sums of a warp's 32 rows and 128 columns (two boxes).
__device__ __forceinline__ void add_chain(uint32_t from, int n, int half, float (&sum)[8][16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (half * 2 + i / 4 < n) {
            uint32_t r[16];
            tmem_ld_x16(from + 16 * i, r);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[i][j] += __uint_as_float(r[j]);
        }
    }
}
// (all lanes of a warp; row0: its first row)
__device__ __forceinline__ void store_sums(const Grad &p, const Walk &w, float *stage, int rt, int half, int row0, int lane, float (&sum)[8][16]) {
    if (row0 >= p.rows) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (half * 2 + i / 4 >= w.n) continue;
        const BoxAt at = box_at(p, rt, w.first + half * 2 + i / 4);
        const int c = at.c + 16 * (i & 3), here = min(16, p.channels - c);
        if (here > 0) store16(p, stage, row0, lane, at.tap * p.channels + c, here, sum[i]);
    }
}

// Zeros in `bytes` of each row (512 at most), by a warp, wherever they begin: 16 bytes a lane, and elements up to the first multiple of 16 and from the last one on.
// (An element a lane, in a loop: 330 cycles a row of 128 in bf16.)
__device__ __forceinline__ void zero_rows(uint8_t *to, int64_t pitch, int rows, int bytes, int size, int lane) {
#pragma unroll 4
    for (int r = 0; r < rows; ++r, to += pitch) {
        const int up = -(int)reinterpret_cast<uintptr_t>(to) & 15, down = bytes - ((int)reinterpret_cast<uintptr_t>(to + bytes) & 15);
        const int piece = up + lane * 16, one = lane < 8 ? lane * size : down + (lane - 16) * size;
        if (piece + 16 <= bytes) *reinterpret_cast<uint4 *>(to + piece) = make_uint4(0, 0, 0, 0);
        if (one < bytes && (lane < 8 ? one < up : lane >= 16 && one >= up)) {
            if (size == 4) *reinterpret_cast<uint32_t *>(to + one) = 0;
            else *reinterpret_cast<uint16_t *>(to + one) = 0;
        }
    }
}

// Zeros in the blocks that are not kept, by `zero_warps` warps of every CTA.
__device__ __forceinline__ void zero_dropped(const Grad &p, int warp, int lane) {
    const int size = p.f32 ? 4 : 2;
    for (int u = blockIdx.x + gridDim.x * warp; u < 4 * p.zeros; u += gridDim.x * p.zero_warps) {
        // (32 rows of a block)
        const int block = u >> 2, rt = block / p.zero_row, kb = block - rt * p.zero_row, row0 = rt * 128 + 32 * (u & 3), rows = min(32, p.rows - row0);
        bool kept = false;
        for (int i = lane; i < p.kkeep; i += 32) kept |= p.blk_col[(int64_t)rt * p.kkeep + i] == kb;
        if (__any_sync(0xFFFFFFFFu, kept)) continue;
        const int bytes = min(128, p.zero_k - kb * 128) * size, across = p.vec && bytes % 16 == 0 ? bytes / 16 : 0;
        uint8_t *to = reinterpret_cast<uint8_t *>(p.dw) + ((int64_t)row0 * p.ld + kb * 128) * size;
        const int64_t pitch = p.ld * size;
        if (across && (across & (across - 1)) == 0) {
            const int at_once = 32 / across, first = lane / across;
            to += first * pitch + (lane & (across - 1)) * 16;
#pragma unroll 8
            for (int r = first; r < rows; r += at_once, to += at_once * pitch) *reinterpret_cast<uint4 *>(to) = make_uint4(0, 0, 0, 0);
        } else {
            zero_rows(to, pitch, rows, bytes, size, lane);
        }
    }
}

template <bool kAMn, int kCount>
__global__ void __launch_bounds__(kGradThreads, 1)
grad8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ MapsOfX<kCount> maps, const __grid_constant__ Grad p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = smem_u32(smem_raw), ring = (base + 1023u) & ~1023u, ctrl = ring + kStages * kStage;
    uint8_t *ctrl_gen = smem_raw + (ctrl - base);
    const uint32_t bar_full = ctrl, bar_empty = ctrl + 64, bar_tfull = ctrl + 128, bar_tempty = ctrl + 144, bar_done = ctrl + 160;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 176);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(ctrl_gen + 180);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 2) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&maps.of[kCount == 1 ? 0 : (p.low + 1) * (p.narrow + 1) - 1]);
        for (int s = 0; s < kStages; ++s) { mbar_init(bar_full + 8 * s, 2); mbar_init(bar_empty + 8 * s, 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + 8 * a, 1); mbar_init(bar_tempty + 8 * a, kDrain); }
        mbar_init(bar_done, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    wait_for_prerequisites();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // The threads that issue copies and products are bound by their own instructions.  Their warps run the loops as a whole, so that addresses stay in uniform registers, where
    // the instructions take them from, and an elected thread issues; dY and x have a warp each.
    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------ dY, x
        const bool leader = elect_one(), rows = warp == 0;
        uint32_t dst = ring + (rows ? 0 : kABytes), full = bar_full, empty = bar_empty, ph = 0;
        int s = 0, fill = 0;
        bool ok = true;
        Walk w;
        for (w.enter(p, blockIdx.x); !w.over(p) && ok; w.enter(p, w.item + gridDim.x)) {
            From box[kBoxes];
#pragma unroll
            for (int i = 0; i < kBoxes; ++i) {
                box[i] = {nullptr, 0, 0, 0};
                if (!rows && i < w.n) box[i] = from_of(p, maps, box_at(p, w.rt, w.first + i));
            }
            const uint32_t bytes = rows ? kABytes : w.n * kBoxBytes;
            const int row = w.rt * 128;
            Pixels at(p, w.c);
            for (int c = w.c; c < w.c1; ++c, at.next(p)) {
                if (!wait_warp<false>(empty, ph ^ 1u, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                if (leader) {
                    mbar_expect_tx(full, bytes);
                    if (fill != p.skip_fill) {
                        if (!rows) {
#pragma unroll
                            for (int i = 0; i < kBoxes; ++i)
                                if (i < w.n) tma_load_4d(dst + i * kBoxBytes, box[i].map, box[i].c, at.x + box[i].dx, at.y + box[i].dy, at.z, full);
                        } else if constexpr (kAMn) {
                            tma_load_4d(dst, &map_a, row, at.x, at.y, at.z, full);
                            tma_load_4d(dst + 8192, &map_a, row + 64, at.x, at.y, at.z, full);
                        } else {
                            tma_load_2d(dst, &map_a, at.x, row, full);
                        }
                    }
                }
                ++fill;
                dst += kStage; full += 8; empty += 8;
                if (++s == kStages) { s = 0; dst -= kStages * kStage; full = bar_full; empty = bar_empty; ph ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ products
        const bool leader = elect_one();
        uint32_t ph = 0, acc = 0, acc_ph = 0, off = 0;
        int s = 0;
        bool ok = true;
        const uint64_t a0 = kAMn ? make_smem_desc(ring, 8192, 1024, kLayoutSw128) : make_smem_desc(ring, 16, 1024, kLayoutSw128);
        const uint64_t b0 = make_smem_desc(ring + kABytes, kBoxBytes, 1024, kLayoutSw128);
        constexpr uint32_t a_step = kAMn ? 128u : 2u;         // sixteen tokens on, in units of 16 bytes
        Walk w;
        for (w.enter(p, blockIdx.x); !w.over(p) && ok; w.enter(p, w.item + gridDim.x)) {
            const uint32_t idesc = make_idesc(64 * w.n, false) | (kAMn ? 1u << 15 : 0u);
            for (int c = w.c; c < w.c1 && ok; c += kChain) {
                ok = wait_warp<false>(bar_tempty + 8 * acc, acc_ph ^ 1u, leader, abort_flag, p.wait_limit);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + acc * 256;
                const int end = min(c + kChain, w.c1);
                for (int i = c; i < end; ++i) {
                    ok = wait_warp<false>(bar_full + 8 * s, ph, leader, abort_flag, p.wait_limit);
                    if (!ok) break;
                    tc_fence_after();
                    if (leader) {
#pragma unroll
                        for (int j = 0; j < kStep / 16; ++j) mma_dense(d, a0 + off + j * a_step, b0 + off + j * 128u, idesc, (uint32_t)((i - c) | j));
                        mma_commit(bar_empty + 8 * s);
                    }
                    off += kStage >> 4;
                    if (++s == kStages) { s = 0; off = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if (leader) mma_commit(bar_tfull + 8 * acc);
                if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
            }
        }
        if (leader) mma_commit(bar_done);                     // (also where a wait has run out: no accumulator is given back under a product)
        wait_warp<false>(bar_done, 0, leader, abort_flag, kWaitLimitCycles);
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ sums
        const int q = warp & 3, half = (warp - 4) >> 2;       // a warp may read the lanes of its quarter only
        if (p.zero_warps > 1) zero_dropped(p, warp - 3, lane);
        uint32_t acc = 0, acc_ph = 0;
        Walk w;
        for (w.enter(p, blockIdx.x); !w.over(p); w.enter(p, w.item + gridDim.x)) {
            float sum[8][16];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[i][j] = 0.f;
            int go = 1;
            for (int c = w.c; c < w.c1; c += kChain) {
                if (lane == 0) go = !*abort_flag && mbar_wait(bar_tfull + 8 * acc, acc_ph, abort_flag, p.wait_limit);
                go = __shfl_sync(0xFFFFFFFFu, go, 0);
                if (!go) break;
                tc_fence_after();
                add_chain(tmem + acc * 256 + half * 128 + ((uint32_t)(32 * q) << 16), w.n, half, sum);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_tempty + 8 * acc);
                if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
            }
            if (!go) break;
            if (p.splits > 1) {
                float *to = p.partial + ((int64_t)w.item * 256 + half * 128) * 128 + 32 * q + lane;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (half * 2 + i / 4 < w.n)
#pragma unroll
                        for (int j = 0; j < 16; ++j) to[(16 * i + j) * 128] = sum[i][j];
            } else {
                store_sums(p, w, reinterpret_cast<float *>(ctrl_gen + 256) + (warp - 4) * 32 * kStaged, w.rt, half, w.rt * 128 + 32 * q, lane, sum);
            }
        }
    } else {
        // -------------------------------------------------------------- zeros of blocks that are not kept
        zero_dropped(p, 0, lane);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0 && p.status) atomicCAS(p.status, 0, (int)CRISP_TIMEOUT);
        // copies that may still be in flight land before shared memory is released
        const unsigned long long t0 = clock64();
        while ((unsigned long long)(clock64() - t0) < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 2) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------------------------------------ pairs of SMs
//
// Two CTAs (a cluster) multiply 256 rows by 256 columns with cta_group::2: each fetches its 128 rows of dY and two of the four boxes of x, and the tensor cores of both read both
// halves: 32 KB a chunk into each instead of 48, and half as many instructions issued (4 to 6 % of the time, see where pairs are chosen).  Not under a mask of blocks, where every row
// tile has boxes of its own.
//
// The CTA of rank 0 issues for both.  The copies of both complete on its barriers, which count the bytes of both (what has landed in the peer's shared memory is acquired at the scope of the
// cluster); commits go to both (multicast); accumulators are handed back by the adding warps of both.  These two are seen at the scope of the cluster, relaxed: what tcgen05
// instructions read and write is ordered by their commits and fences, and nothing else is handed over.
constexpr uint32_t kPairStage = kABytes + kBoxes / 2 * kBoxBytes;
constexpr int kPairStages = 6;
constexpr size_t kPairSmem = kPairStages * kPairStage + 256 + kStaging + 1024;

__device__ __forceinline__ void mma_dense_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tma_load_4d_pair(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, uint32_t cluster_bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(cluster_bar) : "memory");
}

// (p.tiles_row and p.per as for one CTA; Walk's row tiles are pairs of them)
template <bool kAMn, int kCount>
__global__ void __launch_bounds__(kGradThreads, 1)
grad8_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ MapsOfX<kCount> maps, const __grid_constant__ Grad p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = smem_u32(smem_raw), ring = (base + 1023u) & ~1023u, ctrl = ring + kPairStages * kPairStage;
    uint8_t *ctrl_gen = smem_raw + (ctrl - base);
    // barriers: (rank 0) full[s] of both, empty[s]; accumulators full, and (rank 0) empty
    const uint32_t bar_full = ctrl, bar_empty = ctrl + 64, bar_tfull = ctrl + 128, bar_tempty = ctrl + 144, bar_done = ctrl + 160;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 176);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(ctrl_gen + 180);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t *>(tmem_slot))), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&maps.of[kCount == 1 ? 0 : (p.low + 1) * (p.narrow + 1) - 1]);
        for (int s = 0; s < kPairStages; ++s) { mbar_init(bar_full + 8 * s, 2); mbar_init(bar_empty + 8 * s, 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + 8 * a, 1); mbar_init(bar_tempty + 8 * a, 2 * kDrain); }
        mbar_init(bar_done, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    wait_for_prerequisites();
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                        // (the peer's barriers are there, and its tensor memory)
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int item0 = (int)(blockIdx.x >> 1), step = (int)(gridDim.x >> 1);

    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------ this CTA's rows, and its half of the boxes; (rank 0) both CTAs' byte counts
        const bool leader = elect_one(), rows = warp == 0;
        const uint32_t full0 = peer_address(bar_full, 0);
        uint32_t dst = ring + (rows ? 0 : kABytes), full = full0, empty = bar_empty, ph = 0;
        int s = 0, fill = 0;
        bool ok = true;
        Walk w;
        for (w.enter(p, item0); !w.over(p) && ok; w.enter(p, w.item + step)) {
            const int mine = (w.n + 1) / 2, row = (2 * w.rt + (int)rank) * 128;
            From box[kBoxes / 2];
#pragma unroll
            for (int i = 0; i < kBoxes / 2; ++i) {
                const int b = (int)rank * mine + i;
                box[i] = {&maps.of[0], p.cboxes * 64, 0, 0};  // (an odd number of boxes: the last one lies behind the last column and is zeros)
                if (!rows && i < mine && b < w.n) box[i] = from_of(p, maps, box_at(p, w.rt, w.first + b));
            }
            const uint32_t bytes = 2 * (rows ? kABytes : mine * kBoxBytes);
            Pixels at(p, w.c);
            for (int c = w.c; c < w.c1; ++c, at.next(p)) {
                if (!wait_warp<false>(empty, ph ^ 1u, leader, abort_flag, p.wait_limit)) { ok = false; break; }
                mbar_seen_cluster<false>(empty, ph ^ 1u);
                if (leader) {
                    // (the peer's bytes may come first: a phase ends with these arrivals at the earliest, and the peer fills a stage anew when the one before has been multiplied)
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, bytes);
                    if (fill != p.skip_fill) {
                        if (!rows) {
                            tma_load_4d_pair(dst, box[0].map, box[0].c, at.x + box[0].dx, at.y + box[0].dy, at.z, full);
                            if (mine > 1) tma_load_4d_pair(dst + kBoxBytes, box[1].map, box[1].c, at.x + box[1].dx, at.y + box[1].dy, at.z, full);
                        } else if constexpr (kAMn) {
                            tma_load_4d_pair(dst, &map_a, row, at.x, at.y, at.z, full);
                            tma_load_4d_pair(dst + 8192, &map_a, row + 64, at.x, at.y, at.z, full);
                        } else {
                            tma_load_2d_pair(dst, &map_a, at.x, row, full);
                        }
                    }
                }
                ++fill;
                dst += kPairStage; full += 8; empty += 8;
                if (++s == kPairStages) { s = 0; dst -= kPairStages * kPairStage; full = full0; empty = bar_empty; ph ^= 1u; }
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------ products, of both
        const bool leader = elect_one();
        uint32_t ph = 0, acc = 0, acc_ph = 0, off = 0;
        int s = 0;
        bool ok = true;
        const uint64_t a0 = kAMn ? make_smem_desc(ring, 8192, 1024, kLayoutSw128) : make_smem_desc(ring, 16, 1024, kLayoutSw128);
        const uint64_t b0 = make_smem_desc(ring + kABytes, kBoxBytes, 1024, kLayoutSw128);
        constexpr uint32_t a_step = kAMn ? 128u : 2u;
        Walk w;
        for (w.enter(p, item0); !w.over(p) && ok; w.enter(p, w.item + step)) {
            // (as make_idesc, M = 256)
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(128 * ((w.n + 1) / 2) >> 3) << 17) | (16u << 24) | (kAMn ? 1u << 15 : 0u);
            for (int c = w.c; c < w.c1 && ok; c += kChain) {
                ok = wait_warp<false>(bar_tempty + 8 * acc, acc_ph ^ 1u, leader, abort_flag, p.wait_limit);
                if (!ok) break;
                mbar_seen_cluster<false>(bar_tempty + 8 * acc, acc_ph ^ 1u);
                tc_fence_after();
                const uint32_t d = tmem + acc * 256;
                const int end = min(c + kChain, w.c1);
                for (int i = c; i < end; ++i) {
                    ok = wait_warp<false>(bar_full + 8 * s, ph, leader, abort_flag, p.wait_limit);
                    if (!ok) break;
                    mbar_seen_cluster<true>(bar_full + 8 * s, ph);
                    tc_fence_after();
                    if (leader) {
#pragma unroll
                        for (int j = 0; j < kStep / 16; ++j) mma_dense_pair(d, a0 + off + j * a_step, b0 + off + j * 128u, idesc, (uint32_t)((i - c) | j));
                        mma_commit_pair(bar_empty + 8 * s);
                    }
                    off += kPairStage >> 4;
                    if (++s == kPairStages) { s = 0; off = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if (leader) mma_commit_pair(bar_tfull + 8 * acc);
                if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
            }
        }
        if (leader) mma_commit_pair(bar_done);
        wait_warp<false>(bar_done, 0, leader, abort_flag, kWaitLimitCycles);
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ sums
        const int q = warp & 3, half = (warp - 4) >> 2;
        const uint32_t back = peer_address(bar_tempty, 0);
        uint32_t acc = 0, acc_ph = 0;
        Walk w;
        for (w.enter(p, item0); !w.over(p); w.enter(p, w.item + step)) {
            float sum[8][16];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[i][j] = 0.f;
            int go = 1;
            for (int c = w.c; c < w.c1; c += kChain) {
                if (lane == 0) go = !*abort_flag && mbar_wait(bar_tfull + 8 * acc, acc_ph, abort_flag, p.wait_limit);
                go = __shfl_sync(0xFFFFFFFFu, go, 0);
                if (!go) break;
                mbar_seen_cluster<false>(bar_tfull + 8 * acc, acc_ph);
                tc_fence_after();
                add_chain(tmem + acc * 256 + half * 128 + ((uint32_t)(32 * q) << 16), w.n, half, sum);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(back + 8 * acc);
                if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
            }
            if (!go) break;
            store_sums(p, w, reinterpret_cast<float *>(ctrl_gen + 256) + (warp - 4) * 32 * kStaged, w.rt, half, (2 * w.rt + (int)rank) * 128 + 32 * q, lane, sum);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0 && p.status) atomicCAS(p.status, 0, (int)CRISP_TIMEOUT);
        // copies that may still be in flight land before shared memory is released
        const unsigned long long t0 = clock64();
        while ((unsigned long long)(clock64() - t0) < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    cluster_arrive();                                        // neither CTA's memory is read, nor its barriers arrived at, by the other any more
    cluster_wait();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// dW of eight columns of a tile out of the parts of its tokens, added in their order: a warp reads a column of 128 rows (eight parts in flight), a thread writes four columns of a row.
__global__ void __launch_bounds__(256)
add_parts_kernel(const __grid_constant__ Grad p) {
    __shared__ float tile[8][132];
    wait_for_prerequisites();
    const int chunks = 8 * p.per, t = blockIdx.x / chunks, chunk = blockIdx.x - t * chunks;
    const int rt = t / p.tiles_row, first = (t - rt * p.tiles_row) * p.per;
    if (first + chunk / 8 >= p.boxes) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float4 *from = reinterpret_cast<const float4 *>(p.partial + ((int64_t)t * p.splits * 256 + chunk * 8 + warp) * 128) + lane;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < p.splits; ++s) {
        const float4 v = from[s * (256 * 32)];
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    *reinterpret_cast<float4 *>(&tile[warp][lane * 4]) = sum;
    __syncthreads();
    const BoxAt at = box_at(p, rt, first + chunk / 8);
    const int r = threadIdx.x >> 1, row = rt * 128 + r, c = at.c + 8 * (chunk & 7) + 4 * (threadIdx.x & 1), col = at.tap * p.channels + c, n = p.channels - c;
    if (row >= p.rows || n <= 0) return;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = tile[4 * (threadIdx.x & 1) + j][r];
    if (p.nm_bits) {
        const uint32_t bits = mask_bits(p, row, col);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!(bits >> j & 1u)) v[j] = 0.f;
    }
    const int64_t to = (int64_t)row * p.ld + col;
    if (p.f32) {
        float *w = reinterpret_cast<float *>(p.dw) + to;
        if (p.vec && n >= 4 && (col & 3) == 0) {
            float4 o = make_float4(v[0], v[1], v[2], v[3]);
            if (p.accumulate) { const float4 old = *reinterpret_cast<const float4 *>(w); o.x += old.x; o.y += old.y; o.z += old.z; o.w += old.w; }
            *reinterpret_cast<float4 *>(w) = o;
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) w[j] = p.accumulate ? w[j] + v[j] : v[j];
    } else {
        __nv_bfloat16 *w = reinterpret_cast<__nv_bfloat16 *>(p.dw) + to;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) w[j] = __float2bfloat16_rn(p.accumulate ? __bfloat162float(w[j]) + v[j] : v[j]);
    }
}

// Zeros in all of dW: of a layer without kept blocks.
__global__ void __launch_bounds__(256)
zero_kernel(int64_t rows, int k, void *dw, int64_t ld, int f32) {
    wait_for_prerequisites();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x; c < k; c += 256) {
            if (f32) reinterpret_cast<float *>(dw)[r * ld + c] = 0.f;
            else reinterpret_cast<uint16_t *>(dw)[r * ld + c] = 0;
        }
}

// dY's rows with a pitch that TMA takes: a warp copies 16-byte pieces of a row, whose elements it reads as wide as they lie (kWide: 4, 2 or 1 of them).
template <int kWide>
__global__ void __launch_bounds__(256)
repitch_dy_kernel(const uint16_t *dy, int64_t ld, int64_t rows, int64_t cols, uint16_t *to, int64_t pitch, int64_t pieces) {
    wait_for_prerequisites();
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / pieces, c = (u - row * pieces) * 8;
    if (row >= rows) return;
    const uint16_t *from = dy + row * ld + c;
    uint32_t w[4] = {0, 0, 0, 0};
    if (c + 8 <= cols) {
        if constexpr (kWide == 4) {
            const uint2 a = reinterpret_cast<const uint2 *>(from)[0], b = reinterpret_cast<const uint2 *>(from)[1];
            w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = kWide == 2 ? reinterpret_cast<const uint32_t *>(from)[j] : from[2 * j] | (uint32_t)from[2 * j + 1] << 16;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < cols) w[j / 2] |= (uint32_t)from[j] << (16 * (j & 1));
    }
    *reinterpret_cast<uint4 *>(to + row * pitch + c) = make_uint4(w[0], w[1], w[2], w[3]);
}

// A convolution's dY [rows, columns] to [columns, rows] with a pitch that TMA takes: tiles of 64 x 64.
__global__ void __launch_bounds__(256)
transpose_dy_kernel(const uint16_t *dy, int64_t ld, int rows, int64_t ncols, uint16_t *to, int64_t pitch, int row_tiles) {
    __shared__ uint16_t tile[64][66];
    wait_for_prerequisites();
    const int64_t u = blockIdx.x / row_tiles, t0 = u * 64;
    const int r0 = (int)(blockIdx.x - u * row_tiles) * 64, x = threadIdx.x & 63, y = threadIdx.x >> 6;
    for (int i = y; i < 64; i += 4) {
        if (r0 + i < rows && t0 + x < ncols) tile[x][i] = dy[(int64_t)(r0 + i) * ld + t0 + x];
    }
    __syncthreads();
    for (int i = y; i < 64; i += 4)
        if (t0 + i < ncols && r0 + x < rows) to[(t0 + i) * pitch + r0 + x] = tile[i][x];
}

// ------------------------------------------------------------------------------------------------------------------- host

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct GradPlan {
    Grad p;
    bool pair, k_major, copy, blocks;                               // dY as [rows, columns]; through a copy; tiles follow the mask's list
    int64_t pixels, cpitch, pitch;                            // columns of x, pitches of x in bf16 and of a copied dY
    int ho, wo, batch;
    size_t x_off, dy_off, partial_off, total;
    int nrt;
};

crisp_status_t plan_grad(const crisp_weight_grad8_t *g, GradPlan *G) {
    if (!g || (g->dy_layout != 0 && g->dy_layout != 1) || (g->dw_dtype != 0 && g->dw_dtype != 1) || (g->accumulate != 0 && g->accumulate != 1) || g->skip_fill < 0)
        return CRISP_INVALID_ARG;
    if (g->rows <= 0 || g->k <= 0 || g->ncols <= 0) return CRISP_BAD_SHAPE;
    if (g->ncols > 0x7FFFFFFFll - 65536 || g->rows > 65535 * 32 || g->k > kMaxBlocksPerRowTile * 128) return CRISP_UNSUPPORTED;
    *G = GradPlan{};
    Grad &p = G->p;
    p.rows = g->rows;
    p.linear = g->conv == nullptr;
    if (p.linear) {
        p.channels = g->k; p.kernel_w = 1;
        G->pixels = g->ncols; G->batch = 1; G->ho = 1; G->wo = (int)g->ncols;
        p.tw = kStep; p.th = p.tb = 1;
    } else {
        const crisp_conv_desc_t &c = *g->conv;
        if (c.batch <= 0 || c.height <= 0 || c.width <= 0 || c.channels <= 0 || c.kernel_h <= 0 || c.kernel_w <= 0 || c.pad < 0) return CRISP_BAD_SHAPE;
        const int64_t ho = (int64_t)c.height + 2 * (int64_t)c.pad - c.kernel_h + 1, wo = (int64_t)c.width + 2 * (int64_t)c.pad - c.kernel_w + 1;
        if (ho <= 0 || wo <= 0 || (int64_t)c.kernel_h * c.kernel_w > g->k || (int64_t)c.kernel_h * c.kernel_w * c.channels != g->k) return CRISP_BAD_SHAPE;
        if (ho > 0x7FFFFFFF || wo > 0x7FFFFFFF || ho > g->ncols || wo > g->ncols || c.batch > g->ncols || (double)c.batch * (double)ho * (double)wo != (double)g->ncols)
            return CRISP_BAD_SHAPE;
        if ((double)c.batch * c.height * c.width > 2147418112.0) return CRISP_UNSUPPORTED;
        p.channels = c.channels; p.kernel_w = c.kernel_w; p.pad = c.pad;
        G->pixels = (int64_t)c.batch * c.height * c.width; G->batch = c.batch; G->ho = (int)ho; G->wo = (int)wo;
        // the box of 64 output pixels that covers the fewest outside the images, the widest of them.  (Kernels of many taps beside little padding have a box that ends with the lines or with
        // the columns: it needs fewer maps, or none but one.)
        const int left = std::max(0, c.kernel_w - 1 - c.pad), above = std::max(0, c.kernel_h - 1 - c.pad);
        int64_t best = -1;
        for (int tw = kStep; tw >= 1; tw >>= 1)
            for (int th = kStep / tw; th >= 1; th >>= 1) {
                const int tb = kStep / tw / th, narrow = wo % tw ? left : 0, low = ho % th ? above : 0;
                const int64_t n = up(wo, tw) * up(ho, th) * up(c.batch, tb);
                if ((best < 0 || n < best) && (int64_t)(narrow + 1) * (low + 1) <= kMaps) { best = n; p.tw = tw; p.th = th; p.tb = tb; p.narrow = narrow; p.low = low; }
            }
        p.width0 = (int)wo - c.pad; p.height0 = (int)ho - c.pad;
    }
    p.wo = G->wo; p.ho = G->ho;
    p.nx = (int)up(G->wo, p.tw); p.ny = (int)up(G->ho, p.th);
    const int64_t chunks = (int64_t)p.nx * p.ny * up(G->batch, p.tb);
    if (chunks > 0x7FFFFFFFll - 4096) return CRISP_UNSUPPORTED;
    p.chunks = (int)chunks;
    p.cboxes = (int)up(p.channels, 64);
    G->nrt = (int)up(p.rows, 128);
    const int taps = g->k / p.channels;
    p.boxes = taps * p.cboxes;
    if (g->mask) {
        const Geometry &m = g->mask->g;
        if (m.rows != g->rows || m.k != g->k) return CRISP_BAD_SHAPE;
        p.nm_bits = g->mask->d_nm_bits; p.wpr = m.wpr;
        G->blocks = m.bm == 128 && m.bk == 128 && (taps == 1 || p.channels % 128 == 0);
        if (G->blocks && m.kkeep < m.nblk) {
            p.blk_col = g->mask->d_blk_col; p.kkeep = m.kkeep; p.boxes = 2 * m.kkeep;
            if (taps == 1) p.cboxes = 2 * m.nblk;             // (with 192 channels the fourth box is none of a second tap: it is copied as zeros and not stored)
        }
        else G->blocks = false;
    }
    size_t at = 0;
    if (p.boxes > 0) {
        p.tiles_row = (int)up(p.boxes, kBoxes);
        p.per = (int)up(p.boxes, p.tiles_row);
        if (p.blk_col) p.per = kBoxes;                        // (two blocks a tile)
        p.tiles_row = (int)up(p.boxes, p.per);
        const int64_t tiles = (int64_t)G->nrt * p.tiles_row;
        if (tiles > (1 << 24)) return CRISP_UNSUPPORTED;
        // Parts of the tokens where there are fewer tiles than SMs, of 256 tokens at least.  (Half as many parts: 1024 x 1024, 4096 tokens 22.6 us instead of 18.0, 128 x 1152, 25088
        // tokens 32.4 and 30.7; parts of 512 tokens: 256 x 1024, 512 tokens 12.4 and 10.3; of 128 the same.)
        int64_t splits = std::max<int64_t>(1, std::min<int64_t>(148 / tiles, p.chunks / 4));
        p.chunks_split = (int)up(p.chunks, splits);
        p.splits = (int)up(p.chunks, p.chunks_split);
        p.items = (int)(tiles * p.splits);
        // Pairs where a tile is not cut into parts and half of the SMs have one.  Measured, us, one SM a tile and pairs: 64 pairs, 2048 x 2048 and 8192 tokens 61.1 and 57.4; 2304 x 2304
        // and 2048 tokens 44.3 and 41.2; 4096 x 4096 73.8 and 69.1, and 8192 tokens 245 and 235 (with the loops of that time).
        G->pair = !p.blk_col && p.splits == 1 && G->nrt >= 2 && tiles >= 74;
        if (G->pair) p.items = (int)(up(G->nrt, 2) * p.tiles_row);
        G->cpitch = up(p.channels, 64) * 64;
        G->x_off = 0;
        at = align_up((size_t)G->pixels * G->cpitch * 2);
        // a matrix is taken as it lies, [rows, columns] too; a convolution's pixels have to be boxes
        G->k_major = g->dy_layout == 0 && p.linear;
        G->copy = !(aligned_to(g->d_dy, 16) && g->ld_dy % 8 == 0) || (g->dy_layout == 0 && !p.linear);
        if (G->copy) {
            G->pitch = up(G->k_major ? g->ncols : p.rows, 8) * 8;
            G->dy_off = at;
            at += align_up((size_t)(G->k_major ? p.rows : g->ncols) * G->pitch * 2);
        }
        if (p.splits > 1) {
            G->partial_off = at;
            at += (size_t)p.items * 256 * 128 * sizeof(float);
        }
    }
    G->total = at;
    return CRISP_OK;
}

template <auto kernel, int kCount>
cudaError_t launch_grad(const CUtensorMap &a, const MapsOfX<kCount> &b, const Grad &p, size_t smem, unsigned cluster, int sms, int device, cudaStream_t st) {
    static std::atomic<uint64_t> ready{0};                                    // (one a kernel: by device)
    if (device >= 64 || !(ready.load(std::memory_order_relaxed) >> device & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (device < 64) ready.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    return launch_clusters(kernel, cluster * (unsigned)std::min(std::max(p.items, 4 * p.zeros), sms / (int)cluster), kGradThreads, smem, st, cluster, a, b, p);
}

template <int kCount>
cudaError_t launch_product(const GradPlan &G, const CUtensorMap &a, const MapsOfX<kCount> &b, int sms, int device, cudaStream_t st) {
    if constexpr (kCount == 1)
        if (G.k_major)
            return G.pair ? launch_grad<grad8_pair_kernel<false, 1>>(a, b, G.p, kPairSmem, 2, sms, device, st) : launch_grad<grad8_kernel<false, 1>>(a, b, G.p, kGradSmem, 1, sms, device, st);
    return G.pair ? launch_grad<grad8_pair_kernel<true, kCount>>(a, b, G.p, kPairSmem, 2, sms, device, st)
                  : launch_grad<grad8_kernel<true, kCount>>(a, b, G.p, kGradSmem, 1, sms, device, st);
}

cudaError_t run_grad(const crisp_weight_grad8_t &g, GradPlan &G, uint8_t *ws, cudaStream_t st) {
    Grad &p = G.p;
    cudaError_t e;
    p.dw = g.d_dw; p.ld = g.ld_dw; p.f32 = g.dw_dtype; p.accumulate = g.accumulate;
    p.vec = aligned_to(g.d_dw, 16) && g.ld_dw * (g.dw_dtype ? 4 : 2) % 16 == 0;
    p.status = g.d_status;
    p.wait_limit = g.wait_limit_cycles ? g.wait_limit_cycles : kWaitLimitCycles;
    p.skip_fill = g.skip_fill - 1;
    if (p.boxes == 0)
        return g.accumulate ? cudaSuccess : launch_chained(zero_kernel, (unsigned)std::min(g.rows, 4096), 256, 0, st, (int64_t)g.rows, (int)g.k, g.d_dw, g.ld_dw, (int)g.dw_dtype);
    // Few tokens: the adding warps write zeros, too, before there is anything to add.  (2303 x 3301 in fp32, a quarter of the blocks kept, 9 tokens: 88 us with one warp of a CTA and the
    // mask looked up for each element that is stored, 33 with nine and a look-up for a row's 16.)  Where there is much to multiply one warp is enough, and the others stay out of its way.
    if (G.blocks && !g.accumulate) { p.zero_warps = p.chunks_split <= 2 * kChain ? 1 + kDrain : 1; p.zero_row = g.mask->g.nblk; p.zeros = g.mask->g.nrt * g.mask->g.nblk; p.zero_k = g.k; }
    int device = 0;
    e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    e = ensure_context(device);
    if (e != cudaSuccess) return e;
    uint16_t *x = reinterpret_cast<uint16_t *>(ws + G.x_off);
    p.partial = reinterpret_cast<float *>(ws + G.partial_off);
    e = launch_dequantize8(reinterpret_cast<const uint8_t *>(g.d_act), 1, p.channels, G.pixels, x, G.cpitch, st);
    if (e != cudaSuccess) return e;
    const uint16_t *dy = g.d_dy;
    int64_t ld = g.ld_dy;
    if (G.copy) {
        uint16_t *to = reinterpret_cast<uint16_t *>(ws + G.dy_off);
        if (g.dy_layout == 0 && !p.linear) {
            const int64_t row_tiles = up(p.rows, 64), ctas = row_tiles * up(g.ncols, 64);
            if (ctas > 0x7FFFFFFFll) return cudaErrorInvalidValue;
            e = launch_chained(transpose_dy_kernel, (unsigned)ctas, 256, 0, st, g.d_dy, g.ld_dy, p.rows, g.ncols, to, G.pitch, (int)row_tiles);
        } else {
            const int64_t rows = G.k_major ? p.rows : g.ncols, cols = G.k_major ? g.ncols : p.rows, pieces = G.pitch / 8, ctas = up(rows * pieces, 256);
            if (ctas > 0x7FFFFFFFll) return cudaErrorInvalidValue;
            const auto kernel = aligned_to(g.d_dy, 8) && g.ld_dy % 4 == 0 ? repitch_dy_kernel<4> : aligned_to(g.d_dy, 4) && g.ld_dy % 2 == 0 ? repitch_dy_kernel<2> : repitch_dy_kernel<1>;
            e = launch_chained(kernel, (unsigned)ctas, 256, 0, st, g.d_dy, g.ld_dy, rows, cols, to, G.pitch, pieces);
        }
        if (e != cudaSuccess) return e;
        dy = to; ld = G.pitch;
    }
    CUtensorMap a;
    MapsOfX<kMaps> b;
    const uint64_t W = g.conv ? g.conv->width : g.ncols, H = g.conv ? g.conv->height : 1, N = G.batch;
    const uint32_t box[4] = {64u, (uint32_t)p.tw, (uint32_t)p.th, (uint32_t)p.tb};
    const uint64_t xs[3] = {(uint64_t)G.cpitch * 2, W * G.cpitch * 2, W * H * G.cpitch * 2};
    const int maps = (p.low + 1) * (p.narrow + 1);
    for (int i = 0; i < maps; ++i) {
        const int row = i / (p.narrow + 1), column = i - row * (p.narrow + 1);
        const uint64_t xd[4] = {(uint64_t)p.channels, column < p.narrow ? (uint64_t)std::max(1, p.width0 + column) : W, row < p.low ? (uint64_t)std::max(1, p.height0 + row) : H, N};
        if (!make_map_4d(&b.of[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, x, xd, xs, box)) return cudaErrorInvalidValue;
    }
    if (G.k_major) {
        if (!make_map_2d(&a, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy, (uint64_t)g.ncols, (uint64_t)p.rows, (uint64_t)ld, 64, 128)) return cudaErrorInvalidValue;
    } else {
        const uint64_t wo = G.wo, ho = G.ho, yd[4] = {(uint64_t)p.rows, wo, ho, N}, ys[3] = {(uint64_t)ld * 2, wo * ld * 2, wo * ho * ld * 2};
        if (!make_map_4d(&a, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy, yd, ys, box)) return cudaErrorInvalidValue;
    }
    const int sms = sm_count_of(device);
    e = maps > 1 ? launch_product(G, a, b, sms, device, st) : launch_product(G, a, MapsOfX<1>{{b.of[0]}}, sms, device, st);
    if (e == cudaSuccess && p.splits > 1)
        e = launch_chained(add_parts_kernel, (unsigned)(G.nrt * p.tiles_row * 8 * p.per), 256, 0, st, p);
    return e;
}

}  // namespace

}  // namespace crisp

extern "C" {

using namespace crisp;

crisp_status_t crisp_weight_grad8_sizes(const crisp_weight_grad8_t *grad, size_t *workspace_bytes) {
    GradPlan G;
    const crisp_status_t bad = plan_grad(grad, &G);
    if (bad != CRISP_OK) return bad;
    if (!workspace_bytes) return CRISP_INVALID_ARG;
    *workspace_bytes = G.total;
    return CRISP_OK;
}

crisp_status_t crisp_weight_grad8(const crisp_weight_grad8_t *grad, void *d_workspace, void *stream) {
    GradPlan G;
    const crisp_status_t bad = plan_grad(grad, &G);
    if (bad != CRISP_OK) return bad;
    const crisp_weight_grad8_t &g = *grad;
    if (!g.d_dy || !g.d_act || !g.d_dw || (!d_workspace && G.total) || !aligned_to(g.d_dy, 2) || !aligned_to(g.d_act, kAlign) || !aligned_to(g.d_dw, g.dw_dtype ? 4 : 2) ||
        !aligned_to(g.d_status, 4) || !aligned_to(d_workspace, kAlign))
        return CRISP_INVALID_ARG;
    if (g.ld_dy < (g.dy_layout ? (int64_t)g.rows : g.ncols) || g.ld_dw < g.k) return CRISP_BAD_SHAPE;
    size_t bytes = 0;
    if (crisp_quantize8_sizes(G.p.channels, G.pixels, &bytes) != CRISP_OK) return CRISP_UNSUPPORTED;
    const cudaError_t e = run_grad(g, G, reinterpret_cast<uint8_t *>(d_workspace), (cudaStream_t)stream);
    return e == cudaSuccess ? CRISP_OK : e == cudaErrorInvalidValue ? CRISP_UNSUPPORTED : CRISP_CUDA_ERROR;
}

}  // extern "C"
