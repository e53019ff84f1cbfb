// Weights and activations to 8-bit floats with a power-of-two scale for each block of 128, and weights back.
//
//   E = the smallest exponent with max |x| <= 448 * 2^E,   q = x * 2^-E to the nearest e4m3 (even at ties)
//
// The scale is a power of two, so x * 2^-E is exact and the code is rounded once.  All of it moves bytes and little else: each value is read once, held in registers
// while its block's largest one is found, and written once, in the layout of block8.h.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "block8.h"
#include "block8.cuh"
#include "mask_common.cuh"

namespace crisp {

using namespace block8;

namespace {

// -------------------------------------------------------------------------------------------------------------- weights

// One CTA a kept block: thread t takes eight columns (t % 16) of rows t / 16, + 32, ...  `vec`: 8, 2 or 1 columns a load, by what address and pitch allow.
// Bound by the chain of a CTA (list, mask and weights, largest value, codes): 4096 x 4096 2:4 keep 0.5 8.4 us, all of it 13.1, with four CTAs an SM; two 11.3 and
// 18.3, three 10.8 and 15.7.  A thread's loads all ahead of their use spill at four CTAs (16.0), and take 9.1 and 13.2 at three; two rows a thread 10.0 and 15.9.
__global__ void __launch_bounds__(512, 4)
encode8_kernel(Geometry g, const uint16_t *w, int64_t ld, const int32_t *mask_blk_col, const uint32_t *nm_bits, int32_t *blk_col, uint8_t *exps, uint8_t *image,
               uint32_t *header, uint8_t *used, int wide) {
    __shared__ uint32_t largest[16];
    chain_kernels();
    const int slot = blockIdx.x, rt = slot / g.kkeep, kb = g.kkeep == g.nblk ? slot - rt * g.kkeep : mask_blk_col[slot];
    const int chunk = threadIdx.x & 15, row0 = threadIdx.x >> 4;
    const int64_t col = (int64_t)kb * 128 + chunk * 8;
    const int vec = col + 8 <= g.k ? wide : 1;
    uint32_t x[4][4], top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = (int64_t)rt * 128 + row0 + 32 * i;
        uint32_t keep = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = 0;
        if (row < g.rows) {
            keep = g.n == g.m ? 0xFFu : reinterpret_cast<const uint8_t *>(nm_bits + row * g.wpr)[kb * 16 + chunk];
            const uint16_t *p = w + row * ld + col;
            if (vec == 8) {
                const uint4 v = *reinterpret_cast<const uint4 *>(p);
                x[i][0] = v.x; x[i][1] = v.y; x[i][2] = v.z; x[i][3] = v.w;
            } else if (vec == 2) {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] = reinterpret_cast<const uint32_t *>(p)[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < g.k) x[i][j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t two = keep >> (2 * j) & 3u;
            x[i][j] &= (two & 1u ? 0xFFFFu : 0u) | (two & 2u ? 0xFFFF0000u : 0u);
            top = larger(top, x[i][j]);
        }
    }
    if (__syncthreads_or(larger_of(top) >= 0x7F80u)) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                top = larger(top, finite(x[i][j]));
                x[i][j] = nan_for_infinity(x[i][j]);
            }
    }
    top = __reduce_max_sync(0xFFFFFFFFu, larger_of(top));
    if ((threadIdx.x & 31) == 0) largest[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, largest[i]);
    const uint32_t e = exponent_of(top);
    const float down = power_of(254u - e);
    uint8_t *entry = image + (int64_t)slot * kEntry8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + 32 * i;
        uint8_t *at = entry + (row >> 3) * 1024 + (row & 7) * 128 + (((chunk >> 1) ^ (row & 7)) << 4) + (chunk & 1) * 8;
        *reinterpret_cast<uint2 *>(at) = make_uint2(codes2(x[i][0], down) | codes2(x[i][1], down) << 16, codes2(x[i][2], down) | codes2(x[i][3], down) << 16);
    }
    if (threadIdx.x < 128) reinterpret_cast<uint32_t *>(entry + kTile8)[threadIdx.x] = e * 0x01010101u;
    if (threadIdx.x == 0) { blk_col[slot] = kb; exps[slot] = (uint8_t)e; }
    if (slot == 0 && threadIdx.x < 64) header[threadIdx.x] = 0;
    if (g.kkeep == g.nblk) return;
    // which k-blocks any row tile keeps: a CTA looks one of them up in all lists, with its own values stored (a CTA of its own for it held registers that
    // the rest spilled: 4096 x 4096 with half of its blocks took 13.0 us, not 8.5)
    const int n = g.nrt * g.kkeep;
    for (int b = slot; b < g.nblk; b += n) {
        int hit = 0;
        for (int i = threadIdx.x; i < n; i += 512) hit |= mask_blk_col[i] == b;
        hit = __syncthreads_or(hit);
        if (threadIdx.x == 0) used[b] = (uint8_t)(hit != 0);
    }
}

// One CTA a block of the dense matrix, kept or not.
constexpr int kDecode = 256;                                   // (4096 x 4096, half kept: 8.3 us; with 128 threads 9.3, 512 8.6, and 10.4 with loads behind stores)
__global__ void __launch_bounds__(kDecode, 2048 / kDecode)
decode8_kernel(Geometry g, const int32_t *blk_col, const uint8_t *exps, const uint8_t *image, uint16_t *w, int64_t ld, int wide) {
    chain_kernels();
    const int rt = blockIdx.x / g.nblk, kb = blockIdx.x - rt * g.nblk;
    int slot = rt * g.kkeep + kb;
    uint32_t e = 0;
    if (g.kkeep == g.nblk) {
        e = exps[slot];
    } else {
        // where the block is in its row tile's list, if it is, and its exponent (every warp looks for itself)
        slot = -1;
        for (int i0 = 0; i0 < g.kkeep; i0 += 32) {
            const int i = i0 + (int)(threadIdx.x & 31), at = rt * g.kkeep + i;
            const int col = i < g.kkeep ? blk_col[at] : -1;
            const uint32_t here = i < g.kkeep ? exps[at] : 0u, hit = __ballot_sync(0xFFFFFFFFu, col == kb);
            if (hit) {
                slot = rt * g.kkeep + i0 + __ffs(hit) - 1;
                e = __shfl_sync(0xFFFFFFFFu, here, __ffs(hit) - 1);
                break;
            }
        }
    }
    const int chunk = threadIdx.x & 15, row0 = threadIdx.x >> 4;
    const int64_t col = (int64_t)kb * 128 + chunk * 8;
    const float up = power_of(e);
    const uint8_t *entry = image + (int64_t)slot * kEntry8;
    // (all codes ahead of the first store, which the compiler would not move a load over)
    constexpr int kRows = 2048 / kDecode;
    uint2 codes[kRows] = {};
    if (slot >= 0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = row0 + kDecode / 16 * i;
            codes[i] = *reinterpret_cast<const uint2 *>(entry + (r >> 3) * 1024 + (r & 7) * 128 + (((chunk >> 1) ^ (r & 7)) << 4) + (chunk & 1) * 8);
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t row = (int64_t)rt * 128 + row0 + kDecode / 16 * i;
        if (row >= g.rows || col >= g.k) break;
        uint32_t out[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((j < 2 ? codes[i].x : codes[i].y) >> (16 * (j & 1))), __NV_E4M3);
            const float2 v = __half22float2(__half2(h));
            const __nv_bfloat162 b = __floats2bfloat162_rn(v.x * up, v.y * up);
            out[j] = *reinterpret_cast<const uint32_t *>(&b);
        }
        uint16_t *p = w + row * ld + col;
        const int vec = col + 8 <= g.k ? wide : 1;
        if (vec == 8) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(out[0], out[1], out[2], out[3]);
        } else if (vec == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) reinterpret_cast<uint32_t *>(p)[j] = out[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < g.k) p[j] = (uint16_t)(out[j / 2] >> (16 * (j & 1)));
        }
    }
}

// ---------------------------------------------------------------------------------------------------------- activations

__device__ __forceinline__ void put_scale(uint8_t *scales, int64_t chunks, int64_t kb, int64_t col, uint32_t e) {
    *reinterpret_cast<uint32_t *>(scales + (kb * chunks + (col >> 7)) * kScales8 + (col & 31) * 16 + (col >> 5 & 3) * 4) = e * 0x01010101u;
}

// 2 kWords elements that start at any even address, out of the two aligned pieces of as many that hold them.
template <int kWords>
__device__ __forceinline__ void unaligned(const uint16_t *p, uint32_t (&v)[kWords]) {
    const uint32_t by = (uint32_t)(reinterpret_cast<uintptr_t>(p) >> 1) & (2 * kWords - 1);
    uint32_t w[2 * kWords];
    if constexpr (kWords == 4) {
        const uint4 *from = reinterpret_cast<const uint4 *>(p - by);
        const uint4 a = from[0], b = from[1];
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = by & 4 ? w[i + 2] : w[i];
    } else {
        const uint2 *from = reinterpret_cast<const uint2 *>(p - by);
        const uint2 a = from[0], b = from[1];
        w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
    }
#pragma unroll
    for (int i = 0; i <= kWords; ++i)
        if (i + 1 < 2 * kWords) w[i] = by & 2 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < kWords; ++i) v[i] = __funnelshift_r(w[i], w[i + 1], 16 * (by & 1));
}

// X [ncols, k]: a CTA takes eight columns (tokens) and 2 U k-blocks; 16 threads a block of one column, eight values each, U blocks a thread.  Bound by instructions
// (4096 x 8192: 20 a value and 22 us as one loop over the blocks with every question asked in it; now 17.1, 5.9 TB/s): a CTA whose blocks are all there asks nothing,
// and two blocks' largest values travel through the shuffles in one word.  At other addresses each thread reads the two 16-byte pieces around its values (4097 x 8192:
// 29.4 us, 35.6 by single elements).
enum class Read { kAligned, kUnaligned, kParts };             // whole blocks at multiples of 16 bytes, at others, all else
template <int U, Read kRead>
__device__ __forceinline__ void quantize_tokens(const uint16_t *x, int64_t ldx, int64_t k, int64_t ncols, int64_t nblk, int64_t groups, int64_t chunks, uint8_t *codes,
                                                uint8_t *scales, const uint8_t *used, int vec_ok, int64_t group, int64_t kb0) {
    constexpr bool kFull = kRead != Read::kParts;
    const int lane = threadIdx.x & 15, r = threadIdx.x >> 4 & 7, side = threadIdx.x >> 7;
    const int64_t col = group * 8 + r, kb1 = kb0 + side * U;         // (a warp's two columns share their k-blocks)
    uint32_t v[U][4], top[U], word[U / 2], any = 0;
    const uint16_t *from = x + col * ldx + kb1 * 128 + lane * 8;
    bool wanted[U];
#pragma unroll
    for (int i = 0; i < U; ++i) wanted[i] = !used || (kb1 + i < nblk && used[kb1 + i]);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t at = (kb1 + i) * 128 + lane * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = 0;
        if (!wanted[i]) continue;
        if (kRead == Read::kUnaligned) {
            unaligned<4>(from + i * 128, v[i]);
        } else if (kFull || (vec_ok && col < ncols && at + 8 <= k)) {
            const uint4 u = *reinterpret_cast<const uint4 *>(from + i * 128);
            v[i][0] = u.x; v[i][1] = u.y; v[i][2] = u.z; v[i][3] = u.w;
        } else if (col < ncols) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at + j < k) v[i][j / 2] |= (uint32_t)from[i * 128 + j] << (16 * (j & 1));
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        top[i] = larger(larger(larger(larger(0, v[i][0]), v[i][1]), v[i][2]), v[i][3]);
        any = __vmaxu2(any, top[i]);
    }
    if (__any_sync(0xFFFFFFFFu, larger_of(any) >= 0x7F80u)) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            top[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                top[i] = larger(top[i], finite(v[i][j]));
                v[i][j] = nan_for_infinity(v[i][j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < U / 2; ++i) word[i] = larger_of(top[2 * i]) | larger_of(top[2 * i + 1]) << 16;
#pragma unroll
    for (int d = 8; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < U / 2; ++i) word[i] = __vmaxu2(word[i], __shfl_xor_sync(0xFFFFFFFFu, word[i], d));
    uint8_t *to = codes + (kb1 * groups + group) * 1024 + r * 128 + (((lane >> 1) ^ r) << 4) + (lane & 1) * 8;
    uint8_t *scale = scales + (kb1 * chunks + (col >> 7)) * kScales8 + (col & 31) * 16 + (col >> 5 & 3) * 4;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (!kFull && kb1 + i >= nblk) break;
        const uint32_t e = exponent_of(word[i / 2] >> (16 * (i & 1)) & 0xFFFFu);
        const float down = power_of(254u - e);
        if (wanted[i]) {
            *reinterpret_cast<uint2 *>(to) = make_uint2(codes2(v[i][0], down) | codes2(v[i][1], down) << 16, codes2(v[i][2], down) | codes2(v[i][3], down) << 16);
            if (lane == 0 && (kFull || col < ncols)) *reinterpret_cast<uint32_t *>(scale) = e * 0x01010101u;
        }
        to += groups * 1024;
        scale += chunks * kScales8;
    }
}

template <int U>
__global__ void __launch_bounds__(256)
quantize_tokens_kernel(const uint16_t *x, int64_t ldx, int64_t k, int64_t ncols, int64_t nblk, int64_t groups, int64_t chunks, uint8_t *codes, uint8_t *scales,
                       const uint8_t *used, int vec_ok) {
    wait_for_prerequisites();
    launch_dependents();                     // (a product behind this one fetches weights meanwhile: all before this kernel has finished)
    const uint32_t spans = (uint32_t)((nblk + 2 * U - 1) / (2 * U)), g = blockIdx.x / spans;
    const int64_t group = g, kb0 = (int64_t)(blockIdx.x - g * spans) * (2 * U);
    const int64_t end = (kb0 + 2 * U) * 128, first = group * 8;
    if (end > k || first + 8 > ncols)
        quantize_tokens<U, Read::kParts>(x, ldx, k, ncols, nblk, groups, chunks, codes, scales, used, vec_ok, group, kb0);
    else if (vec_ok)
        quantize_tokens<U, Read::kAligned>(x, ldx, k, ncols, nblk, groups, chunks, codes, scales, used, vec_ok, group, kb0);
    else if (first * ldx + kb0 * 128 >= 7 && (first + 7) * ldx + end + 8 <= (ncols - 1) * ldx + k)     // (what lies around the blocks is X, too)
        quantize_tokens<U, Read::kUnaligned>(x, ldx, k, ncols, nblk, groups, chunks, codes, scales, used, vec_ok, group, kb0);
    else
        quantize_tokens<U, Read::kParts>(x, ldx, k, ncols, nblk, groups, chunks, codes, scales, used, vec_ok, group, kb0);
}

// X [k, ncols]: a CTA takes 128 columns of one k-block.  A warp reads 16 rows of it, a lane four columns; the 16 values of a column in a warp are one
// 16-byte chunk of its codes.  Neighbouring CTAs read neighbouring columns.  The tile in shared memory is the atoms' with their chunks in another order in each atom,
// since a warp writes eight atoms' chunks of one place together.  4096 x 8192: 19.7 us (5.1 TB/s); two pairs of columns a lane, 64 apart, 23.4; eight rows a warp, 23.6
// (more partial maxima); X through shared memory by asynchronous copies, 20.5; neighbouring CTAs on neighbouring k-blocks, 64 columns each, 52.  Rows that do not start at multiples of 8 bytes take two loads (4096 x 8191:
// 26.7 us with four CTAs an SM; single elements 41).
template <bool kQuads>
__global__ void __launch_bounds__(256, kQuads ? 3 : 4)
quantize_columns_kernel(const uint16_t *x, int64_t ldx, int64_t k, int64_t ncols, int64_t nblk, int64_t groups, int64_t chunks, uint8_t *codes, uint8_t *scales,
                        const uint8_t *used) {
    __shared__ uint32_t largest[2][8][32];
    __shared__ __align__(16) uint8_t tile[16384];
    wait_for_prerequisites();
    launch_dependents();
    const int64_t kb = blockIdx.x / chunks, c0 = (blockIdx.x - kb * chunks) * 128;
    if (used && !used[kb]) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row0 = kb * 128 + warp * 16;
    uint32_t v[2][16] = {}, top[2] = {0, 0};
    const int64_t col = c0 + 4 * lane, last = min(row0 + 15, k - 1);
    const uint16_t *p = x + row0 * ldx + col;
    if (col + 4 <= ncols && row0 < k && (kQuads || (row0 * ldx + col >= 3 && last * ldx + col + 8 <= (k - 1) * ldx + ncols))) {
        const auto take = [&](int i, int64_t at) {
            if constexpr (kQuads) {
                const uint2 two = *reinterpret_cast<const uint2 *>(p + at);
                v[0][i] = two.x; v[1][i] = two.y;
            } else {
                uint32_t two[2];
                unaligned<2>(p + at, two);                           // (both pieces lie within X)
                v[0][i] = two[0]; v[1][i] = two[1];
            }
        };
        if (row0 + 16 <= k) {
#pragma unroll
            for (int i = 0; i < 16; ++i) take(i, i * ldx);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                take(i, min((int64_t)i, last - row0) * ldx);
                if (row0 + i >= k) v[0][i] = v[1][i] = 0;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (col + j >= ncols) break;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (row0 + i < k) v[j >> 1][i] |= (uint32_t)p[i * ldx + j] << (16 * (j & 1));
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 16; ++i) top[h] = larger(top[h], v[h][i]);
        if (larger_of(top[h]) >= 0x7F80u) {
            top[h] = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                top[h] = larger(top[h], finite(v[h][i]));
                v[h][i] = nan_for_infinity(v[h][i]);
            }
        }
        largest[h][warp][lane] = top[h];
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 8; ++i) top[h] = __vmaxu2(top[h], largest[h][i][lane]);
        const uint32_t e[2] = {exponent_of(top[h] & 0xFFFFu), exponent_of(top[h] >> 16)};
        const float down[2] = {power_of(254u - e[0]), power_of(254u - e[1])};
        uint32_t q[2][4] = {};
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float2 a = floats(v[h][i]), b = floats(v[h][i + 1]);
            q[0][i / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a.x * down[0], b.x * down[0]), __NV_SATFINITE, __NV_E4M3) << (8 * (i & 3));
            q[1][i / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a.y * down[1], b.y * down[1]), __NV_SATFINITE, __NV_E4M3) << (8 * (i & 3));
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int c = 4 * lane + 2 * h + s;
            *reinterpret_cast<uint4 *>(tile + (c >> 3) * 1024 + (c & 7) * 128 + ((warp ^ c ^ (c >> 3)) & 7) * 16) = make_uint4(q[s][0], q[s][1], q[s][2], q[s][3]);
            if (warp == 0 && c0 + c < ncols) put_scale(scales, chunks, kb, c0 + c, e[s]);
        }
    }
    __syncthreads();
    // the atoms lie one behind the other
    const int64_t first = c0 >> 3;
    const int atoms = (int)min((int64_t)16, groups - first);
    uint4 *out = reinterpret_cast<uint4 *>(codes + (kb * groups + first) * 1024);
    for (int i = threadIdx.x; i < atoms * 64; i += 256) out[i] = reinterpret_cast<const uint4 *>(tile)[i ^ (i >> 6 & 7)];
}

// Back to bf16.  Tokens: eight threads a block of a column, 16 values each; 64 threads an atom (eight columns of a block), U blocks a thread, all codes ahead of the
// first store; a CTA takes 32 columns.  vec_ok: 2 for stores of whole sectors (32 bytes at multiples of as many), 1 for 16 bytes.
template <int U>
__global__ void __launch_bounds__(256)
dequantize_tokens_kernel(const uint8_t *codes, const uint8_t *scales, int64_t k, int64_t ncols, int64_t nblk, int64_t groups, int64_t chunks, uint16_t *y, int64_t ldy,
                         int vec_ok) {
    wait_for_prerequisites();
    launch_dependents();
    const int lane = threadIdx.x & 7, r = threadIdx.x >> 3 & 7;
    const uint32_t spans = (uint32_t)((nblk + U - 1) / U), quad = blockIdx.x / spans, g = quad * 4 + (threadIdx.x >> 6);
    uint32_t kb = (blockIdx.x - quad * spans) * U;
    const int64_t col = (int64_t)g * 8 + r;
    uint4 c[U] = {};
    uint32_t e[U] = {};
    int64_t to[U];
    int n[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int at = (int)kb * 128 + lane * 16;
        n[i] = kb < nblk && col < ncols ? (int)min((int64_t)16, k - at) : 0;
        to[i] = col * ldy + at;
        if (n[i] > 0) {
            c[i] = *reinterpret_cast<const uint4 *>(codes + ((int64_t)kb * groups + g) * 1024 + r * 128 + ((lane ^ r) << 4));
            e[i] = scales[((int64_t)kb * chunks + (col >> 7)) * kScales8 + (col & 31) * 16 + (col >> 5 & 3) * 4];
        }
        ++kb;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (n[i] <= 0) continue;
        const uint64_t up = f32x2(power_of(e[i]), power_of(e[i]));
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
        uint32_t out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] = values2(w[j / 2] >> (16 * (j & 1)), up);
        uint16_t *p = y + to[i];
        if (vec_ok == 2 && n[i] == 16) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]), "r"(out[4]), "r"(out[5]),
                         "r"(out[6]), "r"(out[7]) : "memory");
        } else if (vec_ok && n[i] == 16) {
            reinterpret_cast<uint4 *>(p)[0] = make_uint4(out[0], out[1], out[2], out[3]);
            reinterpret_cast<uint4 *>(p)[1] = make_uint4(out[4], out[5], out[6], out[7]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j < n[i]) p[j] = (uint16_t)(out[j / 2] >> (16 * (j & 1)));
        }
    }
}

// [k, ncols]: a CTA takes 128 columns of one k-block; its codes go through shared memory (rows of 132 bytes: neither side's words meet in a bank), a warp then writes
// 16 rows, four columns a lane.
__global__ void __launch_bounds__(256)
dequantize_columns_kernel(const uint8_t *codes, const uint8_t *scales, int64_t k, int64_t ncols, int64_t nblk, int64_t groups, int64_t chunks, uint16_t *y, int64_t ldy,
                          int vec_ok) {
    __shared__ uint32_t tile[128 * 33];
    wait_for_prerequisites();
    const int64_t kb = blockIdx.x / chunks, chunk = blockIdx.x - kb * chunks, c0 = chunk * 128;
    const int atoms = (int)min((int64_t)16, groups - (c0 >> 3));
    const uint32_t *from = reinterpret_cast<const uint32_t *>(codes + (kb * groups + (c0 >> 3)) * 1024);
    for (int i = threadIdx.x; i < atoms * 256; i += 256) {
        const int col = i >> 5, word = i & 31;
        tile[col * 33 + ((((word >> 2) ^ col) & 7) << 2 | (word & 3))] = from[i];
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = c0 + 4 * lane;
    if (col >= ncols) return;
    const int here = (int)min((int64_t)4, ncols - col);
    float up[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < here) up[j] = power_of(scales[(kb * chunks + chunk) * kScales8 + ((col + j) & 31) * 16 + ((col + j) >> 5 & 3) * 4]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t four[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) four[j] = j < here ? tile[(4 * lane + j) * 33 + warp * 4 + w] : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = kb * 128 + warp * 16 + w * 4 + i;
            if (row >= k) return;
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = values2(four[j] >> (8 * i) & 0xFFu, f32x2(up[j], up[j])) & 0xFFFFu;
            uint16_t *p = y + row * ldy + col;
            if (vec_ok && here == 4) {
                *reinterpret_cast<uint2 *>(p) = make_uint2(v[0] | v[1] << 16, v[2] | v[3] << 16);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < here) p[j] = (uint16_t)v[j];
            }
        }
    }
}

// Columns that a load or store may take.
int columns_of(const void *p, int64_t ld) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return a % 16 == 0 && ld % 8 == 0 ? 8 : a % 4 == 0 && ld % 2 == 0 ? 2 : 1;
}
bool aligned16(const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }

}  // namespace

cudaError_t launch_encode8(const Geometry &g, const uint16_t *w, int64_t ld, const int32_t *mask_blk_col, const uint32_t *nm_bits, uint8_t *buf,
                           cudaStream_t st) {
    const Image8 I = image8(g);
    if ((int64_t)g.nrt * g.kkeep == 0) return cudaMemsetAsync(buf, 0, kAlign, st);
    begin_encode(st);
    const cudaError_t e = launch_chained(encode8_kernel, (unsigned)(g.nrt * g.kkeep), 512, 0, st, g, w, ld, mask_blk_col, nm_bits,
                                         reinterpret_cast<int32_t *>(buf + I.col_off), buf + I.exp_off, buf + I.image_off, reinterpret_cast<uint32_t *>(buf),
                                         buf + I.used_off, columns_of(w, ld));
    end_encode();
    return e;
}

cudaError_t launch_decode8(const Geometry &g, const uint8_t *buf, uint16_t *w, int64_t ld, cudaStream_t st) {
    const Image8 I = image8(g);
    return launch_chained(decode8_kernel, (unsigned)(g.nrt * g.nblk), kDecode, 0, st, g, reinterpret_cast<const int32_t *>(buf + I.col_off), buf + I.exp_off,
                          buf + I.image_off, w, ld, columns_of(w, ld));
}

cudaError_t launch_dequantize8(const uint8_t *act, int layout, int64_t k, int64_t ncols, uint16_t *y, int64_t ldy, cudaStream_t st) {
    const Act8 a = act8(k, ncols);
    const int u = a.groups * a.nblk < 16 * 1184 || a.nblk < 2 ? 1 : 2;       // (two blocks a thread where there are CTAs enough; four take 48 registers and more time)
    const int64_t ctas = layout ? (a.groups + 3) / 4 * ((a.nblk + u - 1) / u) : a.nblk * a.chunks;
    if (ctas > 0x1FFFFFFFll) return cudaErrorInvalidValue;
    if (layout) {
        return launch_chained(u == 2 ? dequantize_tokens_kernel<2> : dequantize_tokens_kernel<1>, (unsigned)ctas, 256, 0, st, act, act + a.scale_off, k, ncols, a.nblk, a.groups, a.chunks, y, ldy,
                              reinterpret_cast<uintptr_t>(y) % 32 == 0 && ldy % 16 == 0 ? 2 : (int)aligned16(y, ldy));
    }
    const int quads = reinterpret_cast<uintptr_t>(y) % 8 == 0 && ldy % 4 == 0;
    return launch_chained(dequantize_columns_kernel, (unsigned)ctas, 256, 0, st, act, act + a.scale_off, k, ncols, a.nblk, a.groups, a.chunks, y, ldy, quads);
}

cudaError_t launch_quantize8(const uint16_t *x, int64_t ldx, int layout, int64_t k, int64_t ncols, uint8_t *act, const uint8_t *used, cudaStream_t st) {
    const Act8 a = act8(k, ncols);
    // (four blocks a thread where there are CTAs enough)
    const int u = a.groups * a.nblk >= 8 * 1184 ? 4 : 2;
    const int64_t ctas = layout ? a.groups * ((a.nblk + 2 * u - 1) / (2 * u)) : a.nblk * a.chunks;
    if (ctas > 0x7FFFFFFFll) return cudaErrorInvalidValue;
    if (layout)
        return launch_chained(u == 4 ? quantize_tokens_kernel<4> : quantize_tokens_kernel<2>, (unsigned)ctas, 256, 0, st, x, ldx, k, ncols, a.nblk, a.groups, a.chunks, act,
                              act + a.scale_off, used, (int)aligned16(x, ldx));
    const bool quads = reinterpret_cast<uintptr_t>(x) % 8 == 0 && ldx % 4 == 0;
    return launch_chained(quads ? quantize_columns_kernel<true> : quantize_columns_kernel<false>, (unsigned)ctas, 256, 0, st, x, ldx, k, ncols, a.nblk, a.groups, a.chunks,
                          act, act + a.scale_off, used);
}

}  // namespace crisp
