// The 8-bit product of a few columns (tokens) without tensor cores: one to four columns, where the chain through tensor memory is longer than the work.
//
//   Y[r, c] = act(sum over kept blocks b of 2^(Ew + Ex[b, c]) sum_k qw[r, k] qx[k, c] + bias[r])
//
// The weights are read once, and that bounds a product (4096 x 4096: 16.8 MB, 2.6 us at the copy rate).  A CTA takes the eight rows of an atom (block8.h) and its warps
// the kept blocks in turn: a lane reads 32 bytes of every block, two rows' 16-byte chunks, for four blocks at a time, so that all of the weights are under way at
// once.  Meanwhile the CTA quantises X into shared memory, block by block (its codes as fp32, and the scales).  Codes are multiplied in fp32: products of two codes are
// exact, a block's sum is scaled once, and the sums of lanes and warps are added in a fixed order.
// Not kept: mma.sync on fp16 codes, 16 rows a CTA.  The quantisation of X in every CTA is what is left then: 4096 x 4096 with half of its blocks, 4 tokens 5.3 instead of 6.5 us, but
// 2048 x 8192 1 token 9.5 instead of 8.0, 512 x 4608 with a quarter 3.0 instead of 2.5 (2.3 since a block's scales are made once a column).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "block8.cuh"
#include "block8.h"

namespace crisp {

using namespace block8;

namespace {

constexpr int kFewWarps = 8, kFewBlocks = 4;                  // warps a CTA, blocks of a warp under way
constexpr int kFewBytes = 100 * 1024;                         // most that X's codes may take in shared memory, at 513 bytes a block of a column
constexpr int kFewEach = 128 * 4 + 8;                         // bytes a block of a column: codes as fp32, and the two factors

// A column's 128 codes of a block in shared memory: 16-byte pieces of the 16 codes of chunk c at piece ^ (c / 2 % 4), so that eight lanes that read one piece of eight
// chunks touch all banks.
__device__ __forceinline__ float4 *piece_at(float *block, int chunk, int piece) {
    return reinterpret_cast<float4 *>(block + chunk * 16 + ((piece ^ (chunk >> 1 & 3)) << 2));
}

template <int C>
__global__ void __launch_bounds__(32 * kFewWarps, C == 1 ? 4 : 2)
few8_kernel(const __grid_constant__ FewParams p) {
    extern __shared__ __align__(16) uint8_t shared[];
    float *codes = reinterpret_cast<float *>(shared);         // [kept block][column][128]
    // [kept block][column]: 2^(Ew + Ex) as two factors, each of half the sum of the exponents.  That sum may be out of fp32's range where the product is not, and so may
    // the product with one of the two scales.
    float2 *factors = reinterpret_cast<float2 *>(shared + (size_t)p.kkeep * C * 512);
    __shared__ float sums[kFewWarps][8][C];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rt = blockIdx.x >> 4, atom = blockIdx.x & 15;
    const uint8_t *entries = p.image + (int64_t)rt * p.kkeep * kEntry8;
    if (!p.early) wait_for_prerequisites();
    const bool here = rt * 128 + atom * 8 < p.rows;
    // the warp's first blocks: lane reads chunk lane % 8 of rows lane / 8 and lane / 8 + 4
    uint4 w[kFewBlocks][2];
    const auto fetch = [&](int e0) {
#pragma unroll
        for (int i = 0; i < kFewBlocks; ++i) {
            const int e = e0 + i * kFewWarps;
            if (e < p.kkeep) {
                const uint8_t *at = entries + (int64_t)e * kEntry8;
                const uint4 *a = reinterpret_cast<const uint4 *>(at + atom * 1024);
                w[i][0] = __ldcg(a + lane); w[i][1] = __ldcg(a + 32 + lane);
            }
        }
    };
    if (here) fetch(warp);
    if (p.early) wait_for_prerequisites();
    if (!here) return;                                        // (the whole CTA)

    // X: half a warp a column of a block, eight values a lane
    const int half = lane >> 4, l16 = lane & 15;
    for (int u = warp * 2 + half; u < p.kkeep * C + (p.kkeep * C & 1); u += 2 * kFewWarps) {
        const bool in = u < p.kkeep * C;
        const int e = in ? u / C : 0, c = in ? u - e * C : 0;
        const int at = (p.all ? e : __ldcg(p.blk_col + (int64_t)rt * p.kkeep + e)) * 128 + l16 * 8;
        const uint32_t ew = __ldcg(entries + (int64_t)e * kEntry8 + kTile8);
        uint32_t v[4] = {};
        if (in && c < p.cols) {
            if (p.x_layout == 1 && p.x_vec && at + 8 <= p.k) {
                const uint4 q = *reinterpret_cast<const uint4 *>(p.x + c * p.ldx + at);
                v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (at + j < p.k) v[j / 2] |= (uint32_t)(p.x_layout == 1 ? p.x[c * p.ldx + at + j] : p.x[(int64_t)(at + j) * p.ldx + c]) << (16 * (j & 1));
            }
        }
        uint32_t top = larger(larger(larger(larger(0, v[0]), v[1]), v[2]), v[3]);
        if (__any_sync(0xFFFFFFFFu, larger_of(top) >= 0x7F80u)) {
            top = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                top = larger(top, finite(v[j]));
                v[j] = nan_for_infinity(v[j]);
            }
        }
        uint32_t m = larger_of(top);
#pragma unroll
        for (int d = 8; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
        const uint32_t e8 = exponent_of(m);
        const float down = power_of(254u - e8);
        float2 q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes2(v[j], down), __NV_E4M3)));
        if (in) {
            float *block = codes + (e * C + c) * 128;
            *piece_at(block, l16 >> 1, (l16 & 1) * 2) = make_float4(q[0].x, q[0].y, q[1].x, q[1].y);
            *piece_at(block, l16 >> 1, (l16 & 1) * 2 + 1) = make_float4(q[2].x, q[2].y, q[3].x, q[3].y);
            if (l16 == 0) factors[e * C + c] = make_float2(power_of((ew + e8) >> 1), power_of((ew + e8 + 1) >> 1));
        }
    }
    __syncthreads();

    float acc[2][C] = {};                                     // rows lane / 8 and lane / 8 + 4
    for (int e0 = warp; e0 < p.kkeep; e0 += kFewWarps * kFewBlocks) {
#pragma unroll
        for (int i = 0; i < kFewBlocks; ++i) {
            const int e = e0 + i * kFewWarps;
            if (e >= p.kkeep) break;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = (lane >> 3) + 4 * r, chunk = (lane & 7) ^ row;
                float2 q[8];
                const uint32_t words[4] = {w[i][r].x, w[i][r].y, w[i][r].z, w[i][r].w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    q[j] = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(words[j / 2] >> (16 * (j & 1))), __NV_E4M3)));
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float *block = codes + (e * C + c) * 128;
                    float s[4] = {};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 f = *piece_at(block, chunk, j);
                        s[0] = fmaf(q[2 * j].x, f.x, s[0]); s[1] = fmaf(q[2 * j].y, f.y, s[1]);
                        s[2] = fmaf(q[2 * j + 1].x, f.z, s[2]); s[3] = fmaf(q[2 * j + 1].y, f.w, s[3]);
                    }
                    const float2 f = factors[e * C + c];
                    acc[r][c] = fmaf(((s[0] + s[1]) + (s[2] + s[3])) * f.x, f.y, acc[r][c]);
                }
            }
        }
        if (e0 + kFewWarps * kFewBlocks < p.kkeep) fetch(e0 + kFewWarps * kFewBlocks);
    }
    launch_dependents();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int d = 4; d; d >>= 1) acc[r][c] += __shfl_xor_sync(0xFFFFFFFFu, acc[r][c], d);
            if ((lane & 7) == 0) sums[warp][(lane >> 3) + 4 * r][c] = acc[r][c];
        }
    __syncthreads();
    if (threadIdx.x < 8 * C) {
        const int c = threadIdx.x >> 3, row = threadIdx.x & 7, at = rt * 128 + atom * 8 + row;
        if (c < p.cols && at < p.rows) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < kFewWarps; ++i) v += sums[i][row][c];
            if (p.bias != nullptr) v += p.bias[at];
            if (p.relu && v < 0.f) v = 0.f;                   // (a NaN stays)
            const int64_t to = p.y_layout == 0 ? at * p.ldy + c : c * p.ldy + at;
            if (p.f32) reinterpret_cast<float *>(p.y)[to] = v;
            else reinterpret_cast<__nv_bfloat16 *>(p.y)[to] = __float2bfloat16_rn(v);
        }
    }
}

template <int C>
cudaError_t launch(const FewParams &p, unsigned ctas, int device, cudaStream_t st) {
    constexpr int kMaxDevices = 64;
    static std::atomic<bool> configured[kMaxDevices];
    if (device < 0 || device >= kMaxDevices) return cudaErrorInvalidDevice;
    if (!configured[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(few8_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewBytes / 513 * kFewEach);
        if (e != cudaSuccess) return e;
        configured[device].store(true, std::memory_order_relaxed);
    }
    return launch_chained(few8_kernel<C>, ctas, 32 * kFewWarps, (size_t)p.kkeep * C * kFewEach, st, p);
}

}  // namespace

// Up to four columns whose codes fit in shared memory, and products of no more than 12 million weights times columns: beyond, the multiply-adds take longer than the
// chain through tensor memory.  In a row, us here and there: 300 x 500 1 column 2.2 and 4.7, 4 columns 2.4 and 5.0; 1024 x 4096 3.2 and 6.0, 2 columns 4.5 and 6.0,
// 4 columns 7.5 and 6.4; 4096 x 4096 with half of its blocks 3.9 and 6.2, 4 columns 11.9 and 6.5.  (One column alone crosses later: 4096 x 4096 5.9 and 7.0, 2048 x 8192 6.9 and
// 7.4.  The line was drawn when these took 7.5 and 8.0 here.)
bool few8(const Geometry &g, int64_t ncols) {
    return ncols <= 4 && g.kkeep > 0 && (int64_t)g.kkeep * ncols * 513 <= kFewBytes && (int64_t)g.rows * g.kkeep * 128 * ncols <= 12000000;
}

cudaError_t launch_few8(const FewParams &p, int nrt, int device, cudaStream_t st) {
    const unsigned ctas = (unsigned)nrt * 16;
    switch (p.cols) {
        case 1: return launch<1>(p, ctas, device, st);
        case 2: return launch<2>(p, ctas, device, st);
        case 3: return launch<3>(p, ctas, device, st);
        default: return launch<4>(p, ctas, device, st);
    }
}

}  // namespace crisp
