// The 8-bit forms of weights and activations: e4m3 codes with an exponent for each block of 128, laid out as the tensor cores take them.
//
// A tile of codes is rows (weights) or columns (activations) of 128 bytes, one k-block of one of them each; eight of those form an atom of 1024 bytes whose
// 16-byte chunks are swizzled (chunk j of row r sits at j ^ (r % 8)), the layout that 128-byte-swizzled operands have in shared memory.
//
//   weights       per kept block 16 atoms (128 rows), then 512 bytes of scales: the block's exponent for every row, in the order that tcgen05.cp 32x128b takes
//                 (row r's four bytes at (r % 32) * 16 + (r / 32) * 4, all the same)
//   activations   codes [k-block][8 columns] of atoms; scales [k-block][128 columns] of 512 bytes in that order.  (Of a row's four bytes an MMA takes one, named in its
//                 instruction.  Packed with those of three other k-blocks they would be a quarter of the size, but a tile fetches 512 bytes a block either way, and the issuing
//                 thread would have to know the block's number.)
#pragma once

#include "crisp_internal.h"

namespace crisp {

constexpr uint32_t kTile8 = 16384, kScales8 = 512, kEntry8 = kTile8 + kScales8;

struct Image8 {                              // where the parts of a weight buffer lie
    size_t col_off, exp_off, used_off, image_off, total;
};
inline Image8 image8(const Geometry &g) {
    const size_t n = (size_t)g.nrt * g.kkeep;
    Image8 i;
    i.col_off = kAlign;                      // (the status word in front)
    i.exp_off = i.col_off + align_up(n * 4);
    i.used_off = i.exp_off + align_up(n);    // a byte a k-block: whether any row tile keeps it
    i.image_off = i.used_off + align_up((size_t)g.nblk);
    i.total = i.image_off + align_up(n * kEntry8);
    return i;
}
struct Act8 {                                // and those of activations
    int64_t nblk, groups, chunks;            // k-blocks, groups of 8 columns, of 128 columns
    size_t scale_off, total;
};
inline Act8 act8(int64_t k, int64_t ncols) {
    Act8 a;
    a.nblk = (k + 127) / 128; a.groups = (ncols + 7) / 8; a.chunks = (ncols + 127) / 128;
    a.scale_off = (size_t)a.nblk * a.groups * 1024;
    a.total = a.scale_off + (size_t)a.nblk * a.chunks * kScales8;
    return a;
}

// Products of a few columns on the CUDA cores (spmm8_few.cu): x is quantised by every CTA.
struct FewParams {
    const uint8_t *image;
    const int32_t *blk_col;
    const uint16_t *x;
    void *y;
    const float *bias;
    int64_t ldx, ldy;
    int rows, k, kkeep, all, cols, x_layout, x_vec, y_layout, f32, relu, early;
};
bool few8(const Geometry &g, int64_t ncols);
cudaError_t launch_few8(const FewParams &p, int nrt, int device, cudaStream_t st);

cudaError_t launch_encode8(const Geometry &g, const uint16_t *w, int64_t ld, const int32_t *mask_blk_col, const uint32_t *nm_bits, uint8_t *buf,
                           cudaStream_t st);
cudaError_t launch_decode8(const Geometry &g, const uint8_t *buf, uint16_t *w, int64_t ld, cudaStream_t st);
// used: a byte a k-block, 0 for those that are left out, or nullptr for all
cudaError_t launch_quantize8(const uint16_t *x, int64_t ldx, int layout, int64_t k, int64_t ncols, uint8_t *act, const uint8_t *used, cudaStream_t st);

cudaError_t launch_dequantize8(const uint8_t *act, int layout, int64_t k, int64_t ncols, uint16_t *y, int64_t ldy, cudaStream_t st);

}  // namespace crisp
