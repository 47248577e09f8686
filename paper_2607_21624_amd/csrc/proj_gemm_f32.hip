// proj_gemm_f32.hip -- the projection products for fp32 storage, gfx950.
//
// The same three products as proj_gemm.hip (Y = X W, dX = dY W^T,
// dW = X^T dY; section 4.1's matrix-product gradients, no operand transposed
// in memory) for tensors stored in fp32, with fp32 accumulation on
// v_mfma_f32_32x32x2_f32 (eight per 16-deep chunk, cdna4.hpp's fragment
// convention).  Any extents, any leading dimensions, 4-byte alignment.
//
// The fp32 MFMA rate bounds it (157 TFLOP/s; a large library product reaches
// 138): one 32x32x2 product takes 64 cycles, so LDS has time for column reads
// by single floats and any wavefront tile, and what counts is that every CU has
// work and that loads are hidden.  Operands go through registers (16-byte
// loads, 4-byte alignment) into LDS in their stored orientation, the next step's
// loads under the current step's products; small outputs take small tiles whose
// wavefronts split the contraction.  512 tokens x 768 x 3072: Y 112 -> 26, dX
// 336 -> 30, dW 91 -> 28 us (82 .. 94 TFLOP/s) against 64 x 64 tiles staged by
// single floats; 4096 x 2048 x 2048 252 .. 293 us (117 .. 136 TFLOP/s).
#include "gemm_f32.hpp"

namespace fbl {

namespace {

hipError_t launch_f32(int a_kmajor, int b_nmajor, int tile, const GemmArgs& p, hipStream_t stream) {
    if (a_kmajor && b_nmajor) return hipErrorInvalidValue;  // no product reads both that way
    if (a_kmajor) return launch_f32_tile<true, false, PlainStoreF32>(tile, p, stream);
    return b_nmajor ? launch_f32_tile<false, true, PlainStoreF32>(tile, p, stream)
                    : launch_f32_tile<false, false, PlainStoreF32>(tile, p, stream);
}

}  // namespace

hipError_t launch_proj_gemm_f32(int a_kmajor, int b_nmajor, const GemmArgs& p, hipStream_t stream) {
    return launch_f32(a_kmajor, b_nmajor, f32_tile(p), p, stream);
}

void proj_gemm_f32_info(const GemmArgs& p, int32_t* info) {
    const F32Tile& t = kF32Tiles[f32_tile(p)];
    const int32_t v[6] = {t.bm, t.bn, t.bk, t.wm * t.wn * t.wk, t.wk,
                          (int32_t)std::min<int64_t>(f32_workgroups(t, p), INT32_MAX)};
    for (int i = 0; i < 6; ++i) info[i] = v[i];
}

}  // namespace fbl
