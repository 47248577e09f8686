// proj_gemm.hip -- projection matrix products on token-major operands, bf16,
// gfx950.
//
// One kernel template computes C[M, N] = sum_k A(m, k) B(k, n) (fp32
// accumulation, bf16 result) for the three products of a linear layer:
//   forward          Y  = X W      A = X  [M, K] rows,   B = W  [K, N] rows
//   data gradient    dX = dY W^T   A = dY [M, N] rows,   B = W read as [N, K]
//   weight gradient  dW = X^T dY   A = X read as [K, M], B = dY [M, N] rows
// Section 4.1 classes these as forward-tensor-dependent: the gradients read
// the stored X, W and dY along other axes than the forward (section 4.2: the
// forward reduces along K, the gradients along N and along the tokens M).
// No operand is ever transposed in memory.  Each operand tile is staged once
// into LDS by DMA in its stored orientation (the R-Tile of section 4.2, with
// the XOR swizzle of stage.hpp) and read back either
//   row-wise      (ds_read_b128: 8 consecutive elements of one stored row)
//                 when the contraction runs along the stored rows, or
//   transposed    (ds_read_b64_tr_b16: one element of each of 4 stored rows)
//                 when it runs down the stored columns.
// Both read kinds hand lane group g (lane / 32) contraction elements
// 8g .. 8g+7 of a 16-element chunk, in order, so any pair of them forms a
// consistent MFMA operand pair.
//
// Extents need not be multiples of the tile.  Operand rows past the end of
// an operand read as zeros (buffer resources bound each operand's span);
// columns past an operand's width read whatever follows in memory, which
// only ever meets output rows/columns that are not stored -- and, along the
// contraction, the positions of a partial last step, which are zeroed in LDS
// before that step's products.
//
// Workgroup (gemm_tiles.hpp): a WM x WN grid of wavefront tiles over a
// BM x BN output tile, each computed by WK wavefronts that split every step's
// contraction; BK-deep steps through NS LDS stages (NS - 1 in flight).  The
// WK partial sums of a wavefront tile are added through LDS at the end, in a
// fixed order.  The products accumulate C^T tiles (lane <-> m, in-lane n), so
// each lane stores four consecutive outputs of a row.
#include "gemm_bf16.hpp"

namespace fbl {

hipError_t launch_proj_gemm(int a_kmajor, int b_nmajor, int tile, const GemmArgs& p, hipStream_t stream) {
    if (tile < 0 || tile >= kGemmTileCount) return hipErrorInvalidValue;
    if (a_kmajor)
        return b_nmajor ? launch_gemm_tile<true, true, PlainStore>(tile, p, stream)
                        : launch_gemm_tile<true, false, PlainStore>(tile, p, stream);
    return b_nmajor ? launch_gemm_tile<false, true, PlainStore>(tile, p, stream)
                    : launch_gemm_tile<false, false, PlainStore>(tile, p, stream);
}

}  // namespace fbl
