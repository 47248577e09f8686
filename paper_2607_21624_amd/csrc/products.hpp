// products.hpp -- operands of the matrix products behind the linear layers and the
// losses: checks and kernel arguments (host).
#pragma once

#include <hip/hip_runtime.h>

#include "rows_check.hpp"
#include "tokmap.hpp"

namespace fbl {

// bf16 operands are staged by 16-byte loads: 16-byte aligned pointers and rows; fp32 ones
// need their natural alignment.  Every span is below 2 GiB (32-bit offsets).
inline fbl_status check_operand(const RowsView& v) {
    if (!v.p) return FBL_OK;
    if (v.ld < v.width) return FBL_ERR_LAYOUT;
    if (v.ld > kMaxExtent || !v.addressable()) return FBL_ERR_UNSUPPORTED;
    if (v.es == 2 ? !v.aligned16() : !v.natural()) return FBL_ERR_ALIGN;
    return v.bytes() < ((int64_t)1 << 31) ? FBL_OK : FBL_ERR_UNSUPPORTED;
}

// Bytes a buffer resource covers for loads: the hardware drops every dword that reaches past a
// span, so one that ends inside a dword (an odd width of bf16) ends at its 16-byte
// chunk (aligned rows: the chunk never leaves the row).
inline uint32_t load_span(const RowsView& v) {
    return (uint32_t)(v.es == 2 ? (v.bytes() + 15) / 16 * 16 : v.bytes());
}

// Arguments of product `op` (FBL_PROJ_*) over tokens M, inputs K and outputs N.  The weight
// gradient's contraction runs over any number of tokens: rows past the last read as zeros,
// and the kernel clears the rest of a partial step by whole rows.
inline void product(GemmArgs& p, uint32_t op, const RowsView& a, const RowsView& b, const RowsView& c, int64_t M,
                    int64_t K, int64_t N) {
    p.a = a.p, p.b = b.p, p.c = const_cast<void*>(c.p);
    p.lda = a.ld, p.ldb = b.ld, p.ldc = c.ld;
    p.M = (int)(op == FBL_PROJ_BWD_WEIGHT ? K : M);
    p.N = (int)(op == FBL_PROJ_BWD_DATA ? K : N);
    p.K = (int)(op == FBL_PROJ_FWD ? K : op == FBL_PROJ_BWD_DATA ? N : M);
    p.a_bytes = load_span(a), p.b_bytes = load_span(b);
    p.c_bytes = (uint32_t)c.bytes();
}

constexpr int64_t kMaxWidth = (int64_t)1 << 26;  // of a layer: a launch of 32 threads a column keeps below 2^32

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// A few tokens' layer (api_linear.cpp): how many workgroups share the contraction K of a tile of M x N outputs, the bytes of
// their planes, and the product alone, its shares in `planes` (grad: B stored n-major).
int few_splits(int f32, int64_t M, int64_t K, int64_t N);
inline size_t few_ws(int splits, int64_t M, int64_t N) {
    return splits > 1 ? (size_t)splits * (size_t)M * (size_t)N * 4 : 0;
}
hipError_t launch_shares(int f32, int grad, int splits, const GemmArgs& p, float* planes, hipStream_t s);
// The tile of a bf16 forward that is not shared.
int forward_tile(int64_t M, int64_t K, int64_t N);

}  // namespace fbl
