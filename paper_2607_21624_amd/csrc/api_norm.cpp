// api_norm.cpp -- the C ABI of layer norm: validation and dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kernels.hpp"
#include "rows_check.hpp"

using fbl::overlap;
using fbl::RowsView;

namespace {

// Workgroups of the backward: each walks every groups-th block of rows and leaves one row of
// partial sums, so more of them hide more latency and fewer cost fewer bytes.
int norm_groups(int f32, int64_t M, int N) {
    const int64_t blocks = (M + fbl::layer_norm_slots(f32, N) - 1) / fbl::layer_norm_slots(f32, N);
    // 16 wavefronts a row fill a CU alone (2048 x 16384 bf16, 256 workgroups 59 us, 512 86); else two a CU (16384 x
    // 4096: 256 85, 512 84, 1024 95 us; 16384 x 1600: 57, 43, 40; 4099 x 1001: 13.8, 13.7, 17.8)
    return (int)std::min<int64_t>(blocks, fbl::layer_norm_wide(f32, N) ? 256 : 512);
}

size_t norm_ws(int f32, int64_t M, int N) { return (size_t)norm_groups(f32, M, N) * 2 * (size_t)N * 4; }

fbl_status norm_shape(int32_t dtype, int64_t M, int64_t N) {
    if (!fbl::dtype_size(dtype)) return FBL_ERR_DTYPE;
    if (!fbl::extent(M) || !fbl::extent(N)) return FBL_ERR_SHAPE;
    if (N > fbl::kNormMaxWidth) return FBL_ERR_UNSUPPORTED;
    return FBL_OK;
}

}  // namespace

extern "C" {

fbl_status fbl_layer_norm_fwd(int32_t dtype, int64_t M, int64_t N, const void* x, int64_t ldx, const void* weight,
                              const void* bias, float eps, void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
    fbl_status st = norm_shape(dtype, M, N);
    if (st != FBL_OK) return st;
    if (!x || !y || !mean != !rstd) return FBL_ERR_NULL;
    if (!std::isfinite(eps) || eps < 0) return FBL_ERR_ARG;
    if (ldx < N || ldy < N || ldx > fbl::kMaxExtent || ldy > fbl::kMaxExtent) return FBL_ERR_LAYOUT;
    const int64_t es = fbl::dtype_size(dtype);
    const RowsView in[] = {{x, M, N, ldx, es}, {weight, 1, N, N, es}, {bias, 1, N, N, es}};
    const RowsView out[] = {{y, M, N, ldy, es}, {mean, 1, M, M, 4}, {rstd, 1, M, M, 4}};
    for (const RowsView& v : in) {
        if (!v.addressable()) return FBL_ERR_SHAPE;
        if (!v.natural()) return FBL_ERR_ALIGN;
    }
    for (int i = 0; i < 3; ++i) {
        if (!out[i].addressable()) return FBL_ERR_SHAPE;
        if (!out[i].natural()) return FBL_ERR_ALIGN;
        for (const RowsView& v : in)
            if (overlap(out[i], v)) return FBL_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return FBL_ERR_ARG;
    }
    fbl::NormArgs a{};
    a.x = x, a.w = weight, a.b = bias, a.y = y, a.mean = mean, a.rstd = rstd;
    a.ldx = ldx, a.ldy = ldy, a.M = M, a.N = (int)N, a.eps = eps;
    const hipError_t e = fbl::launch_layer_norm_fwd(dtype == FBL_F32, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

fbl_status fbl_layer_norm_bwd_workspace(int32_t dtype, int64_t M, int64_t N, size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    const fbl_status st = norm_shape(dtype, M, N);
    if (st == FBL_OK) *bytes = norm_ws(dtype == FBL_F32, M, (int)N);
    return st;
}

fbl_status fbl_layer_norm_bwd(int32_t dtype, int64_t M, int64_t N, const void* dy, int64_t lddy, const void* x,
                              int64_t ldx, const void* weight, const float* mean, const float* rstd, void* dx,
                              int64_t lddx, void* dweight, void* dbias, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = norm_shape(dtype, M, N);
    if (st != FBL_OK) return st;
    if (!dy || !x || !mean || !rstd || !dx) return FBL_ERR_NULL;
    if (lddy < N || ldx < N || lddx < N || std::max({lddy, ldx, lddx}) > fbl::kMaxExtent) return FBL_ERR_LAYOUT;
    const int64_t es = fbl::dtype_size(dtype);
    const bool sums = dweight || dbias;
    const size_t need = sums ? norm_ws(dtype == FBL_F32, M, (int)N) : 0;
    if (sums && (!ws || ws_bytes < need)) return FBL_ERR_WORKSPACE;
    const RowsView in[] = {{dy, M, N, lddy, es}, {x, M, N, ldx, es}, {weight, 1, N, N, es},
                           {mean, 1, M, M, 4},   {rstd, 1, M, M, 4}};
    const RowsView out[] = {{dx, M, N, lddx, es}, {dweight, 1, N, N, es}, {dbias, 1, N, N, es},
                            {sums ? ws : nullptr, 1, (int64_t)(need / 4), (int64_t)(need / 4) + 1, 4}};
    for (const RowsView& v : in) {
        if (!v.addressable()) return FBL_ERR_SHAPE;
        if (!v.natural()) return FBL_ERR_ALIGN;
    }
    for (int i = 0; i < 4; ++i) {
        if (!out[i].addressable()) return FBL_ERR_SHAPE;
        if (!out[i].natural()) return FBL_ERR_ALIGN;
        for (const RowsView& v : in)
            if (overlap(out[i], v)) return FBL_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return FBL_ERR_ARG;
    }
    fbl::NormArgs a{};
    a.x = x, a.dy = dy, a.w = weight, a.dx = dx, a.dw = dweight, a.db = dbias;
    a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
    a.part = sums ? static_cast<float*>(ws) : nullptr;
    a.ldx = ldx, a.lddy = lddy, a.lddx = lddx, a.M = M, a.N = (int)N;
    a.groups = norm_groups(dtype == FBL_F32, M, (int)N);
    const hipError_t e = fbl::launch_layer_norm_bwd(dtype == FBL_F32, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

}  // extern "C"
