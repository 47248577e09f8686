// api_gated.cpp -- the C ABI of gated layers: validation and dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act.hpp"
#include "kernels.hpp"
#include "products.hpp"

using fbl::align256;
using fbl::few_splits;
using fbl::few_ws;
using fbl::overlap;
using fbl::RowsView;

namespace {

template <int ACT>
hipError_t run_act(int f32, int tile, const fbl::GatedArgs& p, hipStream_t s) {
    return f32 ? fbl::launch_gated_gemm_f32<ACT>(p, s) : fbl::launch_gated_gemm<ACT>(tile, p, s);
}
hipError_t run_gated_gemm(int f32, int act, int tile, const fbl::GatedArgs& p, hipStream_t s) {
    switch (act) {
        case FBL_ACT_NONE: return run_act<fbl::kActNone>(f32, tile, p, s);
        case FBL_ACT_RELU: return run_act<fbl::kActRelu>(f32, tile, p, s);
        case FBL_ACT_GELU: return run_act<fbl::kActGelu>(f32, tile, p, s);
        case FBL_ACT_GELU_TANH: return run_act<fbl::kActGeluTanh>(f32, tile, p, s);
        default: return run_act<fbl::kActSilu>(f32, tile, p, s);
    }
}

// The tile of a bf16 product of `cols` columns over a contraction kc: the forward's (2F columns) or the data gradient's
// (F).  Both write their tiles by rows, which the costs behind the products' own choice do not know, and more of them: from
// about two thirds of a round of 256 x 256 tiles on those are the fastest (us, own choice and 256 x 256: forward 8192 x
// 1024 -> 4096 195 and 144, 2048 x 1024 -> 2816 34.4 and 31.7, 1500 x 1024 -> 4096 33.9 and 31.9; gradient 4096 x 2048 ->
// 8192 172 and 162, 2000 x 2048 -> 5632 64 and 61; with 128 of them 1024 x 2048 -> 4096 40.9 and 49.7).  Below that the
// forward's single round of 128 x 128 tiles runs them on 8 wavefronts that split each step (128 x 4096 -> 11008 50.6 and 38.5, 256
// x 2048 -> 5632 29.1 and 22.3, 700 x 2048 -> 2048 25.3 and 21.6; 640 x 640 -> 2560 13.2 and 14.1), and the
// gradient's two rounds run two workgroups a CU (1500 x 1024 -> 4096 36.3 and 24.7, 2048 x 1024 -> 2816 27.4 and 23.0).
int gated_tile(int grad, int64_t M, int64_t cols, int64_t kc) {
    const uint32_t op = grad ? FBL_PROJ_BWD_DATA : FBL_PROJ_FWD;
    const int64_t K = grad ? cols : kc, N = grad ? kc : cols;
    const int tuned = fbl_proj_tuned_tile(op, M, K, N);
    if (tuned >= 0) return tuned;
    if ((M + 255) / 256 * ((cols + 255) / 256) >= 160 && M > 256) return 20;
    const int64_t t128 = (M + 127) / 128 * ((cols + 127) / 128);
    if (!grad && M > 64 && t128 >= 160 && t128 <= 256 && kc >= 768) return 8;
    if (grad && t128 > 256 && t128 <= 512) return 4;
    return grad ? fbl::proj_auto_tile(op, M, K, N) : fbl::forward_tile(M, K, N);
}

// Workgroups that share the contraction K of a tile of a few tokens' forward.  bf16 up to 64 tokens: as many as give every CU
// one of its 128-column tiles, of 384 values and more each (us, cold weights, 1 token, alone / so shared / two a CU, as
// linear layers are: 2048 -> 4096 15.1 / 11.9 / 12.9, 2048 -> 8192 19.9 / 16.2 / 17.1, 4096 -> 4096 27.1 / 17.9 / 20.2, 4096 ->
// 8192 37.3 / 27.3 / 28.9, 4096 -> 14336 44.4 / 44.4 / 47.7; 64 tokens 2048 -> 8192 23.1 / 19.7 / 22.8; 1536 -> 4096 12.0 /
// 10.6, but 1024 -> 4096 8.9 / 9.6).
int forward_splits(int f32, int64_t M, int64_t K, int64_t F) {
    if (f32 || M > 64 || 2 * M * F >= (int64_t)1 << 29) return few_splits(f32, M, K, 2 * F);
    if (K <= 1024) return 1;
    return (int)std::max<int64_t>(1, std::min(256 / ((2 * F + 127) / 128), K / 384));
}

// Workspace of the data gradient, a function of the shape: planes of dh, and partial sums of dz: as many rows of them as any
// tile writes (linear_grad_groups), or one for each of a few tokens where that is more.  A shape whose contraction would be
// shared needs room for a tile's rows too: a caller may name a tile, which shares nothing.
struct GatedWs {
    size_t sums, total;
    int splits;
};
GatedWs gated_ws(int f32, int64_t M, int64_t F, int64_t N) {
    GatedWs w;
    w.splits = few_splits(f32, M, N, F);
    w.sums = align256(few_ws(w.splits, M, F));
    w.total = w.sums + (size_t)(w.splits > 1 ? std::max(M, M / 32 + 4) : M / 32 + 4) * 2 * (size_t)F * 4;
    return w;
}

fbl_status gated_shape(int32_t dtype, uint32_t act, int64_t M, int64_t K, int64_t F) {
    const int64_t es = fbl::dtype_size(dtype);
    if (!es) return FBL_ERR_DTYPE;
    if (act > FBL_ACT_SILU) return FBL_ERR_ARG;
    if (!fbl::extent(M) || !fbl::extent(K) || !fbl::extent(F)) return FBL_ERR_SHAPE;
    if (K > fbl::kMaxWidth || 2 * F > fbl::kMaxWidth) return FBL_ERR_UNSUPPORTED;
    if (M * 2 * F >= ((int64_t)1 << 31) / es) return FBL_ERR_UNSUPPORTED;  // factors, dz
    return FBL_OK;
}

}  // namespace

extern "C" {

fbl_status fbl_gated_fwd_workspace(int32_t dtype, int64_t M, int64_t K, int64_t F, size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    const fbl_status st = gated_shape(dtype, FBL_ACT_NONE, M, K, F);
    if (st == FBL_OK) *bytes = few_ws(forward_splits(dtype == FBL_F32, M, K, F), M, 2 * F);
    return st;
}

fbl_status fbl_gated_fwd(int32_t dtype, uint32_t act, int64_t M, int64_t K, int64_t F, const void* x, int64_t ldx,
                         const void* w, int64_t ldw, const void* bias, void* h, int64_t ldh, void* factors,
                         int64_t ldf, int32_t tile, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = gated_shape(dtype, act, M, K, F);
    if (st != FBL_OK) return st;
    if (!x || !w || !h) return FBL_ERR_NULL;
    const int es = (int)fbl::dtype_size(dtype), f32 = es == 4;
    const RowsView vx{x, M, K, ldx, es}, vw{w, K, 2 * F, ldw, es}, vb{bias, 1, 2 * F, (2 * F + 7) / 8 * 8, es},
        vh{h, M, F, ldh, es}, vf{factors, M, 2 * F, ldf, es};
    for (const RowsView* v : {&vx, &vw, &vb, &vh, &vf})
        if ((st = fbl::check_operand(*v)) != FBL_OK) return st;
    if (es == 2 && (K % 8 || F % 8)) return FBL_ERR_UNSUPPORTED;
    if (tile < FBL_GEMM_TILE_AUTO || tile >= fbl::kGemmTileCount || (es == 4 && tile != FBL_GEMM_TILE_AUTO))
        return FBL_ERR_ARG;
    for (const RowsView* out : {&vh, &vf})
        for (const RowsView* in : {&vx, &vw, &vb})
            if (overlap(*out, *in)) return FBL_ERR_ARG;
    if (overlap(vh, vf)) return FBL_ERR_ARG;
    // with a workspace for the shares of it
    const int splits = ws && tile == FBL_GEMM_TILE_AUTO ? forward_splits(f32, M, K, F) : 1;
    if (splits > 1) {
        const size_t need = few_ws(splits, M, 2 * F);
        if (ws_bytes < need) return FBL_ERR_WORKSPACE;
        const RowsView vws{ws, 1, (int64_t)need, (int64_t)need, 1};
        if (vws.begin() % 16) return FBL_ERR_ALIGN;
        for (const RowsView* v : {&vx, &vw, &vb, &vh, &vf})
            if (overlap(vws, *v)) return FBL_ERR_ARG;
    }
    fbl::GatedArgs p{};
    fbl::product(p, FBL_PROJ_FWD, vx, vw, vh, M, K, 2 * F);
    p.bias = bias, p.factors = factors, p.ldf = ldf, p.f_bytes = factors ? (uint32_t)vf.bytes() : 0;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!f32 && tile == FBL_GEMM_TILE_AUTO) tile = gated_tile(0, M, 2 * F, K);
    hipError_t e;
    if (splits > 1) {
        float* const planes = static_cast<float*>(ws);
        e = fbl::launch_shares(f32, 0, splits, p, planes, s);
        if (e == hipSuccess) e = fbl::launch_gated_finish(f32, (int)act, p, planes, splits, s);
    } else {
        e = run_gated_gemm(f32, (int)act, tile, p, s);
    }
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

fbl_status fbl_gated_bwd_workspace(int32_t dtype, int64_t M, int64_t F, int64_t N, size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    const fbl_status st = gated_shape(dtype, FBL_ACT_NONE, M, N, F);
    if (st == FBL_OK) *bytes = gated_ws(dtype == FBL_F32, M, F, N).total;
    return st;
}

fbl_status fbl_gated_bwd(int32_t dtype, int64_t M, int64_t F, int64_t N, const void* dy, int64_t lddy, const void* wd,
                         int64_t ldwd, const void* factors, int64_t ldf, void* dz, int64_t lddz, void* dbias,
                         int32_t tile, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = gated_shape(dtype, FBL_ACT_NONE, M, N, F);
    if (st != FBL_OK) return st;
    if (!dy || !wd || !factors || !dz) return FBL_ERR_NULL;
    const int es = (int)fbl::dtype_size(dtype), f32 = es == 4;
    const RowsView vdy{dy, M, N, lddy, es}, vwd{wd, F, N, ldwd, es}, vf{factors, M, 2 * F, ldf, es}, vdz{dz, M, 2 * F, lddz, es},
        vdb{dbias, 1, 2 * F, 2 * F, es};
    for (const RowsView* v : {&vdy, &vwd, &vf, &vdz})
        if ((st = fbl::check_operand(*v)) != FBL_OK) return st;
    if (!vdb.natural()) return FBL_ERR_ALIGN;
    if (es == 2 && (N % 8 || F % 8)) return FBL_ERR_UNSUPPORTED;
    if (tile < FBL_GEMM_TILE_AUTO || tile >= fbl::kGemmTileCount || (es == 4 && tile != FBL_GEMM_TILE_AUTO))
        return FBL_ERR_ARG;
    const GatedWs gw = gated_ws(f32, M, F, N);
    const bool shared = ws && tile == FBL_GEMM_TILE_AUTO && gw.splits > 1;
    const size_t need = shared || dbias ? gw.total : 0;
    if (need && (!ws || ws_bytes < need)) return FBL_ERR_WORKSPACE;
    const RowsView vws{need ? ws : nullptr, 1, (int64_t)need, (int64_t)need + 1, 1};
    if (vws.begin() % 16) return FBL_ERR_ALIGN;
    const RowsView* outs[] = {&vdz, &vdb, &vws};
    for (int i = 0; i < 3; ++i) {
        for (const RowsView* in : {&vdy, &vwd, &vf})
            if (overlap(*outs[i], *in)) return FBL_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i], *outs[j])) return FBL_ERR_ARG;
    }
    const RowsView vdh{dz, M, F, lddz, es};
    fbl::GatedArgs p{};
    fbl::product(p, FBL_PROJ_BWD_DATA, vdy, vwd, vdh, M, F, N);
    p.c_bytes = (uint32_t)vdz.bytes();
    p.factors = const_cast<void*>(factors), p.ldf = ldf, p.f_bytes = fbl::load_span(vf);
    if (dbias) p.sums = reinterpret_cast<float*>(static_cast<char*>(ws) + gw.sums);
    if (!f32 && tile == FBL_GEMM_TILE_AUTO) tile = gated_tile(1, M, F, N);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (shared) {
        float* const planes = static_cast<float*>(ws);
        e = fbl::launch_shares(f32, 1, gw.splits, p, planes, s);
        if (e == hipSuccess) e = fbl::launch_gated_grad_finish(f32, p, planes, gw.splits, s);
    } else {
        e = fbl::launch_gated_grad(f32, tile, p, s);
    }
    if (e == hipSuccess && dbias) {
        const int64_t groups = shared ? M : fbl::linear_grad_groups(f32, tile, p);
        e = fbl::launch_column_sums(f32, p.sums, (int)groups, 1, (int)(2 * F), dbias, nullptr, s);
    }
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

}  // extern "C"
