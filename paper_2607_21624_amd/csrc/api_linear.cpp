// api_linear.cpp -- the C ABI of linear layers with bias, activation and residual:
// validation and dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act.hpp"
#include "kernels.hpp"
#include "products.hpp"

using fbl::align256;
using fbl::few_splits;
using fbl::few_ws;
using fbl::forward_tile;
using fbl::kMaxWidth;
using fbl::overlap;
using fbl::RowsView;

namespace fbl {

// Workgroups that share the contraction of a few tokens' tiles.  A tile alone has too few of w's bytes on the
// way, and the longer its contraction the more that costs; sharing it costs a second launch and the planes
// (cold weights, us, alone and shared: bf16, 1 token 4096 x 4096 18.3 and 12.3, 8192 x 2048 31.4 and 12.1, 2048 x
// 8192 11.3 and 12.1, 1024 x 4096 6.8 and 8.9; 64 tokens 4096 x 4096 20.1 and 15.1, 128 tokens 22.7 and 25.0, but
// 8192 x 2048 33.6 and 25.4; fp32, 12 tokens 4096 x 4096 38 and 23, 1024 x 1024 11.6 and 7.7, 96 tokens 60 and 52).
// The data gradient, whose contraction is N, the same (dx, bf16, 1 token 2048 x 8192 25.1 and 11.9, 64 tokens 25.1 and
// 14.9; fp32, 1 token 57 and 19, 128 tokens 59 and 52, 200 tokens 92 and 89, but 1024 x 1024 9.4 and 12.1).
int few_splits(int f32, int64_t M, int64_t K, int64_t N) {
    if (M * N >= (int64_t)1 << 29) return 1;  // a plane's offsets
    return (f32 ? M <= 128 && K >= 1024 : M <= 64 ? K > 2048 : M <= 128 && K >= 8192) ? sum_splits(f32, 0, M, N, K, 0) : 1;
}

// The tile of a bf16 forward that is not shared.  Up to 32 tokens and 8192 columns that is 32 x 32 on four
// wavefronts, whose many workgroups have the most loads on the way; wider, the 32 x 128 of the products' own choice
// covers the CUs too and reads x less often (us, cold weights, 32 x 32 and own choice: 1 token 512 x 8192 4.3 and
// 5.2, 2048 x 8192 10.9 and 16.5, 2048 x 8200 12.7 and 16.9, 512 x 12288 6.0 and 5.7, 2048 x 12288 18.4 and 17.0,
// 2048 x 32768 29.9 and 22.7; 17 tokens 2048 x 8192 11.6 and 16.9, 2048 x 12288 19.8 and 17.5).
int forward_tile(int64_t M, int64_t K, int64_t N) {
    if (M <= 32 && N <= 8192 && fbl_proj_tuned_tile(FBL_PROJ_FWD, M, K, N) < 0) return 16;
    return proj_auto_tile(FBL_PROJ_FWD, M, K, N);
}

hipError_t launch_shares(int f32, int grad, int splits, const GemmArgs& p, float* planes, hipStream_t s) {
    SumArgs q{};
    static_cast<GemmArgs&>(q) = p;
    q.sum = planes, q.lds = p.N, q.sum_bytes = (uint32_t)((int64_t)p.M * p.N * 4);
    q.first = 1, q.splits = splits, q.share = (int)((((int64_t)p.K + splits - 1) / splits + 63) / 64 * 64);
    return f32 ? launch_sum_gemm_f32(grad, q, s) : launch_sum_gemm(0, grad, 0, q, s);
}

}  // namespace fbl

namespace {

template <int ACT>
hipError_t run_act(int f32, int grad, int tile, const fbl::LinearArgs& p, hipStream_t s) {
    return f32 ? fbl::launch_linear_gemm_f32<ACT>(grad, p, s) : fbl::launch_linear_gemm<ACT>(grad, tile, p, s);
}
hipError_t run_linear_gemm(int f32, int act, int grad, int tile, const fbl::LinearArgs& p, hipStream_t s) {
    switch (act) {
        case FBL_ACT_NONE: return run_act<fbl::kActNone>(f32, grad, tile, p, s);
        case FBL_ACT_RELU: return run_act<fbl::kActRelu>(f32, grad, tile, p, s);
        case FBL_ACT_GELU: return run_act<fbl::kActGelu>(f32, grad, tile, p, s);
        case FBL_ACT_GELU_TANH: return run_act<fbl::kActGeluTanh>(f32, grad, tile, p, s);
        default: return run_act<fbl::kActSilu>(f32, grad, tile, p, s);
    }
}

// Blocks of rows of the elementwise pass: enough workgroups for eight a CU, no more partial
// sums than 512 rows.
struct ActGrid {
    int64_t rows;
    int groups;
};
ActGrid act_grid(int f32, int64_t M, int64_t N) {
    const int64_t cols = f32 ? 256 : 512, ct = (N + cols - 1) / cols;
    const int64_t want = std::min<int64_t>(512, std::max<int64_t>(1, 2048 / ct));
    const int64_t rows = ((M + want - 1) / want + 3) / 4 * 4;
    return {rows, (int)((M + rows - 1) / rows)};
}

// A product of few rows whose contraction `splits` workgroups a tile share, their planes, and what follows it.
hipError_t run_shared(int f32, int act, int grad, int splits, const fbl::LinearArgs& p, float* planes, hipStream_t s) {
    const hipError_t e = fbl::launch_shares(f32, grad, splits, p, planes, s);
    return e == hipSuccess ? fbl::launch_linear_finish(f32, act, grad, p, planes, splits, s) : e;
}

// Workspace of the backward, a function of the shape (a caller may keep it while fbl_proj_tune's choices come and
// go): partial sums of the bias' gradient, dz, planes of dx, partial sums of dx (as many rows
// of them as any tile writes, linear_grad_groups, or one for each of a few tokens).
struct LinearWs {
    size_t dz, planes, sums, total;
    int64_t ldz;          // of dz: bf16 rows of whole 16-byte chunks, as every operand that the products stage
    int splits, wsplits;  // of dx and of dw: the planes are used by one after the other
};
LinearWs linear_ws(int f32, int64_t M, int64_t K, int64_t N) {
    LinearWs w;
    w.splits = few_splits(f32, M, N, K);
    w.dz = align256((size_t)act_grid(f32, M, N).groups * (size_t)N * 4);
    w.ldz = f32 ? N : (N + 7) / 8 * 8;
    w.planes = w.dz + align256((size_t)M * (size_t)w.ldz * (f32 ? 4 : 2));
    w.wsplits = fbl::weight_splits(f32, M, K, N, f32 ? 0 : fbl::weight_untuned_tile(M, K, N));
    w.sums = w.planes + align256(std::max(few_ws(w.splits, M, K), few_ws(w.wsplits, K, N)));
    w.total = w.sums + (size_t)(w.splits > 1 ? M : M / 32 + 4) * (size_t)K * 4;
    return w;
}

fbl_status linear_shape(int32_t dtype, uint32_t act, int64_t M, int64_t K, int64_t N) {
    if (!fbl::dtype_size(dtype)) return FBL_ERR_DTYPE;
    if (act > FBL_ACT_SILU) return FBL_ERR_ARG;
    if (!fbl::extent(M) || !fbl::extent(K) || !fbl::extent(N)) return FBL_ERR_SHAPE;
    if (M * N >= ((int64_t)1 << 31) / fbl::dtype_size(dtype)) return FBL_ERR_UNSUPPORTED;  // y, dy, dz
    if (K > kMaxWidth || N > kMaxWidth) return FBL_ERR_UNSUPPORTED;
    return FBL_OK;
}

}  // namespace

extern "C" {

fbl_status fbl_linear_fwd_workspace(int32_t dtype, int64_t M, int64_t K, int64_t N, size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    const fbl_status st = linear_shape(dtype, FBL_ACT_NONE, M, K, N);
    if (st == FBL_OK) *bytes = few_ws(few_splits(dtype == FBL_F32, M, K, N), M, N);
    return st;
}

fbl_status fbl_linear_fwd(int32_t dtype, uint32_t act, int64_t M, int64_t K, int64_t N, const void* x, int64_t ldx,
                          const void* w, int64_t ldw, const void* bias, const void* res, int64_t ldr, void* y,
                          int64_t ldy, void* z, int64_t ldz, int32_t tile, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = linear_shape(dtype, act, M, K, N);
    if (st != FBL_OK) return st;
    if (!x || !w || !y) return FBL_ERR_NULL;
    const int es = (int)fbl::dtype_size(dtype);
    const RowsView vx{x, M, K, ldx, es}, vw{w, K, N, ldw, es}, vb{bias, 1, N, (N + 7) / 8 * 8, es},
        vr{res, M, N, ldr, es}, vy{y, M, N, ldy, es}, vz{z, M, N, ldz, es};
    for (const RowsView* v : {&vx, &vw, &vb, &vr, &vy, &vz})
        if ((st = fbl::check_operand(*v)) != FBL_OK) return st;
    if (es == 2 && (K % 8 || N % 4)) return FBL_ERR_UNSUPPORTED;
    if (tile < FBL_GEMM_TILE_AUTO || tile >= fbl::kGemmTileCount || (es == 4 && tile != FBL_GEMM_TILE_AUTO))
        return FBL_ERR_ARG;
    for (const RowsView* out : {&vy, &vz})
        for (const RowsView* in : {&vx, &vw, &vb, &vr})
            if (overlap(*out, *in)) return FBL_ERR_ARG;
    if (overlap(vy, vz)) return FBL_ERR_ARG;
    // with a workspace for the shares of it
    int splits = tile == FBL_GEMM_TILE_AUTO && ws ? few_splits(es == 4, M, K, N) : 1;
    if (splits > 1) {
        const size_t need = few_ws(splits, M, N);
        if (ws_bytes < need) return FBL_ERR_WORKSPACE;
        const RowsView vws{ws, 1, (int64_t)need, (int64_t)need, 1};
        if (vws.begin() % 16) return FBL_ERR_ALIGN;
        for (const RowsView* v : {&vx, &vw, &vb, &vr, &vy, &vz})
            if (overlap(vws, *v)) return FBL_ERR_ARG;
    }
    fbl::LinearArgs p{};
    fbl::product(p, FBL_PROJ_FWD, vx, vw, vy, M, K, N);
    p.bias = bias, p.res = res, p.z = z, p.ldr = ldr, p.ldz = ldz;
    p.res_bytes = res ? fbl::load_span(vr) : 0;
    p.z_bytes = z ? (uint32_t)vz.bytes() : 0;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (splits > 1) {
        const hipError_t e = run_shared(es == 4, (int)act, 0, splits, p, static_cast<float*>(ws), s);
        return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
    }
    if (es == 2 && tile == FBL_GEMM_TILE_AUTO) tile = forward_tile(M, K, N);
    const hipError_t e = run_linear_gemm(es == 4, (int)act, 0, tile, p, s);
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

fbl_status fbl_linear_bwd_workspace(int32_t dtype, int64_t M, int64_t K, int64_t N, size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    const fbl_status st = linear_shape(dtype, FBL_ACT_NONE, M, K, N);
    if (st == FBL_OK) *bytes = linear_ws(dtype == FBL_F32, M, K, N).total;
    return st;
}

fbl_status fbl_linear_bwd(int32_t dtype, uint32_t act, int64_t M, int64_t K, int64_t N, const void* dy, int64_t lddy,
                          const void* x, int64_t ldx, const void* w, int64_t ldw, const void* z, int64_t ldz,
                          uint32_t xact, const void* xz, int64_t ldxz, void* dx, int64_t lddx, void* dxbias,
                          void* dw, int64_t lddw, void* dbias, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = linear_shape(dtype, act, M, K, N);
    if (st != FBL_OK) return st;
    if (xact > FBL_ACT_SILU) return FBL_ERR_ARG;
    if (!dy || (dw && !x) || (dx && !w) || (dxbias && !dx)) return FBL_ERR_NULL;
    const bool has_act = act != FBL_ACT_NONE, has_xact = dx && xact != FBL_ACT_NONE;
    if ((has_act && !z) || (has_xact && !xz)) return FBL_ERR_NULL;
    const int es = (int)fbl::dtype_size(dtype), f32 = es == 4;
    const RowsView vdy{dy, M, N, lddy, es}, vx{dw ? x : nullptr, M, K, ldx, es}, vw{dx ? w : nullptr, K, N, ldw, es},
        vz{has_act ? z : nullptr, M, N, ldz, es}, vxz{has_xact ? xz : nullptr, M, K, ldxz, es}, vdx{dx, M, K, lddx, es},
        vdw{dw, K, N, lddw, es};
    const RowsView vdb{dbias, 1, N, N, es}, vdxb{dxbias, 1, K, K, es};
    for (const RowsView* v : {&vdy, &vx, &vw, &vz, &vxz, &vdx, &vdw})
        if ((st = fbl::check_operand(*v)) != FBL_OK) return st;
    if (!vdb.natural() || !vdxb.natural()) return FBL_ERR_ALIGN;
    if (es == 2 && ((dx && (N % 8 || K % 4)) || (dw && N % 4))) return FBL_ERR_UNSUPPORTED;
    // what is needed of the workspace: partial sums for the bias, dz where an activation makes it
    const LinearWs lw = linear_ws(f32, M, K, N);
    const bool pass = has_act ? (dx || dw || dbias) : dbias != nullptr, shared = dx && lw.splits > 1 && ws,
               wshared = dw && lw.wsplits > 1 && ws;
    const size_t need = pass || shared || wshared || dxbias ? lw.total : 0;
    if (need && (!ws || ws_bytes < need)) return FBL_ERR_WORKSPACE;
    const RowsView vws{need ? ws : nullptr, 1, (int64_t)need, (int64_t)need + 1, 1};
    if (vws.begin() % 16) return FBL_ERR_ALIGN;
    const RowsView* outs[] = {&vdx, &vdw, &vdb, &vdxb, &vws};
    for (int i = 0; i < 5; ++i) {
        for (const RowsView* in : {&vdy, &vx, &vw, &vz, &vxz})
            if (overlap(*outs[i], *in)) return FBL_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i], *outs[j])) return FBL_ERR_ARG;
    }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    RowsView g = vdy;  // the gradient of the pre-activation
    if (pass) {
        const ActGrid ag = act_grid(f32, M, N);
        fbl::LinearActArgs a{};
        a.dy = dy, a.z = z, a.lddy = lddy, a.ldz = ldz, a.M = M, a.N = (int)N, a.rows = ag.rows, a.groups = ag.groups;
        a.part = dbias ? static_cast<float*>(ws) : nullptr;
        if (has_act) {
            // (its span is at most dy's, whose rows are as long at least)
            g = RowsView{static_cast<char*>(ws) + lw.dz, M, N, lw.ldz, es};
            a.dz = const_cast<void*>(g.p), a.lddz = g.ld;
        }
        e = fbl::launch_linear_act_bwd(f32, (int)act, a, s);
        if (e == hipSuccess && dbias) e = fbl::launch_column_sums(f32, a.part, a.groups, 1, (int)N, dbias, nullptr, s);
    }
    if (e == hipSuccess && dx) {
        fbl::LinearArgs p{};
        fbl::product(p, FBL_PROJ_BWD_DATA, g, vw, vdx, M, K, N);
        const int tile = f32 ? 0 : fbl::proj_auto_tile(FBL_PROJ_BWD_DATA, M, K, N);
        if (has_xact) p.z = const_cast<void*>(xz), p.ldz = ldxz, p.z_bytes = fbl::load_span(vxz);
        if (dxbias) p.sums = reinterpret_cast<float*>(static_cast<char*>(ws) + lw.sums);
        const int a = has_xact ? (int)xact : FBL_ACT_NONE;
        e = shared ? run_shared(f32, a, 1, lw.splits, p, reinterpret_cast<float*>(static_cast<char*>(ws) + lw.planes), s)
            : f32 && !has_xact && !dxbias ? fbl::launch_proj_gemm_f32(0, 1, p, s)
                   : run_linear_gemm(f32, a, 1, tile, p, s);
        if (e == hipSuccess && dxbias) {
            const int64_t groups = shared ? M : fbl::linear_grad_groups(f32, tile, p);
            e = fbl::launch_column_sums(f32, p.sums, (int)groups, 1, (int)K, dxbias, nullptr, s);
        }
    }
    if (e == hipSuccess && wshared) {
        fbl::SumArgs q{};
        fbl::product(q, FBL_PROJ_BWD_WEIGHT, vx, g, vdw, M, K, N);
        q.sum = reinterpret_cast<float*>(static_cast<char*>(ws) + lw.planes), q.lds = N;
        q.sum_bytes = (uint32_t)(K * N * 4);
        q.first = 1, q.splits = lw.wsplits, q.share = (int)(((M + q.splits - 1) / q.splits + 63) / 64 * 64);
        e = fbl::launch_weight_shares(f32, q, s);
        if (e == hipSuccess) e = fbl::launch_sum_planes(f32, q.sum, q.splits, K, N, nullptr, dw, lddw, s);
    } else if (e == hipSuccess && dw) {
        fbl::LinearArgs p{};
        fbl::product(p, FBL_PROJ_BWD_WEIGHT, vx, g, vdw, M, K, N);
        e = f32 ? fbl::launch_proj_gemm_f32(1, 0, p, s) : fbl::launch_weight_gemm(fbl::weight_tile(M, K, N), p, s);
    }
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

}  // extern "C"
