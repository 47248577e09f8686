// api_head.cpp -- the C ABI of the softmax losses of a linear head: validation, the
// pieces of the vocabulary, dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cdna4.hpp"
#include "kernels.hpp"
#include "products.hpp"

using fbl::overlap;
using fbl::RowsView;

namespace {

constexpr int64_t kSpan = (int64_t)1 << 31;  // of an operand
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Shape {
    int32_t dtype;
    uint32_t order;
    int64_t M, K, V, top;
    int64_t es() const { return fbl::dtype_size(dtype); }
    bool f32() const { return dtype == FBL_F32; }
    bool table() const { return order == FBL_HEAD_VK; }
};

fbl_status check_shape(const Shape& s) {
    if (!s.es()) return FBL_ERR_DTYPE;
    if (s.order > FBL_HEAD_VK) return FBL_ERR_ARG;
    if (!fbl::extent(s.M) || !fbl::extent(s.K) || !fbl::extent(s.V) || s.top <= 0) return FBL_ERR_SHAPE;
    if (s.top > fbl::kHeadMaxTop) return FBL_ERR_UNSUPPORTED;
    if (!s.f32() && (s.K % 8 || (!s.table() && s.V % 8))) return FBL_ERR_UNSUPPORTED;
    // x, dx and the fp32 sums of dx; a piece of dz of 64 columns at least; target lists
    if (s.M * s.K >= kSpan / 4 || s.M * 64 * s.es() >= kSpan || s.M * s.top >= kSpan / 4) return FBL_ERR_UNSUPPORTED;
    return FBL_OK;
}

// The weight as it is stored, or a piece of the vocabulary of it.
RowsView weight_view(const Shape& s, const void* w, int64_t ld, int64_t first, int64_t width) {
    if (!w) return RowsView{nullptr, 1, 1, 1, s.es()};
    const char* p = static_cast<const char*>(w) + first * (s.table() ? ld : 1) * s.es();
    return s.table() ? RowsView{p, width, s.K, ld, s.es()} : RowsView{p, s.K, width, ld, s.es()};
}
fbl_status check_weight(const Shape& s, const void* w, int64_t ld) {
    const RowsView v = weight_view(s, w, ld, 0, s.V);
    if (!v.p) return FBL_OK;
    if (v.ld < v.width) return FBL_ERR_LAYOUT;
    // a table may be larger than an operand's span: it is read by pieces of whole rows
    if (!v.addressable() || ld > fbl::kMaxExtent || (s.table() ? 256 * ld * s.es() : v.bytes()) >= kSpan) return FBL_ERR_UNSUPPORTED;
    return s.es() == 2 ? (v.aligned16() ? FBL_OK : FBL_ERR_ALIGN) : (v.natural() ? FBL_OK : FBL_ERR_ALIGN);
}

// Vocabulary entries of a forward launch: all of them, or as many rows of a large table as a span holds, or columns
// as keep a launch's threads below 2^32 (at most 2^34 logits; tiles are of 16 a thread at least).
int64_t forward_piece(const Shape& s, int64_t ldw) {
    int64_t most = std::max<int64_t>(256, ((int64_t)1 << 34) / s.M);
    if (s.table()) most = std::min(most, ((kSpan - 1) / s.es() - s.K) / ldw + 1);
    return most >= s.V ? s.V : most / 256 * 256;
}

// Vocabulary entries of a piece of the backward.  dz [M][piece] goes through memory twice and dX's fp32
// sums once a piece, so pieces are large, up to 128 MiB of dz; of those, the width whose tiles
// fill the CUs' rounds best.  (4096 tokens, K 1024, V 50257: 3 pieces of 16384 and one of 1105 make 13 rounds of dz
// and 4 of dW, 4 pieces of 12800 make 15 and 4.)  Many tokens still get 4096 entries, for more memory: with 128 MiB
// of dz in half or a quarter of them the sums' traffic costs more than that is worth (backward, ms, with 4096 and with
// 128 MiB: 32768 tokens, K 2048, V 128256 51.0 and 55.0; K 4096, V 32000 23.2 and 26.8; K 1024, V 50257 11.3 and
// 13.6; 65536 tokens, K 1024 22.7 and 34.9; fp32 16384 tokens, K 512, V 50257 20.7 and 22.4).
int64_t backward_piece(const Shape& s, int64_t ldw) {
    int64_t most = std::max<int64_t>(4096, ((int64_t)128 << 20) / (s.M * s.es()));
    most = std::min(most, std::max<int64_t>(64, (kSpan - 1) / (s.M * s.es()) - 64));
    if (s.table()) most = std::min(most, ((kSpan - 1) / s.es() - s.K) / ldw + 1);
    if (most >= s.V) return s.V;
    if (most < 512) return most / 64 * 64;
    // cost in products of a CU: its rounds of dz tiles (256 x 256: fp32's smaller ones waste less) and of dW tiles,
    // dX's sums read and written (8 bytes at 16 a CU and cycle, 1000 products meanwhile), and the launches
    const auto tiles = [](int64_t n) { return (double)((n + 255) / 256); };
    const auto cost = [&](int64_t width) {
        const double dz = std::ceil(tiles(s.M) * tiles(width) / 256) * 65536.0 * (double)s.K;
        const double dw = std::ceil(tiles(s.K) * tiles(width) / 256) * 65536.0 * (double)s.M;
        return dz + dw + (double)s.M * (double)s.K * 4 + 2e7;
    };
    const int64_t step = std::max<int64_t>(1, most / 256 / 64) * 256;
    int64_t best = 0;
    double best_cost = 0;
    for (int64_t width = most / 256 * 256; width >= std::max<int64_t>(256, most / 4); width -= step) {
        const int64_t whole = s.V / width, rest = s.V % width;
        const double c = (double)whole * cost(width) + (rest ? cost(rest) : 0);
        if (!best || c < best_cost) best = width, best_cost = c;
    }
    return best;
}
int64_t padded64(int64_t n) { return (n + 63) / 64 * 64; }

struct HeadWs {
    size_t index, target, part, entropy, counted, fwd;  // forward
    size_t weight, row, scale, dz, sum, bwd;            // backward
    int splits;                                         // of dX's contraction
};
// Tile of dX over a contraction of kc entries: chosen by `choose`, for a launch or (untuned) for the workspace's layout.
int dx_tile(int (*choose)(uint32_t, int64_t, int64_t, int64_t), const Shape& s, int64_t kc) {
    return s.table() ? choose(FBL_PROJ_FWD, s.M, kc, s.K) : choose(FBL_PROJ_BWD_DATA, s.M, s.K, kc);
}

HeadWs head_ws(const Shape& s, int64_t ldw) {
    HeadWs w{};
    const size_t list = align256((size_t)s.M * (size_t)s.top * 4), row = align256((size_t)s.M * 4);
    const int64_t tw = fbl::head_tile_width(s.f32(), fbl::head_tile(s.f32(), s.table(), s.M, s.V, s.K)), fp = forward_piece(s, ldw);
    const int64_t parts = (s.V + tw - 1) / tw + (s.V + fp - 1) / fp;
    w.index = 0, w.target = list, w.part = w.target + list;
    w.entropy = w.part + align256((size_t)parts * (size_t)s.M * 8);
    w.counted = w.entropy + row, w.fwd = w.counted + row;
    const int64_t bp = backward_piece(s, ldw);
    w.weight = list, w.row = w.weight + list;
    w.scale = w.row + align256((size_t)s.M * 8);
    w.dz = w.scale + 256;
    w.sum = w.dz + align256((size_t)s.M * (size_t)padded64(bp) * (size_t)s.es());
    const size_t plane = (size_t)s.M * (size_t)s.K * 4;
    w.splits = fbl::sum_splits(s.f32(), !s.table(), s.M, s.K, bp, s.f32() ? 0 : dx_tile(fbl::proj_untuned_tile, s, bp));
    w.bwd = w.sum + (w.splits > 1 ? align256((size_t)w.splits * plane) : bp < s.V && !s.f32() ? align256(plane) : 0);
    return w;
}

fbl_status check_overlaps(const RowsView* const* outs, int no, const RowsView* const* ins, int ni) {
    for (int i = 0; i < no; ++i) {
        for (int j = 0; j < ni; ++j)
            if (overlap(*outs[i], *ins[j])) return FBL_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i], *outs[j])) return FBL_ERR_ARG;
    }
    return FBL_OK;
}

fbl::HeadArgs piece_args(const Shape& s, const RowsView& vx, const void* w, int64_t ldw, int64_t first, int64_t width) {
    fbl::HeadArgs p{};
    const RowsView vw = weight_view(s, w, ldw, first, width);
    p.a = vx.p, p.lda = vx.ld, p.a_bytes = fbl::load_span(vx);
    p.b = vw.p, p.ldb = vw.ld, p.b_bytes = fbl::load_span(vw);
    p.M = p.tokens = (int)s.M, p.N = (int)width, p.K = (int)s.K;
    p.first = (int)first, p.width = (int)width, p.top = (int)s.top;
    return p;
}

// What both losses' calls share.
struct Targets {
    const int64_t* labels;
    int64_t ignore;
    const int64_t* given;
    int64_t ldi;
    const void* logits;
    int32_t logits_dtype;
    int64_t ldl;
    float T;
    float* prob;
};

fbl::HeadRowArgs row_args(const Shape& s, const Targets& t) {
    fbl::HeadRowArgs a{};
    a.M = s.M, a.V = (int)s.V, a.top = (int)s.top;
    a.labels = t.labels, a.ignore = t.ignore, a.given = t.given, a.ldi = t.ldi;
    a.logits = t.logits, a.ldl = t.ldl, a.logits_f32 = t.logits_dtype == FBL_F32, a.T = t.T, a.prob = t.prob;
    return a;
}

fbl_status check_targets(const Shape& s, const Targets& t, RowsView* list, RowsView* logits, RowsView* prob) {
    *list = *logits = *prob = RowsView{nullptr, 1, 1, 1, 4};
    if (t.labels) {
        *list = RowsView{t.labels, 1, s.M, s.M, 8};
    } else {
        if (!std::isfinite(t.T) || t.T <= 0) return FBL_ERR_ARG;
        *list = RowsView{t.given, s.M, s.top, t.ldi, 8};
        *prob = RowsView{t.prob, 1, s.M * s.top, s.M * s.top, 4};
        if (t.logits) {
            if (!fbl::dtype_size(t.logits_dtype)) return FBL_ERR_DTYPE;
            *logits = RowsView{t.logits, s.M, s.top, t.ldl, fbl::dtype_size(t.logits_dtype)};
        }
    }
    for (const RowsView* v : {list, logits, prob}) {
        if (!v->p) continue;
        if (v->ld < v->width) return FBL_ERR_LAYOUT;
        if (v->ld > fbl::kMaxExtent * 4 || !v->addressable()) return FBL_ERR_UNSUPPORTED;
        if (!v->natural()) return FBL_ERR_ALIGN;
    }
    return FBL_OK;
}

fbl_status head_fwd(const Shape& s, const void* x, int64_t ldx, const void* w, int64_t ldw, const Targets& t, float* loss,
                    float* lse, float* total, float* mean, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = check_shape(s);
    if (st != FBL_OK) return st;
    if (!x || !w || !(t.labels || (t.given && t.logits && t.prob)) || !loss || !lse || (mean && !total)) return FBL_ERR_NULL;
    const RowsView vx{x, s.M, s.K, ldx, s.es()}, vw = weight_view(s, w, ldw, 0, s.V);
    if ((st = fbl::check_operand(vx)) != FBL_OK) return st;
    if ((st = check_weight(s, w, ldw)) != FBL_OK) return st;
    RowsView list, logits, prob;
    if ((st = check_targets(s, t, &list, &logits, &prob)) != FBL_OK) return st;
    const RowsView vl{loss, 1, s.M, s.M, 4}, ve{lse, 1, s.M, s.M, 4}, vt{total, 1, 2, 2, 4}, vm{mean, 1, 1, 1, 4};
    for (const RowsView* v : {&vl, &ve, &vt, &vm})
        if (!v->natural()) return FBL_ERR_ALIGN;
    const HeadWs lay = head_ws(s, ldw);
    if (!ws || ws_bytes < lay.fwd) return FBL_ERR_WORKSPACE;
    const RowsView vws{ws, 1, (int64_t)lay.fwd, (int64_t)lay.fwd, 1};
    if (vws.begin() % 16) return FBL_ERR_ALIGN;
    const RowsView* outs[] = {&vl, &ve, &vt, &vm, &prob, &vws};
    const RowsView* ins[] = {&vx, &vw, &list, &logits};
    if ((st = check_overlaps(outs, 6, ins, 4)) != FBL_OK) return st;

    char* const base = static_cast<char*>(ws);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    fbl::HeadRowArgs a = row_args(s, t);
    a.index = reinterpret_cast<int*>(base + lay.index);
    a.entropy = reinterpret_cast<float*>(base + lay.entropy), a.counted = reinterpret_cast<float*>(base + lay.counted);
    hipError_t e = fbl::launch_head_targets(a, hs);
    const int64_t piece = forward_piece(s, ldw);
    const int shape = fbl::head_tile(s.f32(), s.table(), s.M, s.V, s.K);
    const int64_t tw = fbl::head_tile_width(s.f32(), shape);
    int tiles = 0;
    for (int64_t v0 = 0; v0 < s.V && e == hipSuccess; v0 += piece) {
        const int64_t width = std::min(piece, s.V - v0);
        fbl::HeadArgs p = piece_args(s, vx, w, ldw, v0, width);
        p.unit = fbl::kLog2e / t.T;
        p.index = a.index;
        p.part = reinterpret_cast<float2*>(base + lay.part), p.target = reinterpret_cast<float*>(base + lay.target);
        p.tile0 = tiles;
        p.shape = shape;
        tiles += (int)((width + tw - 1) / tw);
        e = fbl::launch_head_fwd(s.f32(), s.table(), p, hs);
    }
    if (e != hipSuccess) return FBL_ERR_HIP;
    a.part = reinterpret_cast<const float2*>(base + lay.part), a.target = reinterpret_cast<const float*>(base + lay.target);
    a.parts = tiles, a.loss = loss, a.lse = lse, a.sums = total, a.mean = mean;
    return fbl::launch_head_join(a, hs) == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

fbl_status head_bwd(const Shape& s, const float* dloss, int64_t dloss_stride, const float* total, const void* x, int64_t ldx,
                    const void* w, int64_t ldw, const Targets& t, const float* lse, void* dx, int64_t lddx, void* dw,
                    int64_t lddw, void* ws, size_t ws_bytes, void* stream) {
    fbl_status st = check_shape(s);
    if (st != FBL_OK) return st;
    if (!dloss || !x || !w || !lse || !(t.labels || (t.given && t.prob))) return FBL_ERR_NULL;
    if (dloss_stride < 0 || dloss_stride > fbl::kMaxExtent) return FBL_ERR_LAYOUT;
    const RowsView vx{x, s.M, s.K, ldx, s.es()}, vw = weight_view(s, w, ldw, 0, s.V), vdx{dx, s.M, s.K, lddx, s.es()},
        vdw = weight_view(s, dw, lddw, 0, s.V);
    for (const RowsView* v : {&vx, &vdx})
        if ((st = fbl::check_operand(*v)) != FBL_OK) return st;
    if ((st = check_weight(s, w, ldw)) != FBL_OK || (st = check_weight(s, dw, lddw)) != FBL_OK) return st;
    RowsView list, logits, prob;
    if ((st = check_targets(s, t, &list, &logits, &prob)) != FBL_OK) return st;
    const RowsView vg{dloss, 1, (s.M - 1) * dloss_stride + 1, s.M * (dloss_stride + 1), 4}, vt{total, 1, 2, 2, 4},
        ve{lse, 1, s.M, s.M, 4};
    for (const RowsView* v : {&vg, &vt, &ve})
        if (!v->natural()) return FBL_ERR_ALIGN;
    if (dw && s.table() && backward_piece(s, ldw) * lddw * s.es() >= kSpan) return FBL_ERR_UNSUPPORTED;
    if (!dx && !dw) return FBL_OK;
    const HeadWs lay = head_ws(s, ldw);
    if (!ws || ws_bytes < lay.bwd) return FBL_ERR_WORKSPACE;
    const RowsView vws{ws, 1, (int64_t)lay.bwd, (int64_t)lay.bwd, 1};
    if (vws.begin() % 16) return FBL_ERR_ALIGN;
    const RowsView* outs[] = {&vdx, &vdw, &vws};
    const RowsView* ins[] = {&vg, &vt, &vx, &vw, &list, &prob, &ve};
    if ((st = check_overlaps(outs, 3, ins, 7)) != FBL_OK) return st;

    char* const base = static_cast<char*>(ws);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    fbl::HeadRowArgs a = row_args(s, t);
    a.index = reinterpret_cast<int*>(base + lay.index), a.weight = reinterpret_cast<float*>(base + lay.weight);
    a.row = reinterpret_cast<float2*>(base + lay.row);
    // bf16: one factor for all rows stays out of dz, rows' own are in it
    float* const scale = s.f32() ? nullptr : reinterpret_cast<float*>(base + lay.scale);
    a.scale = scale;
    a.dloss = dloss, a.dloss_stride = dloss_stride, a.total = total, a.lse_in = lse;
    hipError_t e = fbl::launch_head_grad_rows(a, hs);
    const int64_t piece = backward_piece(s, ldw);
    for (int64_t v0 = 0; v0 < s.V && e == hipSuccess; v0 += piece) {
        const int64_t width = std::min(piece, s.V - v0), ldz = padded64(width);
        const bool first = v0 == 0, last = v0 + width == s.V;
        const RowsView vz{base + lay.dz, s.M, ldz, ldz, s.es()};
        fbl::HeadArgs p = piece_args(s, vx, w, ldw, v0, width);
        p.N = (int)ldz;  // dz's padding is written too (zeros)
        p.unit = fbl::kLog2e / t.T;
        p.index = a.index, p.weight = t.labels ? nullptr : a.weight, p.row = a.row;
        p.shape = fbl::head_tile(s.f32(), s.table(), s.M, ldz, s.K);
        p.dz = base + lay.dz, p.ldz = ldz, p.dz_bytes = (uint32_t)vz.bytes();
        e = fbl::launch_head_grad(s.f32(), s.table(), p, hs);
        const RowsView wp = weight_view(s, w, ldw, v0, width);
        if (e == hipSuccess && dx) {
            // the table's rows past its last read as zeros, as dz's padding does: a whole contraction for bf16
            const int64_t kc = s.table() && !s.f32() ? ldz : width;
            const uint32_t op = s.table() ? FBL_PROJ_FWD : FBL_PROJ_BWD_DATA;
            const RowsView az{vz.p, s.M, kc, ldz, s.es()};
            fbl::SumArgs q{};
            if (s.table()) fbl::product(q, op, az, wp, vdx, s.M, kc, s.K);
            else fbl::product(q, op, az, wp, vdx, s.M, s.K, kc);
            q.first = first, q.last = last, q.scale = scale, q.splits = lay.splits;
            q.share = (int)(((kc + lay.splits - 1) / lay.splits + 63) / 64 * 64);
            if (lay.splits > 1 || (!s.f32() && !(first && last))) {
                q.sum = reinterpret_cast<float*>(base + lay.sum), q.lds = s.K;
                q.sum_bytes = (uint32_t)(s.M * s.K * 4);
            }
            const int tile = s.f32() ? 0 : dx_tile(fbl::proj_auto_tile, s, kc);
            e = s.f32() ? fbl::launch_sum_gemm_f32(!s.table(), q, hs) : fbl::launch_sum_gemm(0, !s.table(), tile, q, hs);
            if (e == hipSuccess && last && lay.splits > 1)
                e = fbl::launch_sum_planes(s.f32(), q.sum, lay.splits, s.M, s.K, scale, dx, lddx, hs);
        }
        if (e == hipSuccess && dw) {
            const RowsView dz{vz.p, s.M, width, ldz, s.es()}, dwp = weight_view(s, dw, lddw, v0, width);
            fbl::SumArgs q{};
            const int64_t rows = s.table() ? width : s.K, cols = s.table() ? s.K : width;
            fbl::product(q, FBL_PROJ_BWD_WEIGHT, s.table() ? dz : vx, s.table() ? vx : dz, dwp, s.M, rows, cols);
            q.scale = scale, q.first = q.last = q.splits = 1;
            e = s.f32() ? fbl::launch_proj_gemm_f32(1, 0, q, hs)
                        : fbl::launch_sum_gemm(1, 0, fbl::weight_tile(s.M, rows, cols), q, hs);
        }
    }
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

}  // namespace

extern "C" {

fbl_status fbl_linear_loss_workspace(int32_t dtype, uint32_t order, int64_t M, int64_t K, int64_t V, int64_t top, int64_t ldw,
                                     size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    const Shape s{dtype, order, M, K, V, top};
    fbl_status st = check_shape(s);
    if (st != FBL_OK) return st;
    if ((st = check_weight(s, reinterpret_cast<const void*>(uintptr_t(256)), ldw)) != FBL_OK) return st;
    const HeadWs w = head_ws(s, ldw);
    *bytes = std::max(w.fwd, w.bwd);
    return FBL_OK;
}

fbl_status fbl_linear_ce_fwd(int32_t dtype, uint32_t order, int64_t M, int64_t K, int64_t V, const void* x, int64_t ldx,
                             const void* w, int64_t ldw, const int64_t* labels, int64_t ignore, float* loss, float* lse,
                             float* total, float* mean, void* ws, size_t ws_bytes, void* stream) {
    const Targets t{labels, ignore, nullptr, 0, nullptr, 0, 0, 1.f, nullptr};
    return head_fwd(Shape{dtype, order, M, K, V, 1}, x, ldx, w, ldw, t, loss, lse, total, mean, ws, ws_bytes, stream);
}

fbl_status fbl_linear_ce_bwd(int32_t dtype, uint32_t order, int64_t M, int64_t K, int64_t V, const float* dloss,
                             int64_t dloss_stride, const float* total, const void* x, int64_t ldx, const void* w,
                             int64_t ldw, const int64_t* labels, int64_t ignore, const float* lse, void* dx, int64_t lddx,
                             void* dw, int64_t lddw, void* ws, size_t ws_bytes, void* stream) {
    const Targets t{labels, ignore, nullptr, 0, nullptr, 0, 0, 1.f, nullptr};
    return head_bwd(Shape{dtype, order, M, K, V, 1}, dloss, dloss_stride, total, x, ldx, w, ldw, t, lse, dx, lddx, dw, lddw,
                    ws, ws_bytes, stream);
}

fbl_status fbl_linear_kd_fwd(int32_t dtype, uint32_t order, int64_t M, int64_t K, int64_t V, int64_t top, const void* x,
                             int64_t ldx, const void* w, int64_t ldw, const int64_t* index, int64_t ldi,
                             int32_t logits_dtype, const void* logits, int64_t ldl, float temperature, float* prob,
                             float* loss, float* lse, float* total, float* mean, void* ws, size_t ws_bytes, void* stream) {
    const Targets t{nullptr, 0, index, ldi, logits, logits_dtype, ldl, temperature, prob};
    return head_fwd(Shape{dtype, order, M, K, V, top}, x, ldx, w, ldw, t, loss, lse, total, mean, ws, ws_bytes, stream);
}

fbl_status fbl_linear_kd_bwd(int32_t dtype, uint32_t order, int64_t M, int64_t K, int64_t V, int64_t top, const float* dloss,
                             int64_t dloss_stride, const float* total, const void* x, int64_t ldx, const void* w,
                             int64_t ldw, const int64_t* index, int64_t ldi, float temperature, const float* prob,
                             const float* lse, void* dx, int64_t lddx, void* dw, int64_t lddw, void* ws, size_t ws_bytes,
                             void* stream) {
    const Targets t{nullptr, 0, index, ldi, nullptr, 0, 0, temperature, const_cast<float*>(prob)};
    return head_bwd(Shape{dtype, order, M, K, V, top}, dloss, dloss_stride, total, x, ldx, w, ldw, t, lse, dx, lddx, dw, lddw,
                    ws, ws_bytes, stream);
}

}  // extern "C"
