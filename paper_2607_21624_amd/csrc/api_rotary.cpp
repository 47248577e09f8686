// api_rotary.cpp -- the C ABI of the norms of queries and keys for each head and their
// rotation by position: validation and dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kernels.hpp"
#include "layout_check.hpp"

using fbl::aligned16;
using fbl::check_layout;
using fbl::overlaps;
using fbl::same_extents;
using fbl::span_bytes;
using fbl::tokmap;
using fbl::views_overlap;

namespace {

// How the heads of all tokens are dealt to wavefronts, four a workgroup.  Workgroups walk the items: with sums two a CU of the
// three that fit are enough, and leave fewer rows of partial sums (us backward, 512 / 768 / 1536 workgroups: 4096 tokens of 32 + 32 heads
// of 128 41.5 / 42.1 / 45.7, of 32 + 8 heads of 64 19.6 / 20.0 / 23.5, 16384 of 32 + 8 heads of 128 101.4 / 103.7 / 105.7); without,
// more than fit cost nothing (1280, 2560 and 5120 the same).
void plan(fbl::RotaryArgs& p, int f32, int64_t D, bool sums) {
    const int rows = fbl::rotary_rows(f32, (int)D), H = p.Hq + p.Hkv;
    const int64_t tokens = (int64_t)p.B * p.S;
    p.heads = rows;
    while (p.heads > 1 && p.heads / 2 >= H) p.heads /= 2;
    const int64_t per_group = rows / p.heads;
    p.groups = (tokens + per_group - 1) / per_group;
    const int steps = (H + p.heads - 1) / p.heads;
    // few tokens: their heads go to wavefronts of their own, up to two a SIMD (1024 to 8192 of them: within 3%, but 3333 tokens of
    // 12 + 4 heads of 128 backward 21.1, and 16.6 from 2048 on)
    const int64_t parts = std::min<int64_t>(steps, std::max<int64_t>(1, 2048 / p.groups));
    p.per = (int)((steps + parts - 1) / parts);
    p.parts = (steps + p.per - 1) / p.per;
    const int64_t wgs = (p.groups * p.parts + 3) / 4;
    p.workgroups = (int)std::min<int64_t>(wgs, sums ? 512 : 2560);
}

// Extents and layouts of queries and (where there) keys.
fbl_status check_heads(const fbl_layout* lq, const fbl_layout* lk) {
    fbl_status st = check_layout(lq);
    if (st != FBL_OK) return st;
    if (lk) {
        if ((st = check_layout(lk)) != FBL_OK) return st;
        if (lq->dtype != lk->dtype) return FBL_ERR_DTYPE;
        if (lq->B != lk->B || lq->S != lk->S || lq->D != lk->D) return FBL_ERR_SHAPE;
    }
    if (lq->D != 32 && lq->D != 64 && lq->D != 128) return FBL_ERR_UNSUPPORTED;
    if (lq->B * lq->S > INT32_MAX) return FBL_ERR_UNSUPPORTED;
    return FBL_OK;
}

fbl_status check_tensor(const fbl_layout* l, const void* p, const fbl_layout* like) {
    if (!l || !p) return FBL_ERR_NULL;
    const fbl_status st = check_layout(l);
    if (st != FBL_OK) return st;
    if (!same_extents(l, like)) return l->dtype != like->dtype ? FBL_ERR_DTYPE : FBL_ERR_SHAPE;
    return aligned16(p) ? FBL_OK : FBL_ERR_ALIGN;
}

fbl_status set_rotation(fbl::RotaryArgs& p, const fbl_rotary* rot, const fbl_layout* l) {
    p.num_axes = 1;
    if (!rot) return FBL_OK;
    if (!rot->turns) return FBL_ERR_NULL;
    if (rot->reserved || (rot->neighbours & ~1)) return FBL_ERR_ARG;
    if (rot->dims <= 0 || rot->dims > l->D) return FBL_ERR_SHAPE;
    if (rot->dims % 16) return FBL_ERR_UNSUPPORTED;
    if (rot->num_axes < 1 || rot->num_axes > FBL_ROTARY_MAX_AXES) return FBL_ERR_ARG;
    if (rot->num_axes > 1 && !rot->positions) return FBL_ERR_NULL;
    const int64_t most = (int64_t)1 << 56;  // of a stride times its extent: no address of a position wraps
    if (rot->stride_axis < 0 || rot->stride_batch < 0 || rot->stride_token < 0 || rot->stride_axis > most / rot->num_axes ||
        rot->stride_batch > most / l->B || rot->stride_token > most / l->S)
        return FBL_ERR_LAYOUT;
    if (reinterpret_cast<uintptr_t>(rot->turns) % 8 || reinterpret_cast<uintptr_t>(rot->positions) % 8) return FBL_ERR_ALIGN;
    for (int i = 0; i < rot->dims / 2; ++i) {
        if (rot->num_axes == 1) break;
        if (rot->axes[i] >= rot->num_axes) return FBL_ERR_ARG;
        p.axes[i / 32] |= (uint64_t)rot->axes[i] << i % 32 * 2;
    }
    p.dims = rot->dims, p.num_axes = rot->num_axes, p.turns = rot->turns, p.pos = rot->positions;
    p.pos_axis = rot->stride_axis, p.pos_batch = rot->stride_batch, p.pos_token = rot->stride_token;
    return FBL_OK;
}

fbl_status set_norm(fbl::RotaryArgs& p, const fbl_head_norm* norm, int64_t es) {
    if (!norm) return FBL_OK;
    if (!std::isfinite(norm->eps) || norm->eps < 0) return FBL_ERR_ARG;
    if (norm->reserved) return FBL_ERR_ARG;
    p.wq = norm->q_weight, p.wk = norm->k_weight, p.eps = norm->eps;
    for (const void* w : {p.wq, p.wk})
        if (reinterpret_cast<uintptr_t>(w) % (uintptr_t)es) return FBL_ERR_ALIGN;
    return FBL_OK;
}

bool same_layout(const void* pa, const fbl_layout* a, const void* pb, const fbl_layout* b) {
    return pa == pb && a->ss == b->ss && a->sh == b->sh && (a->B == 1 || a->sb == b->sb);
}

struct View {
    const fbl_layout* l;
    const void* p;
};
// Whether an output may be written while the inputs are read: it lies apart from all of them, or exactly on `on`.
bool clear_of(const View& out, const View* in, int n, int on) {
    for (int i = 0; i < n; ++i)
        if (in[i].p && !(i == on && same_layout(out.p, out.l, in[i].p, in[i].l)) &&
            views_overlap(out.p, out.l, in[i].p, in[i].l))
            return false;
    return true;
}
bool clear_of(const View& out, const void* p, int64_t bytes) { return !p || !overlaps(out.p, span_bytes(out.l), p, bytes); }

// The span of positions and turns, in bytes.
int64_t positions_span(const fbl_rotary* r, int64_t B, int64_t S) {
    return 8 * ((r->num_axes - 1) * r->stride_axis + (B - 1) * r->stride_batch + (S - 1) * r->stride_token + 1);
}
bool clear_of_plan(const View& out, const fbl_rotary* rot, const fbl_head_norm* norm, int64_t es) {
    if (rot && !(clear_of(out, rot->turns, rot->dims * 4) && clear_of(out, rot->positions, positions_span(rot, out.l->B, out.l->S))))
        return false;
    return !norm || (clear_of(out, norm->q_weight, out.l->D * es) && clear_of(out, norm->k_weight, out.l->D * es));
}

}  // namespace

extern "C" {

fbl_status fbl_rotary_turns(const double* frequencies, int64_t n, uint64_t* turns) {
    if (!frequencies || !turns) return FBL_ERR_NULL;
    if (n <= 0) return FBL_ERR_SHAPE;
    for (int64_t i = 0; i < n; ++i)
        if (!std::isfinite(frequencies[i])) return FBL_ERR_ARG;
    for (int64_t i = 0; i < n; ++i) {
        long double t = (long double)frequencies[i] / 6.283185307179586476925286766559L;
        t -= std::floor(t);
        t = std::floor(std::ldexp(t, 64) + 0.5L);
        turns[i] = t >= 18446744073709551616.0L ? 0 : (uint64_t)t;
    }
    return FBL_OK;
}

fbl_status fbl_qk_norm_rotary_fwd(const fbl_layout* lq, const void* q, const fbl_layout* lk, const void* k,
                                  const fbl_rotary* rot, const fbl_head_norm* norm, const fbl_layout* lqo, void* qo,
                                  const fbl_layout* lko, void* ko, void* stream) {
    if (!lq || !q || !lqo || !qo || !lk != !k || !lko != !ko || !k != !ko) return FBL_ERR_NULL;
    if (!rot && !norm) return FBL_ERR_ARG;
    fbl_status st = check_heads(lq, lk);
    if (st != FBL_OK) return st;
    if ((st = check_tensor(lq, q, lq)) != FBL_OK || (st = check_tensor(lqo, qo, lq)) != FBL_OK) return st;
    if (k && ((st = check_tensor(lk, k, lk)) != FBL_OK || (st = check_tensor(lko, ko, lk)) != FBL_OK)) return st;
    const int f32 = lq->dtype == FBL_F32;
    const int64_t es = f32 ? 4 : 2;
    fbl::RotaryArgs p{};
    if ((st = set_rotation(p, rot, lq)) != FBL_OK || (st = set_norm(p, norm, es)) != FBL_OK) return st;
    const View in[] = {{lq, q}, {lk, k}}, out[] = {{lqo, qo}, {lko, ko}};
    for (int i = 0; i < (k ? 2 : 1); ++i)
        if (!clear_of(out[i], in, 2, i) || !clear_of_plan(out[i], rot, norm, es)) return FBL_ERR_ARG;
    if (k && views_overlap(qo, lqo, ko, lko)) return FBL_ERR_ARG;
    p.q = q, p.oq = qo, p.mq = tokmap(lq), p.moq = tokmap(lqo);
    if (k) p.k = k, p.ok = ko, p.mk = tokmap(lk), p.mok = tokmap(lko);
    p.B = (int)lq->B, p.S = (int)lq->S, p.Hq = (int)lq->H, p.Hkv = k ? (int)lk->H : 0;
    plan(p, f32, lq->D, false);
    const hipError_t e = fbl::launch_qk_norm_rotary(f32, (int)lq->D, rot && rot->neighbours, norm != nullptr, 0, p,
                                                    static_cast<hipStream_t>(stream));
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

fbl_status fbl_qk_norm_rotary_bwd_workspace(const fbl_layout* lq, const fbl_layout* lk, size_t* bytes) {
    if (!lq || !bytes) return FBL_ERR_NULL;
    const fbl_status st = check_heads(lq, lk);
    if (st != FBL_OK) return st;
    fbl::RotaryArgs p{};
    p.B = (int)lq->B, p.S = (int)lq->S, p.Hq = (int)lq->H, p.Hkv = lk ? (int)lk->H : 0;
    plan(p, lq->dtype == FBL_F32, lq->D, true);
    *bytes = (size_t)p.workgroups * 2 * (size_t)lq->D * 4;
    return FBL_OK;
}

fbl_status fbl_qk_norm_rotary_bwd(const fbl_layout* lgq, const void* gq, const fbl_layout* lgk, const void* gk,
                                  const fbl_layout* lq, const void* q, const fbl_layout* lk, const void* k,
                                  const fbl_rotary* rot, const fbl_head_norm* norm, const fbl_layout* ldq, void* dq,
                                  const fbl_layout* ldk, void* dk, void* dq_weight, void* dk_weight, void* ws,
                                  size_t ws_bytes, void* stream) {
    if (!lgq || !gq || !ldq || !dq || !lgk != !gk || !ldk != !dk || !gk != !dk) return FBL_ERR_NULL;
    if (!rot && !norm) return FBL_ERR_ARG;
    if (norm && (!lq || !q || !lk != !gk || !k != !gk)) return FBL_ERR_NULL;
    if (!norm && (dq_weight || dk_weight)) return FBL_ERR_ARG;
    if (dk_weight && !gk) return FBL_ERR_ARG;
    fbl_status st = check_heads(lgq, lgk);
    if (st != FBL_OK) return st;
    if ((st = check_tensor(lgq, gq, lgq)) != FBL_OK || (st = check_tensor(ldq, dq, lgq)) != FBL_OK) return st;
    if (gk && ((st = check_tensor(lgk, gk, lgk)) != FBL_OK || (st = check_tensor(ldk, dk, lgk)) != FBL_OK)) return st;
    if (norm && (st = check_tensor(lq, q, lgq)) != FBL_OK) return st;
    if (norm && gk && (st = check_tensor(lk, k, lgk)) != FBL_OK) return st;
    const int f32 = lgq->dtype == FBL_F32;
    const int64_t es = f32 ? 4 : 2, D = lgq->D;
    fbl::RotaryArgs p{};
    if ((st = set_rotation(p, rot, lgq)) != FBL_OK || (st = set_norm(p, norm, es)) != FBL_OK) return st;
    p.B = (int)lgq->B, p.S = (int)lgq->S, p.Hq = (int)lgq->H, p.Hkv = gk ? (int)lgk->H : 0;
    const bool sums = dq_weight || dk_weight;
    plan(p, f32, D, sums);
    const int64_t need = sums ? (int64_t)p.workgroups * 2 * D * 4 : 0;
    if (sums && (!ws || ws_bytes < (size_t)need)) return FBL_ERR_WORKSPACE;
    if (sums && reinterpret_cast<uintptr_t>(ws) % 4) return FBL_ERR_ALIGN;
    const View in[] = {{lgq, gq}, {lgk, gk}, {lq, norm ? q : nullptr}, {lk, norm ? k : nullptr}}, out[] = {{ldq, dq}, {ldk, dk}};
    for (int i = 0; i < (gk ? 2 : 1); ++i)
        if (!clear_of(out[i], in, 4, i) || !clear_of_plan(out[i], rot, norm, es)) return FBL_ERR_ARG;
    if (gk && views_overlap(dq, ldq, dk, ldk)) return FBL_ERR_ARG;
    // the weights' gradients and the workspace: apart from everything and from each other
    struct Span {
        const void* p;
        int64_t bytes;
    };
    const Span small[] = {{dq_weight, D * es}, {dk_weight, D * es}, {sums ? ws : nullptr, need}};
    for (int i = 0; i < 3; ++i) {
        if (!small[i].p) continue;
        if (reinterpret_cast<uintptr_t>(small[i].p) % (uintptr_t)es) return FBL_ERR_ALIGN;
        for (const View& v : in)
            if (v.p && overlaps(v.p, span_bytes(v.l), small[i].p, small[i].bytes)) return FBL_ERR_ARG;
        for (int j = 0; j < (gk ? 2 : 1); ++j)
            if (!clear_of(out[j], small[i].p, small[i].bytes)) return FBL_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (small[j].p && overlaps(small[j].p, small[j].bytes, small[i].p, small[i].bytes)) return FBL_ERR_ARG;
        for (const void* w : {p.wq, p.wk})
            if (w && overlaps(w, D * es, small[i].p, small[i].bytes)) return FBL_ERR_ARG;
        if (rot && overlaps(rot->turns, rot->dims * 4, small[i].p, small[i].bytes)) return FBL_ERR_ARG;
        if (rot && rot->positions && overlaps(rot->positions, positions_span(rot, p.B, p.S), small[i].p, small[i].bytes))
            return FBL_ERR_ARG;
    }
    p.gq = gq, p.oq = dq, p.mgq = tokmap(lgq), p.moq = tokmap(ldq);
    if (gk) p.gk = gk, p.ok = dk, p.mgk = tokmap(lgk), p.mok = tokmap(ldk);
    if (norm) {
        p.q = q, p.mq = tokmap(lq);
        if (gk) p.k = k, p.mk = tokmap(lk);
    }
    p.sums = sums ? static_cast<float*>(ws) : nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = fbl::launch_qk_norm_rotary(f32, (int)D, rot && rot->neighbours, norm != nullptr, 1, p, s);
    if (e == hipSuccess && sums) e = fbl::launch_column_sums(f32, p.sums, p.workgroups, 2, (int)D, dq_weight, dk_weight, s);
    return e == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

}  // extern "C"
