// api_grad.cpp -- the C ABI of the global gradient norm and of clipping by it: validation
// and dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "kernels.hpp"
#include "rows_check.hpp"

namespace {

using fbl::GradList;

constexpr int kWorkgroups = 1024;  // of a launch: their sums are added by every workgroup that clips (85 M values within the limit: 2048 41, 1024 38 us)
constexpr int64_t kMostBytes = (int64_t)1 << 44;  // of a list: its chunks count to 2^30
static_assert(kMostBytes / fbl::kGradChunk + fbl::kGradTensors < INT32_MAX - kWorkgroups, "a chunk's index is an int");

int64_t launches(int64_t count) { return (count + fbl::kGradTensors - 1) / fbl::kGradTensors; }
size_t norm_ws(int64_t count) { return (size_t)launches(count) * kWorkgroups * sizeof(double); }

struct Range {
    uintptr_t begin, end;
};

// Every tensor by itself, and all that is read or written apart: `also` are further ranges (norm, workspace).
fbl_status check(int64_t count, const fbl_grad* g, bool outs, const Range* also, int n) {
    if (count <= 0 || count > INT32_MAX) return FBL_ERR_SHAPE;
    if (!g) return FBL_ERR_NULL;
    try {
        std::vector<Range> r(also, also + n);
        r.reserve((size_t)(2 * count + n));
        int64_t total = 0;
        for (int64_t i = 0; i < count; ++i) {
            const int64_t es = fbl::dtype_size(g[i].dtype);
            if (!es) return FBL_ERR_DTYPE;
            if (g[i].n < 0) return FBL_ERR_SHAPE;
            if (g[i].n > kMostBytes / es || (total += g[i].n * es) > kMostBytes) return FBL_ERR_UNSUPPORTED;
            if (g[i].reserved) return FBL_ERR_ARG;
            if (g[i].n == 0) continue;
            if (!g[i].p || (outs && !g[i].out)) return FBL_ERR_NULL;
            const uintptr_t p = reinterpret_cast<uintptr_t>(g[i].p), o = reinterpret_cast<uintptr_t>(g[i].out);
            if (p % (uintptr_t)es || (outs && o % (uintptr_t)es)) return FBL_ERR_ALIGN;
            r.push_back({p, p + (uintptr_t)(g[i].n * es)});
            if (outs && o != p) r.push_back({o, o + (uintptr_t)(g[i].n * es)});
        }
        std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
        for (size_t i = 1; i < r.size(); ++i)
            if (r[i].begin < r[i - 1].end) return FBL_ERR_ARG;
    } catch (...) {  // no memory on the host
        return FBL_ERR_ARG;
    }
    return FBL_OK;
}

// f(list, workgroups) for the tensors of each launch in turn.
template <typename F>
fbl_status for_lists(int64_t count, const fbl_grad* g, bool outs, F&& f) {
    for (int64_t i = 0; i < count;) {
        GradList a;
        a.count = 0, a.in_place = 1;
        int64_t chunks = 0;
        for (; i < count && a.count < fbl::kGradTensors; ++i) {
            if (g[i].n == 0) continue;
            const int64_t bytes = g[i].n * fbl::dtype_size(g[i].dtype);
            auto& t = a.t[a.count];
            t.p = g[i].p, t.out = outs ? g[i].out : nullptr, t.n = g[i].n, t.f32 = g[i].dtype == FBL_F32;
            if (t.out != t.p) a.in_place = 0;
            a.first[a.count++] = (int)chunks;
            chunks += (bytes + fbl::kGradChunk - 1) / fbl::kGradChunk;
        }
        if (a.count == 0) break;
        a.first[a.count] = a.chunks = (int)chunks;
        if (f(a, (int)std::min<int64_t>(chunks, kWorkgroups)) != hipSuccess) return FBL_ERR_HIP;
    }
    return FBL_OK;
}

fbl_status squares(int64_t count, const fbl_grad* g, double* sums, int* n, hipStream_t s) {
    *n = 0;
    return for_lists(count, g, false, [&](const GradList& a, int workgroups) {
        const hipError_t e = fbl::launch_grad_squares(a, sums + *n, workgroups, s);
        *n += workgroups;
        return e;
    });
}

Range range(const void* p, size_t bytes) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {b, b + bytes};
}

}  // namespace

extern "C" {

fbl_status fbl_grad_norm_workspace(int64_t count, size_t* bytes) {
    if (!bytes) return FBL_ERR_NULL;
    if (count <= 0 || count > INT32_MAX) return FBL_ERR_SHAPE;
    *bytes = norm_ws(count);
    return FBL_OK;
}

fbl_status fbl_grad_norm(int64_t count, const fbl_grad* grads, float* norm, void* ws, size_t ws_bytes, void* stream) {
    if (count <= 0 || count > INT32_MAX) return FBL_ERR_SHAPE;
    if (!norm) return FBL_ERR_NULL;
    if (!ws || ws_bytes < norm_ws(count)) return FBL_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(norm) % 4 || reinterpret_cast<uintptr_t>(ws) % 8) return FBL_ERR_ALIGN;
    const Range also[] = {range(norm, 4), range(ws, norm_ws(count))};
    fbl_status st = check(count, grads, false, also, 2);
    if (st != FBL_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int n;
    st = squares(count, grads, static_cast<double*>(ws), &n, s);
    if (st != FBL_OK) return st;
    return fbl::launch_grad_norm(static_cast<double*>(ws), n, norm, s) == hipSuccess ? FBL_OK : FBL_ERR_HIP;
}

fbl_status fbl_grad_clip(int64_t count, const fbl_grad* grads, const float* norm, float limit, void* stream) {
    if (count <= 0 || count > INT32_MAX) return FBL_ERR_SHAPE;
    if (!norm) return FBL_ERR_NULL;
    if (!(limit >= 0)) return FBL_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(norm) % 4) return FBL_ERR_ALIGN;
    const Range also[] = {range(norm, 4)};
    const fbl_status st = check(count, grads, true, also, 1);
    if (st != FBL_OK) return st;
    return for_lists(count, grads, true, [&](const GradList& a, int workgroups) {
        return fbl::launch_grad_scale(a, nullptr, 0, const_cast<float*>(norm), limit, workgroups, static_cast<hipStream_t>(stream));
    });
}

fbl_status fbl_clip_grad_norm(int64_t count, const fbl_grad* grads, float limit, float* norm, void* ws, size_t ws_bytes,
                              void* stream) {
    if (count <= 0 || count > INT32_MAX) return FBL_ERR_SHAPE;
    if (!norm) return FBL_ERR_NULL;
    if (!(limit >= 0)) return FBL_ERR_ARG;
    if (!ws || ws_bytes < norm_ws(count)) return FBL_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(norm) % 4 || reinterpret_cast<uintptr_t>(ws) % 8) return FBL_ERR_ALIGN;
    const Range also[] = {range(norm, 4), range(ws, norm_ws(count))};
    fbl_status st = check(count, grads, true, also, 2);
    if (st != FBL_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    double* const sums = static_cast<double*>(ws);
    int n;
    st = squares(count, grads, sums, &n, s);
    if (st != FBL_OK) return st;
    if (n == 0) return fbl::launch_grad_norm(sums, 0, norm, s) == hipSuccess ? FBL_OK : FBL_ERR_HIP;
    return for_lists(count, grads, true, [&](const GradList& a, int workgroups) {
        return fbl::launch_grad_scale(a, sums, n, norm, limit, workgroups, s);
    });
}

}  // extern "C"
