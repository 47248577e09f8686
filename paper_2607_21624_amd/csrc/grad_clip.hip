// grad_clip.hip -- the global norm over a list of tensors, and the tensors clipped by it, gfx950.
//
//   norm = sqrt(sum of squares over all values of all tensors),  out = g * min(1, limit / (norm + 1e-6))
//
// Bound by memory: the norm reads every value once, clipping reads and writes it once more, or does
// neither where it is in place and the norm is within the limit.  The list travels in the kernel's arguments, so that a
// call copies nothing and can be captured.  Tensors are cut into chunks of 16 KB; a workgroup walks every gridDim-th of
// them.  Squares are summed in float64: no square overflows or vanishes, and a sum of 2^30 terms keeps fp32's digits.
// Each workgroup leaves one sum; whoever needs the norm adds them in the same fixed order.  Clipping walks the chunks from
// the last one back: the norm has read the end of the list last (bf16, both launches, in the norm's order and back: into other
// tensors 268 M values 311 -> 297 us, 134 M 152.8 -> 148.1; in place 268 M 319 -> 313, lists of 134 M and less the same).
//
// 268 M values bf16: squares 108 us (5.0 TB/s), scaling into other tensors 185 (5.8).  85 M in place within the limit: 27 and 5.
#include "kernels.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

constexpr int kLoads = 4;                      // 16-byte loads of a thread and chunk
constexpr int kChunkBytes = 256 * 16 * kLoads;
static_assert(kChunkBytes == kGradChunk, "chunks as the host counts them");

FBL_DEV double wave_sum(double x) {
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) x += __shfl_xor(x, d);
    return x;
}
FBL_DEV double group_sum(double x, double* red) {  // over 256 threads, the same in each
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// The tensor that chunk c belongs to: the last whose first chunk is not behind it.
FBL_DEV int tensor_of(const GradList& a, int c) {
    int lo = 0, hi = a.count;  // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A thread's share of a chunk, `left` elements long: 16 bytes of every 4 KB.  What would reach past the chunk's end is
// read from before it and its own elements kept (Pack), so that all loads are on the way at once at any length; in
// place, what others may have written meanwhile is not among them.
template <typename T>
struct Share {
    using P = Pack<T>;
    P x[kLoads];
    static FBL_DEV int at(int k) { return (k * 256 + (int)threadIdx.x) * P::N; }
    FBL_DEV void load(const T* p, int left) {
        if (left == kChunkBytes / (int)sizeof(T)) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) x[k].fetch(p, at(k), kChunkBytes / (int)sizeof(T));
        } else if (left >= P::N) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) x[k].fetch(p, at(k), left);
#pragma unroll
            for (int k = 0; k < kLoads; ++k) x[k].settle(at(k), left);
        } else {  // the first thread's alone
#pragma unroll
            for (int k = 1; k < kLoads; ++k) x[k] = P{};
            x[0].template fetch<true>(p, at(0), left);
        }
    }
};

template <typename T>
FBL_DEV double square_sum(const void* base, int64_t i0, int64_t n) {
    Share<T> a;
    a.load(static_cast<const T*>(base) + i0, (int)min(n - i0, (int64_t)(kChunkBytes / sizeof(T))));
    double s = 0;
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
        for (int e = 0; e < Pack<T>::N; ++e) {
            const double v = (double)a.x[k][e];
            s = __builtin_fma(v, v, s);
        }
    return s;
}

template <typename T>
FBL_DEV void scaled(const void* from, void* to, int64_t i0, int64_t n, float scale) {
    Share<T> a;
    const int left = (int)min(n - i0, (int64_t)(kChunkBytes / sizeof(T)));
    a.load(static_cast<const T*>(from) + i0, left);
    T* const q = static_cast<T*>(to) + i0;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
#pragma unroll
        for (int e = 0; e < Pack<T>::N; ++e) a.x[k].set(e, a.x[k][e] * scale);
        a.x[k].store(q, a.at(k), left);
    }
}

__global__ __launch_bounds__(256) void grad_squares(GradList a, double* sums) {
    __shared__ double red[4];
    double s = 0;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int t = tensor_of(a, c);
        const int64_t at = (int64_t)(c - a.first[t]) * kChunkBytes;  // bytes
        s += a.t[t].f32 ? square_sum<float>(a.t[t].p, at / 4, a.t[t].n) : square_sum<bf16>(a.t[t].p, at / 2, a.t[t].n);
    }
    s = group_sum(s, red);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// The norm from all workgroups' sums, the same in every thread.
FBL_DEV float norm_of(const double* sums, int n, double* red) {
    double s = 0;
    for (int i = threadIdx.x; i < n; i += 256) s += sums[i];
    return (float)__builtin_sqrt(group_sum(s, red));
}

__global__ __launch_bounds__(256) void grad_norm(const double* sums, int n, float* norm) {
    __shared__ double red[4];
    const float x = norm_of(sums, n, red);
    if (threadIdx.x == 0) norm[0] = x;
}

__global__ __launch_bounds__(256) void grad_scale(GradList a, const double* sums, int n, float* norm, float limit) {
    __shared__ double red[4];
    const float x = sums ? norm_of(sums, n, red) : norm[0];
    if (sums && norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = x;
    const double ratio = (double)limit / ((double)x + 1e-6);
    // (a norm that is nan makes everything nan; without a limit nothing changes, whatever the norm)
    const float scale = ratio >= 1.0 || limit == __builtin_inff() ? 1.f : (float)ratio;
    if (scale == 1.f && a.in_place) return;
    for (int c = a.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const int t = tensor_of(a, c);
        const int64_t at = (int64_t)(c - a.first[t]) * kChunkBytes;
        if (a.t[t].f32) scaled<float>(a.t[t].p, a.t[t].out, at / 4, a.t[t].n, scale);
        else scaled<bf16>(a.t[t].p, a.t[t].out, at / 2, a.t[t].n, scale);
    }
}

}  // namespace

hipError_t launch_grad_squares(const GradList& a, double* sums, int workgroups, hipStream_t s) {
    hipLaunchKernelGGL(grad_squares, dim3((unsigned)workgroups), dim3(256), 0, s, a, sums);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const double* sums, int n, float* norm, hipStream_t s) {
    hipLaunchKernelGGL(grad_norm, dim3(1), dim3(256), 0, s, sums, n, norm);
    return hipGetLastError();
}

hipError_t launch_grad_scale(const GradList& a, const double* sums, int n, float* norm, float limit, int workgroups, hipStream_t s) {
    hipLaunchKernelGGL(grad_scale, dim3((unsigned)workgroups), dim3(256), 0, s, a, sums, n, norm, limit);
    return hipGetLastError();
}

}  // namespace fbl
