// layer_norm.hip -- layer norm over rows of N values, forward and backward, gfx950.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r
//   y  = xh * w + b
//   dx = r (g - mean(g) - xh mean(g xh)),  g = dy * w
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Both passes are bound by memory: the forward reads x and writes y, the
// backward reads x and dy and writes dx, once.  A row is shared by LPR lanes (16, a
// wavefront, 4 or 16 wavefronts) that hold all of it in registers, C 16-byte chunks
// each, so the variance is taken about the mean (two sums, no cancellation)
// without a second read.  Statistics and sums are fp32.
//
// The weight's and bias' gradients are sums down the columns.  Every lane keeps
// them in registers for its columns over all rows its workgroup walks; the
// workgroup adds its row slots through LDS and writes one row of partial sums,
// which layer_norm_cols adds in a fixed order (no atomics: bitwise
// repeatable).
#include "kernels.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

// Rows of a workgroup: LPR lanes a row, 256 threads or the 1024 of one row.
template <typename T, int LPR, int C>
struct NormCfg {
    static constexpr int NT = LPR > 256 ? LPR : 256;
    static constexpr int SLOTS = NT / LPR;
    static constexpr int VEC = Pack<T>::N;
    static constexpr int CAP = LPR * VEC * C;  // values of the longest row
    static constexpr int NWR = LPR / 64;       // wavefronts that share a row (0: less than one)
};

// Sums over the LPR lanes of a row; `red` is the caller's own LDS for this call
// (its next use at least one other row_sums in between).
template <int LPR, int K>
FBL_DEV void row_sums(float (&x)[K], float* red) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = lane_sum<(LPR < 64 ? 16 : 64)>(x[k]);
    if constexpr (LPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) red[wave * K + k] = x[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            x[k] = red[k];
#pragma unroll
            for (int w = 1; w < LPR / 64; ++w) x[k] += red[w * K + k];
        }
    }
}

template <typename T, int LPR, int C>
__global__ __launch_bounds__((NormCfg<T, LPR, C>::NT)) void layer_norm_fwd(NormArgs a) {
    using Cfg = NormCfg<T, LPR, C>;
    using P = Pack<T>;
    __shared__ float red[2][16];
    const int slot = threadIdx.x / LPR, l = threadIdx.x % LPR, n = a.N;
    const float inv = 1.f / (float)n;
    const T* w = static_cast<const T*>(a.w);
    const T* b = static_cast<const T*>(a.b);
    for (int64_t m = (int64_t)blockIdx.x * Cfg::SLOTS + slot; m < a.M; m += (int64_t)gridDim.x * Cfg::SLOTS) {
        const T* x = static_cast<const T*>(a.x) + m * a.ldx;
        P px[C];
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            px[c].load(x, (c * LPR + l) * P::N, n);
#pragma unroll
            for (int e = 0; e < P::N; ++e) s[0] += px[c][e];
        }
        row_sums<LPR>(s, red[0]);
        const float mean = s[0] / (float)n;  // a row of equal values has them for its mean, where their sum is exact
        float q[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
                const float d = px[c][e] - mean;
                if ((c * LPR + l) * P::N + e < n) q[0] = __builtin_fmaf(d, d, q[0]);
            }
        row_sums<LPR>(q, red[1]);
        const float rstd = 1.f / sqrtf(q[0] * inv + a.eps);
        if (l == 0 && a.mean) {
            a.mean[m] = mean;
            a.rstd[m] = rstd;
        }
        T* y = static_cast<T*>(a.y) + m * a.ldy;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * LPR + l) * P::N;
            if (col >= n) break;
            P pw, pb, py;
            if (w) pw.load(w, col, n);
            if (b) pb.load(b, col, n);
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
                const float xh = (px[c][e] - mean) * rstd;
                py.set(e, __builtin_fmaf(xh, w ? pw[e] : 1.f, b ? pb[e] : 0.f));
            }
            py.store(y, col, n);
        }
    }
}

template <typename T, int LPR, int C>
__global__ __launch_bounds__((NormCfg<T, LPR, C>::NT)) void layer_norm_bwd(NormArgs a) {
    using Cfg = NormCfg<T, LPR, C>;
    using P = Pack<T>;
    constexpr int V = P::N;
    __shared__ float red[2][32];
    __shared__ float cols[Cfg::SLOTS > 1 ? Cfg::SLOTS * Cfg::CAP : 1];
    const int slot = threadIdx.x / LPR, l = threadIdx.x % LPR, n = a.N;
    const float inv = 1.f / (float)n;
    const T* w = static_cast<const T*>(a.w);
    float sw[C][V], sb[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) sw[c][e] = sb[c][e] = 0.f;
    int turn = 0;
    for (int64_t m = (int64_t)blockIdx.x * Cfg::SLOTS + slot; m < a.M; m += (int64_t)gridDim.x * Cfg::SLOTS) {
        const T* x = static_cast<const T*>(a.x) + m * a.ldx;
        const T* dy = static_cast<const T*>(a.dy) + m * a.lddy;
        const float mean = a.mean[m], rstd = a.rstd[m];
        P px[C], pd[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            px[c].load(x, (c * LPR + l) * V, n);
            pd[c].load(dy, (c * LPR + l) * V, n);
        }
        P pw[C];
        float s[2] = {0.f, 0.f};  // sums of g and of g xh
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (w) pw[c].load(w, (c * LPR + l) * V, n);
#pragma unroll
            for (int e = 0; e < V; ++e) {  // past the row's end dy is 0, and so are both terms
                const float xh = (px[c][e] - mean) * rstd, d = pd[c][e], g = w ? d * pw[c][e] : d;
                s[0] += g;
                s[1] = __builtin_fmaf(g, xh, s[1]);
                sw[c][e] = __builtin_fmaf(d, xh, sw[c][e]);
                sb[c][e] += d;
            }
        }
        row_sums<LPR>(s, red[turn]);
        turn ^= 1;
        const float c1 = s[0] * inv, c2 = s[1] * inv;
        T* dx = static_cast<T*>(a.dx) + m * a.lddx;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * LPR + l) * V;
            if (col >= n) break;
            P po;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (px[c][e] - mean) * rstd, g = w ? pd[c][e] * pw[c][e] : pd[c][e];
                po.set(e, rstd * (g - c1 - xh * c2));
            }
            po.store(dx, col, n);
        }
    }
    if (!a.part) return;
    // one row of partial sums per workgroup: [2][N], dw then db
    float* part = a.part + (int64_t)blockIdx.x * 2 * n;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float(&v)[C][V] = k == 0 ? sw : sb;
        if constexpr (Cfg::SLOTS == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int col = (c * LPR + l) * V + e;
                    if (col < n) part[k * n + col] = v[c][e];
                }
        } else {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < V; ++e) cols[slot * Cfg::CAP + (c * LPR + l) * V + e] = v[c][e];
            __syncthreads();
            for (int col = threadIdx.x; col < n; col += Cfg::NT) {
                float t = cols[col];
#pragma unroll
                for (int i = 1; i < Cfg::SLOTS; ++i) t += cols[i * Cfg::CAP + col];
                part[k * n + col] = t;
            }
        }
    }
}

// lanes and chunks of a row of N values
template <typename T, template <typename, int, int> class F>
hipError_t for_width(int N, const NormArgs& a, hipStream_t s) {
    constexpr int V = Pack<T>::N;
    if (N <= 16 * V) return F<T, 16, 1>::run(a, s);  // (layer_norm_slots has the same limits)
    if (N <= 64 * V) return F<T, 64, 1>::run(a, s);
    if (N <= 128 * V) return F<T, 64, 2>::run(a, s);
    if (N <= 256 * V) return F<T, 256, 1>::run(a, s);
    if (N <= 512 * V) return F<T, 256, 2>::run(a, s);
    if constexpr (V == 4) {
        if (N <= 1024 * V) return F<T, 256, 4>::run(a, s);
        if (N <= 2048 * V) return F<T, 1024, 2>::run(a, s);
        return F<T, 1024, 4>::run(a, s);
    } else {
        if (N <= 1024 * V) return F<T, 1024, 1>::run(a, s);
        return F<T, 1024, 2>::run(a, s);
    }
}

template <typename T, int LPR, int C>
struct RunFwd {
    static hipError_t run(const NormArgs& a, hipStream_t s) {
        using Cfg = NormCfg<T, LPR, C>;
        const int64_t wgs = (a.M + Cfg::SLOTS - 1) / Cfg::SLOTS;
        hipLaunchKernelGGL((layer_norm_fwd<T, LPR, C>), dim3((unsigned)(wgs < (1 << 20) ? wgs : 1 << 20)), dim3(Cfg::NT), 0, s, a);
        return hipGetLastError();
    }
};

template <typename T, int LPR, int C>
struct RunBwd {
    static hipError_t run(const NormArgs& a, hipStream_t s) {
        using Cfg = NormCfg<T, LPR, C>;
        hipLaunchKernelGGL((layer_norm_bwd<T, LPR, C>), dim3((unsigned)a.groups), dim3(Cfg::NT), 0, s, a);
        return hipGetLastError();
    }
};

}  // namespace

int layer_norm_slots(int f32, int N) {
    const int v = f32 ? Pack<float>::N : Pack<bf16>::N;
    return N <= 16 * v ? 16 : N <= 128 * v ? 4 : 1;
}

hipError_t launch_layer_norm_fwd(int f32, const NormArgs& a, hipStream_t s) {
    return f32 ? for_width<float, RunFwd>(a.N, a, s) : for_width<bf16, RunFwd>(a.N, a, s);
}

hipError_t launch_layer_norm_bwd(int f32, const NormArgs& a, hipStream_t s) {
    const hipError_t e = f32 ? for_width<float, RunBwd>(a.N, a, s) : for_width<bf16, RunBwd>(a.N, a, s);
    if (e != hipSuccess || !a.part) return e;
    return launch_column_sums(f32, a.part, a.groups, 2, a.N, a.dw, a.db, s);
}

}  // namespace fbl
