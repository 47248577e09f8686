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
// without a second read.  The next row is on its way while this one is summed.  Statistics
// and sums are fp32.  16384 x 4096 bf16: forward 47 us (5.8 TB/s, part of it from the last-level cache),
// backward 84 us (4.8 TB/s; a 1 GiB copy reaches 4.8); 52 and 136 us with loads that decided about the
// row's end where they were issued, which made each wait for the one before.
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
    // 16 wavefronts' registers have no room for the sums of 16 columns a lane: these keep them in LDS,
    // each lane its own (128 KB; 2048 x 16384 bf16 159 -> 59 us)
    static constexpr bool kLdsSums = LPR == 1024 && VEC * C > 8;
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

template <typename T, int LPR, int C, bool SHORT>
__global__ __launch_bounds__((NormCfg<T, LPR, C>::NT)) void layer_norm_fwd(NormArgs a) {
    using Cfg = NormCfg<T, LPR, C>;
    using P = Pack<T>;
    __shared__ float red[2][16];
    const int slot = threadIdx.x / LPR, l = threadIdx.x % LPR, n = a.N;
    const bool has_w = a.w != nullptr, has_b = a.b != nullptr;
    const int64_t step = (int64_t)gridDim.x * Cfg::SLOTS;
    int64_t m = (int64_t)blockIdx.x * Cfg::SLOTS + slot;
    if (m >= a.M) return;  // whole rows of lanes, and where they are more than a wavefront the workgroup
    P pw[C], pb[C], next[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * LPR + l) * P::N;
        next[c].template fetch<SHORT>(static_cast<const T*>(a.x) + m * a.ldx, col, n);
        if (has_w) pw[c].template fetch<SHORT>(static_cast<const T*>(a.w), col, n);
        if (has_b) pb[c].template fetch<SHORT>(static_cast<const T*>(a.b), col, n);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (has_w) pw[c].template settle<SHORT>((c * LPR + l) * P::N, n);
        if (has_b) pb[c].template settle<SHORT>((c * LPR + l) * P::N, n);
    }
    for (; m < a.M; m += step) {
        P px[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            px[c] = next[c];
            px[c].template settle<SHORT>((c * LPR + l) * P::N, n);
        }
        if (m + step < a.M) {  // the next row is on its way during this one's sums
#pragma unroll
            for (int c = 0; c < C; ++c)
                next[c].template fetch<SHORT>(static_cast<const T*>(a.x) + (m + step) * a.ldx, (c * LPR + l) * P::N, n);
        }
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < P::N; ++e) s[0] += px[c][e];
        row_sums<LPR>(s, red[0]);
        const float mean = s[0] / (float)n;  // a row of equal values has them for its mean, where their sum is exact
        float q[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
                const float d = (c * LPR + l) * P::N + e < n ? px[c][e] - mean : 0.f;
                q[0] = __builtin_fmaf(d, d, q[0]);
            }
        row_sums<LPR>(q, red[1]);
        const float rstd = 1.f / sqrtf(q[0] / (float)n + a.eps);
        if (l == 0 && a.mean) {
            a.mean[m] = mean;
            a.rstd[m] = rstd;
        }
        T* y = static_cast<T*>(a.y) + m * a.ldy;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            P py;
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
                const float xh = (px[c][e] - mean) * rstd;
                py.set(e, __builtin_fmaf(xh, has_w ? pw[c][e] : 1.f, has_b ? pb[c][e] : 0.f));
            }
            py.store(y, (c * LPR + l) * P::N, n);
        }
    }
}

template <typename T, int LPR, int C, bool SHORT>
__global__ __launch_bounds__((NormCfg<T, LPR, C>::NT)) void layer_norm_bwd(NormArgs a) {
    using Cfg = NormCfg<T, LPR, C>;
    using P = Pack<T>;
    constexpr int V = P::N;
    extern __shared__ __attribute__((aligned(16))) float wide[];  // kLdsSums: [2][CAP]
    __shared__ float red[2][32];
    __shared__ float cols[Cfg::SLOTS > 1 ? Cfg::SLOTS * Cfg::CAP : 1];
    const int slot = threadIdx.x / LPR, l = threadIdx.x % LPR, n = a.N;
    const bool has_w = a.w != nullptr;
    float sw[C][V], sb[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (Cfg::kLdsSums) wide[(c * LPR + l) * V + e] = wide[Cfg::CAP + (c * LPR + l) * V + e] = 0.f;
            else sw[c][e] = sb[c][e] = 0.f;
        }
    int turn = 0;
    const int64_t step = (int64_t)gridDim.x * Cfg::SLOTS;
    int64_t m = (int64_t)blockIdx.x * Cfg::SLOTS + slot;
    P pw[C], nx[C], nd[C];
    float nmean, nrstd;
    const auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        nmean = a.mean[row], nrstd = a.rstd[row];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            nx[c].template fetch<SHORT>(static_cast<const T*>(a.x) + row * a.ldx, (c * LPR + l) * V, n);
            nd[c].template fetch<SHORT>(static_cast<const T*>(a.dy) + row * a.lddy, (c * LPR + l) * V, n);
        }
    };
    if (m < a.M) fetch(m);
    if (has_w) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            pw[c].template fetch<SHORT>(static_cast<const T*>(a.w), (c * LPR + l) * V, n);
            pw[c].template settle<SHORT>((c * LPR + l) * V, n);
        }
    }
    for (; m < a.M; m += step) {
        const float mean = nmean, rstd = nrstd;
        P px[C], pd[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            px[c] = nx[c], pd[c] = nd[c];
            px[c].template settle<SHORT>((c * LPR + l) * V, n);
            pd[c].template settle<SHORT>((c * LPR + l) * V, n);
        }
        if (m + step < a.M) fetch(m + step);  // the next row is on its way during this one's sums
        float s[2] = {0.f, 0.f};  // sums of g and of g xh
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float* const lw = wide + (c * LPR + l) * V;
#pragma unroll
            for (int e = 0; e < V; ++e) {  // past the row's end dy is 0, and so are both terms
                const float xh = (px[c][e] - mean) * rstd, d = pd[c][e], g = has_w ? d * pw[c][e] : d;
                s[0] += g;
                s[1] = __builtin_fmaf(g, xh, s[1]);
                if constexpr (Cfg::kLdsSums) {
                    lw[e] = __builtin_fmaf(d, xh, lw[e]);
                    lw[Cfg::CAP + e] += d;
                } else {
                    sw[c][e] = __builtin_fmaf(d, xh, sw[c][e]);
                    sb[c][e] += d;
                }
            }
        }
        row_sums<LPR>(s, red[turn]);
        turn ^= 1;
        const float c1 = s[0] / (float)n, c2 = s[1] / (float)n;
        T* dx = static_cast<T*>(a.dx) + m * a.lddx;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            P po;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (px[c][e] - mean) * rstd, g = has_w ? pd[c][e] * pw[c][e] : pd[c][e];
                po.set(e, rstd * (g - c1 - xh * c2));
            }
            po.store(dx, (c * LPR + l) * V, n);
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
                    if (col < n) part[k * n + col] = Cfg::kLdsSums ? wide[k * Cfg::CAP + col] : v[c][e];
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
template <typename T, template <typename, int, int, bool> class F>
hipError_t for_width(int N, const NormArgs& a, hipStream_t s) {
    constexpr int V = Pack<T>::N;
    if (N < V) return F<T, 16, 1, true>::run(a, s);
    if (N <= 16 * V) return F<T, 16, 1, false>::run(a, s);  // (layer_norm_slots has the same limits)
    if (N <= 64 * V) return F<T, 64, 1, false>::run(a, s);
    if (N <= 128 * V) return F<T, 64, 2, false>::run(a, s);
    if (N <= 256 * V) return F<T, 256, 1, false>::run(a, s);
    if (N <= 512 * V) return F<T, 256, 2, false>::run(a, s);
    if constexpr (V == 4) {
        if (N <= 1024 * V) return F<T, 256, 4, false>::run(a, s);
        if (N <= 2048 * V) return F<T, 1024, 2, false>::run(a, s);
        return F<T, 1024, 4, false>::run(a, s);
    } else {
        if (N <= 1024 * V) return F<T, 1024, 1, false>::run(a, s);
        return F<T, 1024, 2, false>::run(a, s);
    }
}

template <typename T, int LPR, int C, bool SHORT>
struct RunFwd {
    static hipError_t run(const NormArgs& a, hipStream_t s) {
        using Cfg = NormCfg<T, LPR, C>;
        const int64_t wgs = (a.M + Cfg::SLOTS - 1) / Cfg::SLOTS, most = 256 * 2048 / Cfg::NT;
        hipLaunchKernelGGL((layer_norm_fwd<T, LPR, C, SHORT>), dim3((unsigned)(wgs < most ? wgs : most)), dim3(Cfg::NT), 0, s, a);
        return hipGetLastError();
    }
};

template <typename T, int LPR, int C, bool SHORT>
struct RunBwd {
    static hipError_t run(const NormArgs& a, hipStream_t s) {
        using Cfg = NormCfg<T, LPR, C>;
        constexpr auto kernel = &layer_norm_bwd<T, LPR, C, SHORT>;
        constexpr int lds = Cfg::kLdsSums ? 2 * Cfg::CAP * 4 : 0;
        if constexpr (lds > 0) {
            const hipError_t once = ensure_dynamic_lds<kernel>(lds);
            if (once != hipSuccess) return once;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.groups), dim3(Cfg::NT), lds, s, a);
        return hipGetLastError();
    }
};

}  // namespace

int layer_norm_slots(int f32, int N) {
    const int v = f32 ? Pack<float>::N : Pack<bf16>::N;
    return N <= 16 * v ? 16 : N <= 128 * v ? 4 : 1;
}

bool layer_norm_wide(int f32, int N) { return N > (f32 ? 1024 * Pack<float>::N : 512 * Pack<bf16>::N); }

hipError_t launch_layer_norm_fwd(int f32, const NormArgs& a, hipStream_t s) {
    return f32 ? for_width<float, RunFwd>(a.N, a, s) : for_width<bf16, RunFwd>(a.N, a, s);
}

hipError_t launch_layer_norm_bwd(int f32, const NormArgs& a, hipStream_t s) {
    const hipError_t e = f32 ? for_width<float, RunBwd>(a.N, a, s) : for_width<bf16, RunBwd>(a.N, a, s);
    if (e != hipSuccess || !a.part) return e;
    return launch_column_sums(f32, a.part, a.groups, 2, a.N, a.dw, a.db, s);
}

}  // namespace fbl
