// column_sums.hip -- the last step of the gradients that are sums over rows: the
// partial sums of up to a few hundred workgroups added down the columns, gfx950.
//
// part is [groups][K][N] fp32; out[k][n] = sum over groups, always in the same order:
// 32 threads a column take every 32nd group each, then their sums are added one after the
// other.  Bound by the latency of its few loads; 32 columns a workgroup are whole 128-byte lines.
#include "kernels.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

template <typename T>
__global__ __launch_bounds__(1024) void column_sums(const float* part, int groups, int K, int N, T* out0, T* out1) {
    __shared__ float sums[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, k = blockIdx.y;
    const int n = blockIdx.x * 32 + c;
    T* out = k == 0 ? out0 : out1;
    if (!out) return;
    float t = 0.f;
    if (n < N) {
        const float* p = part + (int64_t)k * N + n;
        const int64_t step = (int64_t)K * N;
        int g = r;
        for (; g + 96 < groups; g += 128) {
            const float a = p[g * step], b = p[(g + 32) * step], d = p[(g + 64) * step], e = p[(g + 96) * step];
            t += a;
            t += b;
            t += d;
            t += e;
        }
        for (; g < groups; g += 32) t += p[g * step];
    }
    sums[r][c] = t;
    __syncthreads();
    if (r == 0 && n < N) {
#pragma unroll
        for (int i = 1; i < 32; ++i) t += sums[i][c];
        out[n] = (T)t;
    }
}

}  // namespace

hipError_t launch_column_sums(int f32, const float* part, int groups, int K, int N, void* out0, void* out1, hipStream_t s) {
    const dim3 grid((unsigned)((N + 31) / 32), (unsigned)K);
    if (f32)
        hipLaunchKernelGGL(column_sums<float>, grid, dim3(1024), 0, s, part, groups, K, N, (float*)out0, (float*)out1);
    else
        hipLaunchKernelGGL(column_sums<bf16>, grid, dim3(1024), 0, s, part, groups, K, N, (bf16*)out0, (bf16*)out1);
    return hipGetLastError();
}

}  // namespace fbl
