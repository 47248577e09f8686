// linear_act.hip -- the elementwise half of a linear layer's backward, gfx950:
//   dz = dy act'(z),  and the bias' gradient, the sum of dz down its rows.
//
// Bound by memory: dy and z are read and dz is written once.  A workgroup's four
// wavefronts take every fourth row of a block of rows, each 64 chunks of 16 bytes wide;
// the sums stay in registers over the block, are added through LDS and go out as one row of
// partial sums, which column_sums adds in a fixed order.  Without an activation dz is dy and
// only the sums are made.
#include "act.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

template <typename T, int ACT>
__global__ __launch_bounds__(256) void linear_act_bwd(LinearActArgs a) {
    using P = Pack<T>;
    constexpr int V = P::N;
    __shared__ float sums[4][64 * V];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int col = (blockIdx.x * 64 + l) * V;
    const int64_t m0 = (int64_t)blockIdx.y * a.rows, m1 = min(a.M, m0 + a.rows);
    float s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
    if (col < a.N) {
        for (int64_t m = m0 + w; m < m1; m += 4) {
            P d, z;
            d.load(static_cast<const T*>(a.dy) + m * a.lddy, col, a.N);
            if constexpr (ACT != kActNone) {
                z.load(static_cast<const T*>(a.z) + m * a.ldz, col, a.N);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float v = d[e] * act_grad<ACT, sizeof(T) == 2>(z[e]);
                    d.set(e, v);
                    s[e] += v;
                }
                d.store(static_cast<T*>(a.dz) + m * a.lddz, col, a.N);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) s[e] += d[e];
            }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) sums[w][l * V + e] = s[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * V; i += 256) {
        const int n = blockIdx.x * 64 * V + i;
        if (n < a.N) a.part[(int64_t)blockIdx.y * a.N + n] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    }
}

template <typename T>
hipError_t launch(int act, const LinearActArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.N + 64 * Pack<T>::N - 1) / (64 * Pack<T>::N)), (unsigned)a.groups);
    switch (act) {
        case kActNone: hipLaunchKernelGGL((linear_act_bwd<T, kActNone>), grid, dim3(256), 0, s, a); break;
        case kActRelu: hipLaunchKernelGGL((linear_act_bwd<T, kActRelu>), grid, dim3(256), 0, s, a); break;
        case kActGelu: hipLaunchKernelGGL((linear_act_bwd<T, kActGelu>), grid, dim3(256), 0, s, a); break;
        case kActGeluTanh: hipLaunchKernelGGL((linear_act_bwd<T, kActGeluTanh>), grid, dim3(256), 0, s, a); break;
        default: hipLaunchKernelGGL((linear_act_bwd<T, kActSilu>), grid, dim3(256), 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_act_bwd(int f32, int act, const LinearActArgs& a, hipStream_t s) {
    return f32 ? launch<float>(act, a, s) : launch<bf16>(act, a, s);
}

}  // namespace fbl
