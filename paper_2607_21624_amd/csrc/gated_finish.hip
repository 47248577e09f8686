// gated_finish.hip -- a gated layer's forward for a few tokens (serving), gfx950: what follows the product
// whose contraction several workgroups shared.
//   z = sum over the shares + bias,  h = act(gate) up
// or, of the data gradient,  dh = sum over the shares,  d gate = dh up act'(gate),  d up = dh act(gate)
//
// As linear_finish.hip: the fp32 planes, just written and a few MB at most, are added in order, a thread a
// column of h.
#include "act.hpp"
#include "kernels.hpp"

namespace fbl {

namespace {

FBL_DEV float plane_sum(const float* planes, int64_t at, int64_t plane, int splits) {
    float z = 0.f;
    int i = 0;
    for (; i + 4 <= splits; i += 4) {
        const float a = planes[i * plane + at], b = planes[(i + 1) * plane + at], c = planes[(i + 2) * plane + at],
                    d = planes[(i + 3) * plane + at];
        z += a, z += b, z += c, z += d;
    }
    for (; i < splits; ++i) z += planes[i * plane + at];
    return z;
}

template <typename T, int ACT, bool GRAD>
__global__ __launch_bounds__(256) void gated_finish(GatedArgs p, const float* planes, int splits) {
    constexpr bool FAST = sizeof(T) == 2;
    const int n = blockIdx.x * 256 + threadIdx.x, F = GRAD ? p.N : p.N / 2;
    const int64_t m = blockIdx.y, plane = (int64_t)p.M * p.N, at = m * p.N + n;
    if (n >= F) return;
    T* const z = static_cast<T*>(p.z);
    T* const c = static_cast<T*>(p.c) + m * p.ldc + n;
    if constexpr (GRAD) {
        const float v = plane_sum(planes, at, plane, splits), gate = (float)z[m * p.ldz + n], up = (float)z[m * p.ldz + F + n];
        const float dg = v * up * act_grad<ACT, FAST>(gate), du = v * act<ACT, FAST>(gate);
        c[0] = (T)dg;
        c[F] = (T)du;
        if (p.sums) {  // every row a block of its own
            p.sums[m * 2 * F + n] = dg;
            p.sums[m * 2 * F + F + n] = du;
        }
    } else {
        float gate = plane_sum(planes, at, plane, splits), up = plane_sum(planes, at + F, plane, splits);
        if (p.bias) gate += (float)static_cast<const T*>(p.bias)[n], up += (float)static_cast<const T*>(p.bias)[F + n];
        if (z) z[m * p.ldz + n] = (T)gate, z[m * p.ldz + F + n] = (T)up;
        c[0] = (T)(act<ACT, FAST>(gate) * up);
    }
}

template <typename T, bool GRAD>
hipError_t finish(int act, const GatedArgs& p, const float* planes, int splits, hipStream_t s) {
    const int F = GRAD ? p.N : p.N / 2;
    const dim3 grid((unsigned)((F + 255) / 256), (unsigned)p.M);
    switch (act) {
        case kActNone: hipLaunchKernelGGL((gated_finish<T, kActNone, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActRelu: hipLaunchKernelGGL((gated_finish<T, kActRelu, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActGelu: hipLaunchKernelGGL((gated_finish<T, kActGelu, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActGeluTanh: hipLaunchKernelGGL((gated_finish<T, kActGeluTanh, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        default: hipLaunchKernelGGL((gated_finish<T, kActSilu, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gated_finish(int f32, int act, int grad, const GatedArgs& p, const float* planes, int splits, hipStream_t s) {
    if (grad) return f32 ? finish<float, true>(act, p, planes, splits, s) : finish<bf16, true>(act, p, planes, splits, s);
    return f32 ? finish<float, false>(act, p, planes, splits, s) : finish<bf16, false>(act, p, planes, splits, s);
}

}  // namespace fbl
