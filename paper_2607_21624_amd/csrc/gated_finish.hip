// gated_finish.hip -- a gated layer's forward for a few tokens (serving), gfx950: what follows the product
// whose contraction several workgroups shared.
//   (gate, up) = sum over the shares + bias,  h = act(gate) up  and the factors of h's gradient
// or, of the data gradient,  dh = sum over the shares,  dz = dh times the factors
//
// As linear_finish.hip: the fp32 planes, just written and a few MB at most, are added in order, a thread a
// column of h.
#include "act.hpp"
#include "factors.hpp"
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

template <typename T, int ACT>
__global__ __launch_bounds__(256) void gated_finish(GatedArgs p, const float* planes, int splits) {
    constexpr bool FAST = sizeof(T) == 2;
    const int n = blockIdx.x * 256 + threadIdx.x, F = p.N / 2;
    const int64_t m = blockIdx.y, plane = (int64_t)p.M * p.N, at = m * p.N + n;
    if (n >= F) return;
    float gate = plane_sum(planes, at, plane, splits), up = plane_sum(planes, at + F, plane, splits);
    if (p.bias) gate += (float)static_cast<const T*>(p.bias)[n], up += (float)static_cast<const T*>(p.bias)[F + n];
    const float a = act<ACT, FAST>(gate);
    if (p.factors) {
        const float d = up * act_grad<ACT, FAST>(gate);
        if constexpr (FAST) {  // F is a multiple of 8: eight lanes are there or none
            uint16_t* const f = static_cast<uint16_t*>(p.factors) + m * p.ldf + n;
            f[0] = pack_factor(d);
            f[F] = pack_factor(a);
        } else {
            T* const f = static_cast<T*>(p.factors) + m * p.ldf + n;
            f[0] = d;
            f[F] = a;
        }
    }
    static_cast<T*>(p.c)[m * p.ldc + n] = (T)(a * up);
}

template <typename T>
__global__ __launch_bounds__(256) void gated_grad_finish(GatedArgs p, const float* planes, int splits) {
    const int n = blockIdx.x * 256 + threadIdx.x, F = p.N;
    const int64_t m = blockIdx.y, at = m * F + n;
    if (n >= F) return;
    const float v = plane_sum(planes, at, (int64_t)p.M * F, splits);
    float dg, du;
    if constexpr (sizeof(T) == 2) {
        const uint16_t* const f = static_cast<const uint16_t*>(p.factors) + m * p.ldf + n;
        dg = v * unpack_factor(f[0]), du = v * unpack_factor(f[F]);
    } else {
        const T* const f = static_cast<const T*>(p.factors) + m * p.ldf + n;
        dg = v * f[0], du = v * f[F];
    }
    T* const c = static_cast<T*>(p.c) + m * p.ldc + n;
    c[0] = (T)dg;
    c[F] = (T)du;
    if (p.sums) {  // every row a block of its own
        p.sums[m * 2 * F + n] = dg;
        p.sums[m * 2 * F + F + n] = du;
    }
}

template <typename T>
hipError_t finish(int act, const GatedArgs& p, const float* planes, int splits, hipStream_t s) {
    const dim3 grid((unsigned)((p.N / 2 + 255) / 256), (unsigned)p.M);
    switch (act) {
        case kActNone: hipLaunchKernelGGL((gated_finish<T, kActNone>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActRelu: hipLaunchKernelGGL((gated_finish<T, kActRelu>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActGelu: hipLaunchKernelGGL((gated_finish<T, kActGelu>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActGeluTanh: hipLaunchKernelGGL((gated_finish<T, kActGeluTanh>), grid, dim3(256), 0, s, p, planes, splits); break;
        default: hipLaunchKernelGGL((gated_finish<T, kActSilu>), grid, dim3(256), 0, s, p, planes, splits); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gated_finish(int f32, int act, const GatedArgs& p, const float* planes, int splits, hipStream_t s) {
    return f32 ? finish<float>(act, p, planes, splits, s) : finish<bf16>(act, p, planes, splits, s);
}

hipError_t launch_gated_grad_finish(int f32, const GatedArgs& p, const float* planes, int splits, hipStream_t s) {
    const dim3 grid((unsigned)((p.N + 255) / 256), (unsigned)p.M);
    if (f32) hipLaunchKernelGGL(gated_grad_finish<float>, grid, dim3(256), 0, s, p, planes, splits);
    else hipLaunchKernelGGL(gated_grad_finish<bf16>, grid, dim3(256), 0, s, p, planes, splits);
    return hipGetLastError();
}

}  // namespace fbl
