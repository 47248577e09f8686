// linear_finish.hip -- a linear layer's forward for a few tokens (serving), gfx950: what
// follows a product whose contraction several workgroups shared.
//   z = sum over the shares + bias,  y = act(z) + residual
// or, of the data gradient,  dx = (sum over the shares) act'(z)
//
// Such a layer is bound by reading w once, and its tiles alone have too few bytes on the way for that: the
// shares (launch_sum_gemm) give every CU two tiles' loads.  This adds their fp32 planes in order, a thread an
// element; they have just been written and are at most a few MB.
#include "act.hpp"
#include "kernels.hpp"

namespace fbl {

namespace {

template <typename T, int ACT, bool GRAD>
__global__ __launch_bounds__(256) void linear_finish(LinearArgs p, const float* planes, int splits) {
    const int n = blockIdx.x * 256 + threadIdx.x;
    const int64_t m = blockIdx.y, at = m * p.N + n, plane = (int64_t)p.M * p.N;
    if (n >= p.N) return;
    float z = 0.f;
    int i = 0;
    for (; i + 4 <= splits; i += 4) {
        const float a = planes[i * plane + at], b = planes[(i + 1) * plane + at], c = planes[(i + 2) * plane + at],
                    d = planes[(i + 3) * plane + at];
        z += a, z += b, z += c, z += d;
    }
    for (; i < splits; ++i) z += planes[i * plane + at];
    if constexpr (GRAD) {
        if constexpr (ACT != kActNone) z *= act_grad<ACT, sizeof(T) == 2>((float)static_cast<const T*>(p.z)[m * p.ldz + n]);
        static_cast<T*>(p.c)[m * p.ldc + n] = (T)z;
        if (p.sums) p.sums[at] = z;  // every row a block of its own
        return;
    }
    if (p.bias) z += (float)static_cast<const T*>(p.bias)[n];
    if (p.z) static_cast<T*>(p.z)[m * p.ldz + n] = (T)z;
    float y = act<ACT, sizeof(T) == 2>(z);
    if (p.res) y += (float)static_cast<const T*>(p.res)[m * p.ldr + n];
    static_cast<T*>(p.c)[m * p.ldc + n] = (T)y;
}

template <typename T, bool GRAD>
hipError_t finish(int act, const LinearArgs& p, const float* planes, int splits, hipStream_t s) {
    const dim3 grid((unsigned)((p.N + 255) / 256), (unsigned)p.M);
    switch (act) {
        case kActNone: hipLaunchKernelGGL((linear_finish<T, kActNone, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActRelu: hipLaunchKernelGGL((linear_finish<T, kActRelu, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActGelu: hipLaunchKernelGGL((linear_finish<T, kActGelu, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        case kActGeluTanh: hipLaunchKernelGGL((linear_finish<T, kActGeluTanh, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
        default: hipLaunchKernelGGL((linear_finish<T, kActSilu, GRAD>), grid, dim3(256), 0, s, p, planes, splits); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_finish(int f32, int act, int grad, const LinearArgs& p, const float* planes, int splits, hipStream_t s) {
    if (grad) return f32 ? finish<float, true>(act, p, planes, splits, s) : finish<bf16, true>(act, p, planes, splits, s);
    return f32 ? finish<float, false>(act, p, planes, splits, s) : finish<bf16, false>(act, p, planes, splits, s);
}

}  // namespace fbl
