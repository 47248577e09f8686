// act.hpp -- the activations of a linear layer and their derivatives (device).
//
// Each comes in two grades.  fp32 storage calls the library's erf, exp and tanh.  bf16
// storage, whose results keep 8 bits, takes the hardware's exp2 and reciprocal (1 ulp) and for
// the normal distribution function a polynomial that is good to 2.2e-7 and, in the negative tail where GELU's
// values are small but not 0, to 8e-5 of its value, a twentieth of a rounding: a
// wavefront's share of a 256 x 256 tile has 128 values a lane and nothing beside it to hide
// them behind.
#pragma once

#include "cdna4.hpp"

namespace fbl {

enum Act { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

constexpr float kGeluC = 0.7978845608028654f;  // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

// Phi(z), the normal distribution function, and e = exp(-z^2 / 2):
// 1 - Phi(|z|) = e/2 (a1 t + .. + a6 t^6), t = 1 / (1 + p |z|).
// (p and the a's: the least largest error over 0 <= |z| <= 14, weighted 1e-7 where the tail is large and 1.2e-4 of it
// where it is small, by iterated least squares.  With five a's fitted to the error alone, as in Abramowitz and
// Stegun's 7.1.26, t falls off by another factor than the tail does: 0.05% at z = -4, 0.36% at -6, 3.7% at -13.
// The sixth costs 0.9 us of 137, 4096 x 8192 from 2048 with z stored.)
FBL_DEV float normal_cdf(float z, float& e) {
    const float x = __builtin_fabsf(z);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.292f, x, 1.f));
    e = fast_exp2(z * z * (-0.5f * kLog2e));
    float s = __builtin_fmaf(-0.173455447f, t, 0.541312450f);
    s = __builtin_fmaf(s, t, -0.152120707f);
    s = __builtin_fmaf(s, t, 0.341441498f);
    s = __builtin_fmaf(s, t, 0.207963596f);
    s = __builtin_fmaf(s, t, 0.234858490f);
    const float tail = 0.5f * e * s * t;
    return z < 0.f ? tail : 1.f - tail;
}

FBL_DEV float fast_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * z)); }

template <int ACT, bool FAST>
FBL_DEV float act(float z) {
    if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;
    if constexpr (ACT == kActGelu) {
        if constexpr (FAST) {
            float e;
            return z * normal_cdf(z, e);
        } else {
            return 0.5f * z * (1.f + erff(z * 0.7071067811865476f));
        }
    }
    if constexpr (ACT == kActGeluTanh) {
        const float u = kGeluC * z * __builtin_fmaf(kGeluA, z * z, 1.f);
        if constexpr (FAST) return z * fast_sigmoid(2.f * u);
        return 0.5f * z * (1.f + tanhf(u));
    }
    if constexpr (ACT == kActSilu) return FAST ? z * fast_sigmoid(z) : z / (1.f + expf(-z));
    return z;
}

template <int ACT, bool FAST>
FBL_DEV float act_grad(float z) {
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : 0.f;
    if constexpr (ACT == kActGelu) {
        if constexpr (FAST) {
            float e;
            const float c = normal_cdf(z, e);
            return __builtin_fmaf(z * 0.3989422804014327f, e, c);
        } else {
            return 0.5f * (1.f + erff(z * 0.7071067811865476f)) + z * 0.3989422804014327f * expf(-0.5f * z * z);
        }
    }
    if constexpr (ACT == kActGeluTanh) {
        const float zz = z * z, u = kGeluC * z * __builtin_fmaf(kGeluA, zz, 1.f);
        const float du = kGeluC * __builtin_fmaf(3.f * kGeluA, zz, 1.f);
        if constexpr (FAST) {
            const float s = fast_sigmoid(2.f * u);
            return __builtin_fmaf(2.f * z * du, s * (1.f - s), s);
        } else {
            const float t = tanhf(u);
            return 0.5f * (1.f + t) + 0.5f * z * (1.f - t * t) * du;
        }
    }
    if constexpr (ACT == kActSilu) {
        const float s = FAST ? fast_sigmoid(z) : 1.f / (1.f + expf(-z));
        return __builtin_fmaf(z * s, 1.f - s, s);
    }
    return 1.f;
}

}  // namespace fbl
