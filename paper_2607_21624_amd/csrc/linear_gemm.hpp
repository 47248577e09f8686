// linear_gemm.hpp -- the matrix products of a linear layer with its bias, activation
// and residual in their epilogue, and the data gradient times the previous layer's
// activation derivative, gfx950.  One translation unit per activation
// (linear_gemm_*.hip) defines FBL_ACT and includes this.
//
//   forward        z = X W + bias;  y = act(z) + residual   (z stored too where the backward needs it)
//   data gradient  dX = (dZ W^T) act'(zp)                   (zp: the layer before's z)
//                  and the sums of dX's columns over a tile's rows, that layer's bias gradient
//
// The tile loops are those of the projection products; the epilogue works on the
// accumulators where they are, so the layer writes y once and reads nothing back: a
// separate pass over y would cost 2 to 3 times its bytes again.  The sums of dX are taken here, unrounded, for the same
// reason (4096 x 8192: a pass over dX 13 us).  bf16: the sums stay in
// fp32 up to the one rounding of y and of z each.
#include "act.hpp"
#include "gemm_bf16.hpp"
#include "gemm_f32.hpp"

namespace fbl {

namespace {

template <int ACT, bool GRAD>
struct LinearEp {
    using Args = LinearArgs;
    static constexpr bool kByRows = true, kSplits = false;

    // bf16: 8 columns of a row in a lane
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t lds, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rz = span(p.z, p.z_bytes), rr = span(p.res, p.res_bytes);
        const bool has_res = p.res != nullptr, has_z = p.z != nullptr;
        // every turn is at the same columns
        constexpr int LANES = 4 * C::TN;
        const int nb = n0 + wn * C::TN * 32 + (threadIdx.x & 63) % LANES * 8;
        float b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (!GRAD && p.bias) {
            const bf16x8 x = load8(span(p.bias, (uint32_t)p.N * 2), (uint32_t)nb * 2);  // past N: 0
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = (float)x[e];
        }
        const auto offset = [&](int m, int n, int64_t ld) __attribute__((always_inline)) {
            return m < p.M && n < p.N ? (uint32_t)(((int64_t)m * ld + n) * 2) : kNowhere;
        };
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};  // of the lane's columns over its rows
        const auto rows = [&](auto&& ahead, auto&& beside) __attribute__((always_inline)) {
            by_rows<C>(lds, acc, m0, n0, wm, wn, ahead, [&](int m, int n, float (&v)[8], const auto& x) __attribute__((always_inline)) {
                if constexpr (!GRAD) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += b[e];
                    if (has_z) store8(rz, offset(m, n, p.ldz), v, n, p.N);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = act<ACT, true>(v[e]);
                }
                beside(v, x);
                if constexpr (GRAD) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += m < p.M ? v[e] : 0.f;
                }
                store8(rc, offset(m, n, p.ldc), v, n, p.N);
            });
        };
        if constexpr (GRAD && ACT != kActNone) {
            rows([&](int m, int n) __attribute__((always_inline)) { return load8(rz, offset(m, n, p.ldz)); },
                 [](float (&v)[8], const bf16x8& z) __attribute__((always_inline)) {
#pragma unroll
                     for (int e = 0; e < 8; ++e) v[e] *= act_grad<ACT, true>((float)z[e]);
                 });
        } else if (!GRAD && has_res) {
            rows([&](int m, int n) __attribute__((always_inline)) { return load8(rr, offset(m, n, p.ldr)); },
                 [](float (&v)[8], const bf16x8& x) __attribute__((always_inline)) {
#pragma unroll
                     for (int e = 0; e < 8; ++e) v[e] += (float)x[e];
                 });
        } else {
            rows([](int, int) __attribute__((always_inline)) { return Nothing{}; },
                 [](float (&)[8], Nothing) __attribute__((always_inline)) {});
        }
        if constexpr (GRAD) {
            if (!p.sums) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) s[e] += __shfl_xor(s[e], d);
            }
            float* const out = p.sums + (int64_t)(m0 / C::BM * C::WM + wm) * p.N + nb;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if ((threadIdx.x & 63) < LANES && nb + 4 * h < p.N)  // N is a multiple of 4
                    *reinterpret_cast<f32x4*>(out + 4 * h) = f32x4{s[4 * h], s[4 * h + 1], s[4 * h + 2], s[4 * h + 3]};
        }
    }

    // fp32: 32 consecutive columns of a row across the lanes of a half
    template <typename C>
    static FBL_DEV void done(const Args& p, float*, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        const int lane = threadIdx.x & 63, g = lane >> 5;
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rz = span(p.z, p.z_bytes), rr = span(p.res, p.res_bytes),
                                     rb = span(p.bias, (uint32_t)p.N * 4);
        const auto load = [](__amdgpu_buffer_rsrc_t r, uint32_t off) __attribute__((always_inline)) {
            return __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
        };
        const bool has_res = p.res != nullptr, has_z = p.z != nullptr;
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn) {
            const int n = n0 + (wn * C::TN + tn) * 32 + (lane & 31);
            const float b = GRAD ? 0.f : load(rb, n < p.N ? (uint32_t)n * 4 : kNowhere);
            float s = 0.f;
#pragma unroll
            for (int tm = 0; tm < C::TM; ++tm) {
                const auto offset = [&](int r, int64_t ld) __attribute__((always_inline)) {
                    const int m = m0 + (wm * C::TM + tm) * 32 + acc_row(r, g);
                    return m < p.M && n < p.N ? (uint32_t)(((int64_t)m * ld + n) * 4) : kNowhere;
                };
                float x[16];  // z of the layer before, or the residual: all on the way before the first store
                if (GRAD ? ACT != kActNone : has_res) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[r] = GRAD ? load(rz, offset(r, p.ldz)) : load(rr, offset(r, p.ldr));
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float v = acc[tm][tn][r];
                    if constexpr (GRAD) {
                        if constexpr (ACT != kActNone) v *= act_grad<ACT, false>(x[r]);
                        s += offset(r, 0) != kNowhere ? v : 0.f;
                    } else {
                        v += b;
                        if (has_z) __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(v), rz, offset(r, p.ldz), 0, 0);
                        v = act<ACT, false>(v);
                        if (has_res) v += x[r];
                    }
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(v), rc, offset(r, p.ldc), 0, 0);
                }
            }
            if constexpr (GRAD) {
                s += other_half(s);
                if (p.sums && g == 0 && n < p.N) p.sums[(int64_t)(m0 / C::t.bm * C::t.wm + wm) * p.N + n] = s;
            }
        }
    }
};

}  // namespace

template <>
hipError_t launch_linear_gemm<FBL_ACT>(int grad, int tile, const LinearArgs& p, hipStream_t stream) {
    if (grad) return launch_gemm_tile<false, true, LinearEp<FBL_ACT, true>>(tile, p, stream);
    return launch_gemm_tile<false, false, LinearEp<FBL_ACT, false>>(tile, p, stream);
}

#if FBL_ACT == 0
int64_t linear_grad_groups(int f32, int tile, const GemmArgs& p) {
    if (f32) {
        const F32Tile& t = kF32Tiles[f32_tile(p)];
        return ((int64_t)p.M + t.bm - 1) / t.bm * t.wm;
    }
    const GemmTile& t = kGemmTiles[tile];
    return ((int64_t)p.M + t.bm - 1) / t.bm * t.wm;
}

// A weight gradient, its tiles written by rows.
hipError_t launch_weight_gemm(int tile, const LinearArgs& p, hipStream_t stream) {
    return launch_gemm_tile<true, false, LinearEp<kActNone, false>>(tile, p, stream);
}
#endif

template <>
hipError_t launch_linear_gemm_f32<FBL_ACT>(int grad, const LinearArgs& p, hipStream_t stream) {
    if (grad) return launch_f32_tile<false, true, LinearEp<FBL_ACT, true>>(f32_tile(p), p, stream);
    return launch_f32_tile<false, false, LinearEp<FBL_ACT, false>>(f32_tile(p), p, stream);
}

}  // namespace fbl
