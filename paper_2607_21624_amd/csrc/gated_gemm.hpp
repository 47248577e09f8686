// gated_gemm.hpp -- a gated layer's forward product with the activation and the product of its two halves in
// its epilogue, gfx950.  One translation unit per activation (gated_gemm_*.hip) defines FBL_ACT and
// includes this.
//
//   (gate, up) = X W + bias for W [K, 2F], gate then up columns;  h = act(gate) up
//   and where the backward needs them the factors  d h / d gate = up act'(gate),  d h / d up = act(gate)
//
// The tile loops are those of the projection products.  A tile's columns are gate and up columns in turns of eight
// (EP::kPairs), so both projections are one product that reads X once, and the gate and up of a value of h are
// registers of one lane (fp32: of two lanes in a row of 16).
//
// The factors are kept, and not gate and up: they are as many bytes, and the backward (gated_grad.hip) is then one kernel
// for all activations that multiplies (4096 tokens 4096 -> 11008: 391 -> 381 us).  The derivative costs the forward a few
// operations beside an exponential that it makes anyway.  bf16 dx and dw of a step are off by 0.24% of their norm: the
// roundings of dz, which the matrix instructions take in bf16, and of the result, 0.17% each.  Factors in bf16 added as much
// (0.29%; rounded gate and up 0.30%), so they are kept in as many bytes of a form with 11 digits (factors.hpp).
//
// 4096 tokens bf16 with factors, one call after another: 2048 -> 8192 248 us (1.11 PFLOP/s), 4096 -> 11008 708 us (1.04), without
// any 229 and 672; within a step, behind the backward of the one before, medians of 271 and 736.  fp32, 2048 tokens 1024 -> 4096 277 us
// (124 TFLOP/s), without factors 269; one token of 2048 -> 8192, cold weights, 30.
// The plain products of the same bf16 sizes, stored by the lanes as the accumulators lie, took 296 and 711 (with factors 264 and 720
// at that time).
#include "act.hpp"
#include "factors.hpp"
#include "gemm_bf16.hpp"
#include "gemm_f32.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

// A wavefront's accumulators of pairs by rows, as by_rows (gemm_bf16.hpp): f(m, n, g, u) gets 8 columns n .. of row m
// of both matrices.
template <typename C, typename F>
FBL_DEV void by_pairs(uint32_t lds, const f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn, F&& f) {
    constexpr int PITCH = 32 * C::TN + 4, LANES = 2 * C::TN, ROWS = 64 / LANES;  // lanes a row, rows a turn
    const int lane = threadIdx.x & 63, g = lane >> 5;
    const uint32_t mine = lds + (uint32_t)((wn * C::WM + wm) * 32 * PITCH * 4);
    const uint32_t put = mine + (uint32_t)(((lane & 31) * PITCH + 4 * g) * 4);
    const uint32_t get = mine + (uint32_t)((lane / LANES * PITCH + lane % LANES * 16) * 4);
    __syncthreads();  // the stages have been read
    const int nl = n0 / 2 + wn * C::TN * 16 + lane % LANES * 8, ml = m0 + wm * C::TM * 32 + lane / LANES;
#pragma unroll
    for (int tm = 0; tm < C::TM; ++tm) {
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(FBL_LDS f32x4*)(uintptr_t)(put + (tn * 32 + 8 * q) * 4) =
                    f32x4{acc[tn][tm][4 * q], acc[tn][tm][4 * q + 1], acc[tn][tm][4 * q + 2], acc[tn][tm][4 * q + 3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) {
            float x[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 a = *(const FBL_LDS f32x4*)(uintptr_t)(get + i * ROWS * PITCH * 4 + q * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * q + e] = a[e];
            }
            f(ml + 32 * tm + i * ROWS, nl, *(float(*)[8])(x), *(float(*)[8])(x + 8));
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

template <int ACT>
struct GatedEp {
    using Args = GatedArgs;
    static constexpr bool kByRows = true, kSplits = false, kPairs = true;

    // bf16: 8 columns of a row in a lane
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t lds, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rf = span(p.factors, p.f_bytes);
        const int F = p.N / 2;
        const auto offset = [&](int m, int n, int64_t ld) __attribute__((always_inline)) {
            return m < p.M && n < F ? (uint32_t)(((int64_t)m * ld + n) * 2) : kNowhere;
        };
        const auto up_of = [&](uint32_t off) __attribute__((always_inline)) {
            return off == kNowhere ? kNowhere : off + (uint32_t)F * 2;
        };
        const bool keep = p.factors != nullptr;
        constexpr int LANES = 2 * C::TN;
        const int nb = n0 / 2 + wn * C::TN * 16 + (threadIdx.x & 63) % LANES * 8;  // every turn is at the same columns
        float bg[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bu[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (p.bias) {
            const __amdgpu_buffer_rsrc_t rb = span(p.bias, (uint32_t)p.N * 2);
            const bf16x8 x = load8(rb, offset(0, nb, 0)), y = load8(rb, up_of(offset(0, nb, 0)));
#pragma unroll
            for (int e = 0; e < 8; ++e) bg[e] = (float)x[e], bu[e] = (float)y[e];
        }
        by_pairs<C>(lds, acc, m0, n0, wm, wn, [&](int m, int n, float (&g)[8], float (&u)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] += bg[e], u[e] += bu[e];
            float a[8], h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = act<ACT, true>(g[e]), h[e] = a[e] * u[e];
            if (keep) {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = u[e] * act_grad<ACT, true>(g[e]);
                const uint32_t off = offset(m, n, p.ldf);  // F is a multiple of 8
                __builtin_amdgcn_raw_buffer_store_b128(pack_factors(g), rf, off, 0, kOnce);
                __builtin_amdgcn_raw_buffer_store_b128(pack_factors(a), rf, up_of(off), 0, kOnce);
            }
            store8(rc, offset(m, n, p.ldc), h, n, F);
        });
    }

    // fp32: a column of the tile in a lane, 32 of them across a half
    template <typename C>
    static FBL_DEV void done(const Args& p, float*, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        const int lane = threadIdx.x & 63, g = lane >> 5;
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rf = span(p.factors, p.f_bytes),
                                     rb = span(p.bias, (uint32_t)p.N * 4);
        const auto store = [](__amdgpu_buffer_rsrc_t r, uint32_t off, float v) __attribute__((always_inline)) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(v), r, off, 0, 0);
        };
        const int F = p.N / 2, up = lane >> 3 & 1;  // which of the two matrices the lane's column is of
        const bool keep = p.factors != nullptr;
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn) {
            const int n = n0 / 2 + (wn * C::TN + tn) * 16 + (lane >> 4 & 1) * 8 + (lane & 7);
            const float b = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rb, n < F ? (uint32_t)(up * F + n) * 4 : kNowhere, 0, 0));
#pragma unroll
            for (int tm = 0; tm < C::TM; ++tm) {
                const auto offset = [&](int r, int64_t ld, int col) __attribute__((always_inline)) {
                    const int m = m0 + (wm * C::TM + tm) * 32 + acc_row(r, g);
                    return m < p.M && n < F ? (uint32_t)(((int64_t)m * ld + col) * 4) : kNowhere;
                };
                f32x16& v = acc[tm][tn];
#pragma unroll
                for (int r = 0; r < 16; ++r) v[r] += b;
                // the pair of lanes shares its 16 rows: the gate's lane makes the first eight, the other the rest
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float other = dpp<0x128>(up ? v[r] : v[r + 8]);  // row_ror 8: from eight lanes on
                    const float gate = up ? other : v[r], x = up ? v[r + 8] : other, a = act<ACT, false>(gate);
                    const auto at = [&](int64_t ld, int col) __attribute__((always_inline)) {
                        return up ? offset(r + 8, ld, col) : offset(r, ld, col);
                    };
                    if (keep) {
                        store(rf, at(p.ldf, n), x * act_grad<ACT, false>(gate));
                        store(rf, at(p.ldf, F + n), a);
                    }
                    store(rc, at(p.ldc, n), a * x);
                }
            }
        }
    }
};

}  // namespace

template <>
hipError_t launch_gated_gemm<FBL_ACT>(int tile, const GatedArgs& p, hipStream_t stream) {
    return launch_gemm_tile<false, false, GatedEp<FBL_ACT>>(tile, p, stream);
}

template <>
hipError_t launch_gated_gemm_f32<FBL_ACT>(const GatedArgs& p, hipStream_t stream) {
    return launch_f32_tile<false, false, GatedEp<FBL_ACT>>(f32_tile(p), p, stream);
}

}  // namespace fbl
