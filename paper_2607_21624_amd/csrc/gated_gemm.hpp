// gated_gemm.hpp -- the matrix products of a gated layer with the activation and the product of its two halves in
// their epilogue, gfx950.  One translation unit per activation (gated_gemm_*.hip) defines FBL_ACT and
// includes this.
//
//   forward        z = X W + bias for W [K, 2F], gate then up columns;  h = act(gate) up   (z stored where the backward needs it)
//   data gradient  dh = dY Wd^T;  d gate = dh up act'(gate),  d up = dh act(gate)
//                  and their sums over a tile's rows, the bias' gradient
//
// The tile loops are those of the projection products.  A forward tile's columns are gate and up columns in turns of eight
// (EP::kPairs), so both projections are one product that reads X once, and the two factors of a value of h are
// registers of one lane (fp32: of two lanes in a row of 16).  The data gradient reads z beside a tile and writes both
// gradients; h's own is never stored.
#include "act.hpp"
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

template <int ACT, bool GRAD>
struct GatedEp {
    using Args = GatedArgs;
    static constexpr bool kByRows = true, kSplits = false, kPairs = !GRAD;

    // bf16: 8 columns of a row in a lane
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t lds, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rz = span(p.z, p.z_bytes);
        const int F = GRAD ? p.N : p.N / 2;
        const auto offset = [&](int m, int n, int64_t ld) __attribute__((always_inline)) {
            return m < p.M && n < F ? (uint32_t)(((int64_t)m * ld + n) * 2) : kNowhere;
        };
        const auto up_of = [&](uint32_t off) __attribute__((always_inline)) {
            return off == kNowhere ? kNowhere : off + (uint32_t)F * 2;
        };
        if constexpr (!GRAD) {
            const bool has_z = p.z != nullptr;
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
                float h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] += bg[e], u[e] += bu[e];
                if (has_z) {
                    store8(rz, offset(m, n, p.ldz), g, n, F);
                    store8(rz, up_of(offset(m, n, p.ldz)), u, n, F);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = act<ACT, true>(g[e]) * u[e];
                store8(rc, offset(m, n, p.ldc), h, n, F);
            });
        } else {
            struct Z {
                bf16x8 g, u;
            };
            float sg[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, su[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            by_rows<C>(
                lds, acc, m0, n0, wm, wn,
                [&](int m, int n) __attribute__((always_inline)) {
                    const uint32_t off = offset(m, n, p.ldz);
                    return Z{load8(rz, off), load8(rz, up_of(off))};
                },
                [&](int m, int n, float (&v)[8], const Z& z) __attribute__((always_inline)) {
                    float g[8], u[8];
                    const bool there = m < p.M;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        g[e] = v[e] * (float)z.u[e] * act_grad<ACT, true>((float)z.g[e]);
                        u[e] = v[e] * act<ACT, true>((float)z.g[e]);
                        sg[e] += there ? g[e] : 0.f;
                        su[e] += there ? u[e] : 0.f;
                    }
                    store8(rc, offset(m, n, p.ldc), g, n, F);
                    store8(rc, up_of(offset(m, n, p.ldc)), u, n, F);
                });
            if (!p.sums) return;
            constexpr int LANES = 4 * C::TN;
            const int nb = n0 + wn * C::TN * 32 + (threadIdx.x & 63) % LANES * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) sg[e] += __shfl_xor(sg[e], d), su[e] += __shfl_xor(su[e], d);
            }
            float* const out = p.sums + (int64_t)(m0 / C::BM * C::WM + wm) * 2 * F + nb;
            if ((threadIdx.x & 63) < LANES && nb < F) {  // F is a multiple of 8
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    *reinterpret_cast<f32x4*>(out + 4 * h) = f32x4{sg[4 * h], sg[4 * h + 1], sg[4 * h + 2], sg[4 * h + 3]};
                    *reinterpret_cast<f32x4*>(out + F + 4 * h) = f32x4{su[4 * h], su[4 * h + 1], su[4 * h + 2], su[4 * h + 3]};
                }
            }
        }
    }

    // fp32: a column of the tile in a lane, 32 of them across a half
    template <typename C>
    static FBL_DEV void done(const Args& p, float*, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        const int lane = threadIdx.x & 63, g = lane >> 5;
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rz = span(p.z, p.z_bytes);
        const auto load = [](__amdgpu_buffer_rsrc_t r, uint32_t off) __attribute__((always_inline)) {
            return __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
        };
        const auto store = [](__amdgpu_buffer_rsrc_t r, uint32_t off, float v) __attribute__((always_inline)) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(v), r, off, 0, 0);
        };
        if constexpr (!GRAD) {
            const __amdgpu_buffer_rsrc_t rb = span(p.bias, (uint32_t)p.N * 4);
            const int F = p.N / 2, up = lane >> 3 & 1;  // which of the two matrices the lane's column is of
            const bool has_z = p.z != nullptr;
#pragma unroll
            for (int tn = 0; tn < C::TN; ++tn) {
                const int n = n0 / 2 + (wn * C::TN + tn) * 16 + (lane >> 4 & 1) * 8 + (lane & 7);
                const float b = load(rb, n < F ? (uint32_t)(up * F + n) * 4 : kNowhere);
#pragma unroll
                for (int tm = 0; tm < C::TM; ++tm) {
                    const auto offset = [&](int r, int64_t ld, int col) __attribute__((always_inline)) {
                        const int m = m0 + (wm * C::TM + tm) * 32 + acc_row(r, g);
                        return m < p.M && n < F ? (uint32_t)(((int64_t)m * ld + col) * 4) : kNowhere;
                    };
                    f32x16& v = acc[tm][tn];
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        v[r] += b;
                        if (has_z) store(rz, offset(r, p.ldz, up * F + n), v[r]);
                    }
                    // the pair of lanes shares its 16 rows: the gate's lane makes h in the first eight, the other in the rest
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const float other = dpp<0x128>(up ? v[r] : v[r + 8]);  // row_ror 8: from eight lanes on
                        const float gate = up ? other : v[r], x = up ? v[r + 8] : other;
                        store(rc, up ? offset(r + 8, p.ldc, n) : offset(r, p.ldc, n), act<ACT, false>(gate) * x);
                    }
                }
            }
        } else {
            const int F = p.N;
#pragma unroll
            for (int tn = 0; tn < C::TN; ++tn) {
                const int n = n0 + (wn * C::TN + tn) * 32 + (lane & 31);
                float sg = 0.f, su = 0.f;
#pragma unroll
                for (int tm = 0; tm < C::TM; ++tm) {
                    const auto offset = [&](int r, int64_t ld, int col) __attribute__((always_inline)) {
                        const int m = m0 + (wm * C::TM + tm) * 32 + acc_row(r, g);
                        return m < p.M && n < F ? (uint32_t)(((int64_t)m * ld + col) * 4) : kNowhere;
                    };
                    float zg[16], zu[16];  // all on the way before the first store
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        zg[r] = load(rz, offset(r, p.ldz, n)), zu[r] = load(rz, offset(r, p.ldz, F + n));
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float v = acc[tm][tn][r], dg = v * zu[r] * act_grad<ACT, false>(zg[r]),
                                    du = v * act<ACT, false>(zg[r]);
                        const bool there = offset(r, 0, 0) != kNowhere;
                        sg += there ? dg : 0.f;
                        su += there ? du : 0.f;
                        store(rc, offset(r, p.ldc, n), dg);
                        store(rc, offset(r, p.ldc, F + n), du);
                    }
                }
                sg += other_half(sg);
                su += other_half(su);
                if (p.sums && g == 0 && n < F) {
                    float* const out = p.sums + (int64_t)(m0 / C::t.bm * C::t.wm + wm) * 2 * F + n;
                    out[0] = sg;
                    out[F] = su;
                }
            }
        }
    }
};

}  // namespace

template <>
hipError_t launch_gated_gemm<FBL_ACT>(int grad, int tile, const GatedArgs& p, hipStream_t stream) {
    if (grad) return launch_gemm_tile<false, true, GatedEp<FBL_ACT, true>>(tile, p, stream);
    return launch_gemm_tile<false, false, GatedEp<FBL_ACT, false>>(tile, p, stream);
}

template <>
hipError_t launch_gated_gemm_f32<FBL_ACT>(int grad, const GatedArgs& p, hipStream_t stream) {
    if (grad) return launch_f32_tile<false, true, GatedEp<FBL_ACT, true>>(f32_tile(p), p, stream);
    return launch_f32_tile<false, false, GatedEp<FBL_ACT, false>>(f32_tile(p), p, stream);
}

}  // namespace fbl
