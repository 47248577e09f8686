// gated_grad.hip -- the data gradient of a gated feed-forward part through its second projection, with what
// follows in its epilogue, gfx950:
//   dh = dY Wd^T;  dz = (dh f_gate, dh f_up)  by the factors that the forward kept (gated_gemm.hpp, factors.hpp)
//   and the sums of dz over a tile's rows, the bias' gradient
//
// A tile reads its factors and writes both halves of dz, in whole lines by rows (by_rows); dh is never stored.  Without
// that its memory traffic would be 7 values for each of dh's instead of 4.  The sums are of dz unrounded.
#include "factors.hpp"
#include "gemm_bf16.hpp"
#include "gemm_f32.hpp"

namespace fbl {

namespace {

struct GatedGradEp {
    using Args = GatedArgs;
    static constexpr bool kByRows = true, kSplits = false;

    // bf16: 8 columns of a row in a lane
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t lds, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rf = span(p.factors, p.f_bytes);
        const int F = p.N;
        const auto offset = [&](int m, int n, int64_t ld) __attribute__((always_inline)) {
            return m < p.M && n < F ? (uint32_t)(((int64_t)m * ld + n) * 2) : kNowhere;
        };
        const auto up_of = [&](uint32_t off) __attribute__((always_inline)) {
            return off == kNowhere ? kNowhere : off + (uint32_t)F * 2;
        };
        struct Factors {
            FactorWords g, u;
        };
        float sg[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, su[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        by_rows<C>(
            lds, acc, m0, n0, wm, wn,
            [&](int m, int n) __attribute__((always_inline)) {
                const uint32_t off = offset(m, n, p.ldf);
                return Factors{__builtin_bit_cast(FactorWords, __builtin_amdgcn_raw_buffer_load_b128(rf, off, 0, kOnce)),
                               __builtin_bit_cast(FactorWords, __builtin_amdgcn_raw_buffer_load_b128(rf, up_of(off), 0, kOnce))};
            },
            [&](int m, int n, float (&v)[8], const Factors& f) __attribute__((always_inline)) {
                float g[8], u[8];
                unpack_factors(f.g, g);
                unpack_factors(f.u, u);
                const bool there = m < p.M;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    g[e] *= v[e];
                    u[e] *= v[e];
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

    // fp32: 32 consecutive columns of a row across the lanes of a half
    template <typename C>
    static FBL_DEV void done(const Args& p, float*, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        const int lane = threadIdx.x & 63, g = lane >> 5, F = p.N;
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes), rf = span(p.factors, p.f_bytes);
        const auto load = [](__amdgpu_buffer_rsrc_t r, uint32_t off) __attribute__((always_inline)) {
            return __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
        };
        const auto store = [](__amdgpu_buffer_rsrc_t r, uint32_t off, float v) __attribute__((always_inline)) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(v), r, off, 0, 0);
        };
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
                float fg[16], fu[16];  // all on the way before the first store
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    fg[r] = load(rf, offset(r, p.ldf, n)), fu[r] = load(rf, offset(r, p.ldf, F + n));
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float dg = acc[tm][tn][r] * fg[r], du = acc[tm][tn][r] * fu[r];
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
};

}  // namespace

hipError_t launch_gated_grad(int f32, int tile, const GatedArgs& p, hipStream_t stream) {
    return f32 ? launch_f32_tile<false, true, GatedGradEp>(f32_tile(p), p, stream)
               : launch_gemm_tile<false, true, GatedGradEp>(tile, p, stream);
}

}  // namespace fbl
