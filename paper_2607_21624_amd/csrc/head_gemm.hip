// head_gemm.hip -- softmax losses of a linear head over a large vocabulary without
// keeping the logits, gfx950: the products.
//
//   z = X W,  lse = log sum_v exp(z_v / T)                        forward
//   dz = g (exp(z / T - lse) - targets),  dX = dz W^T,  dW = X^T dz   backward
//
// The logits exist only as accumulators.  The forward reduces each tile to its
// rows' maximum and sum of exponentials (8 bytes for 256 columns instead of 512) and picks the
// targets' logits out of it; the backward computes a piece of the vocabulary again, turns it into dz
// where it stands and writes that, for the two gradient products to read.  With
// tokens along the lanes and the vocabulary along the registers (C^T accumulators)
// a row's reduction is in-lane but for one exchange between the halves of a wavefront and
// one between the wavefronts that share its columns.
//
// Bound by the matrix products: 2 M K V forward and 6 M K V backward (one third of it z again).
#include "gemm_bf16.hpp"
#include "gemm_cost.hpp"
#include "gemm_f32.hpp"

namespace fbl {

namespace {

// A wavefront's share of a tile: NV x NM blocks of 32 x 32, vocabulary entries v0 + 32 i + acc_row(r, g)
// (within the piece) and tokens m0 + 32 j + lane % 32.
//
// Entries of the list `index` that fall on this lane's registers: hit(j, a, here, m, t) for target t of token m,
// the lane's j-th: entry v0 + a where `here`.  Few tiles hold any: called only where some
// lane of the wavefront has one.
template <int NV, int NM, typename F>
FBL_DEV void for_targets(const HeadArgs& p, int v0, int m0, F&& hit) {
    const int lane = threadIdx.x & 63, g = lane >> 5;
    // 16 reads at a time, for all the wavefront's tokens: one by one each waits out its latency
    constexpr int U = 16 / NM;
    for (int t0 = 0; t0 < p.top; t0 += U) {
        int at[NM][U];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < NM; ++j) {
                const int m = m0 + 32 * j + (lane & 31);
                at[j][u] = t0 + u < p.top && m < p.tokens ? p.index[(int64_t)(t0 + u) * p.tokens + m] : -1;
            }
        unroll_steps(std::make_integer_sequence<int, NM>{}, [&](auto j_c) __attribute__((always_inline)) {
            constexpr int J = decltype(j_c)::value;
            bool any = false;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                at[J][u] -= p.first + v0;
                if (((at[J][u] >> 2) & 1) != g) at[J][u] = -1;
                any |= (unsigned)at[J][u] < 32u * NV;
            }
            if (__builtin_amdgcn_ballot_w64(any) == 0) return;
            const int here = p.top - t0 < U ? p.top - t0 : U;
            for (int u = 0; u < here; ++u) {
                int a = at[J][0];
#pragma unroll
                for (int k = 1; k < U; ++k) a = u == k ? at[J][k] : a;
                if (__builtin_amdgcn_ballot_w64((unsigned)a < 32u * NV) == 0) continue;
                hit(j_c, a, (unsigned)a < 32u * NV, m0 + 32 * J + (lane & 31), t0 + u);
            }
        });
    }
}

// Forward: part[tile][m] and target[t][m].  WV wavefronts share a token's columns; wv is this
// one's place among them and mw its first token within the tile.
template <int NV, int NM, int WV, int TOKENS, int NT>
FBL_DEV void head_stats(const HeadArgs& p, f32x16 (&acc)[NV][NM], float2* shared, int v0, int m0, int wv, int mw, int tile,
                        int tile_m0) {
    const int lane = threadIdx.x & 63, g = lane >> 5;
    for_targets<NV, NM>(p, v0, m0, [&](auto j_c, int a, bool here, int m, int t) __attribute__((always_inline)) {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) z = a == 32 * i + acc_row(r, g) ? acc[i][decltype(j_c)::value][r] : z;
        if (here) p.target[(int64_t)t * p.tokens + m] = z;
    });
    if (v0 + 32 * NV > p.width) {  // columns past the piece count for nothing
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (v0 + 32 * i + acc_row(r, g) >= p.width) {
#pragma unroll
                    for (int j = 0; j < NM; ++j) acc[i][j][r] = -INFINITY;
                }
    }
    __syncthreads();  // the last step's operands have been read
#pragma unroll
    for (int j = 0; j < NM; ++j) {
        float top = acc[0][j][0];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
        top = fmaxf(top, other_half(top)) * p.unit;
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += fast_exp2(__builtin_fmaf(acc[i][j][r], p.unit, -ref));
        sum += other_half(sum);
        if (g == 0) shared[wv * TOKENS + mw + 32 * j + lane] = make_float2(top, sum);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TOKENS; i += NT) {
        if (tile_m0 + i >= p.tokens) break;
        float2 s = shared[i];
#pragma unroll
        for (int w = 1; w < WV; ++w) {
            const float2 o = shared[w * TOKENS + i];
            const float top = fmaxf(s.x, o.x), ref = top == -INFINITY ? 0.f : top;
            s = make_float2(top, s.y * fast_exp2(s.x - ref) + o.y * fast_exp2(o.x - ref));
        }
        p.part[(int64_t)(p.tile0 + tile) * p.tokens + tile_m0 + i] = s;
    }
}

// Backward: the accumulators become dz, columns past the piece 0.
template <int NV, int NM>
FBL_DEV void head_dz(const HeadArgs& p, f32x16 (&acc)[NV][NM], int v0, int m0) {
    const int lane = threadIdx.x & 63, g = lane >> 5;
    float scale[NM];
#pragma unroll
    for (int j = 0; j < NM; ++j) {
        const int m = m0 + 32 * j + (lane & 31);
        const float2 row = m < p.tokens ? p.row[m] : make_float2(0.f, 0.f);
        scale[j] = row.x;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = fast_exp2(__builtin_fmaf(acc[i][j][r], p.unit, -row.y));
    }
    for_targets<NV, NM>(p, v0, m0, [&](auto j_c, int a, bool here, int m, int t) __attribute__((always_inline)) {
        const float w = here && p.weight ? p.weight[(int64_t)t * p.tokens + m] : 1.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][decltype(j_c)::value][r] -= a == 32 * i + acc_row(r, g) ? w : 0.f;
    });
#pragma unroll
    for (int j = 0; j < NM; ++j)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = v0 + 32 * i + acc_row(r, g) < p.width && scale[j] != 0.f ? acc[i][j][r] * scale[j] : 0.f;
}

struct HeadFwd {
    using Args = HeadArgs;
    static constexpr bool kByRows = false, kSplits = false;
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        extern __shared__ __attribute__((aligned(1024))) unsigned char gemm_smem[];
        constexpr int BM = C::BM, BN = C::BN;
        head_stats<C::TN, C::TM, C::WN, BM, 64 * C::WM * C::WN>(p, acc, (float2*)gemm_smem, n0 + wn * C::TN * 32,
                                                        m0 + wm * C::TM * 32, wn, wm * C::TM * 32, n0 / BN, m0);
    }
    template <typename C>
    static FBL_DEV void done(const Args& p, float* smem, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        head_stats<C::TM, C::TN, C::t.wm, C::t.bn, 64 * C::t.wm * C::t.wn>(p, acc, (float2*)smem, m0 + wm * C::TM * 32, n0 + wn * C::TN * 32,
                                                          wm, wn * C::TN * 32, m0 / C::t.bm, n0);
    }
};

struct HeadGrad {
    using Args = HeadArgs;
    static constexpr bool kByRows = true, kSplits = false;
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t lds, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        head_dz(p, acc, n0 + wn * C::TN * 32, m0 + wm * C::TM * 32);
        const __amdgpu_buffer_rsrc_t rz = span(p.dz, p.dz_bytes);
        const auto nothing = [](int, int) __attribute__((always_inline)) { return Nothing{}; };
        by_rows<C>(lds, acc, m0, n0, wm, wn, nothing, [&](int m, int n, float (&v)[8], Nothing) __attribute__((always_inline)) {
            const bool in = m < p.tokens && n < p.ldz;
            store8(rz, in ? (uint32_t)(((int64_t)m * p.ldz + n) * 2) : kNowhere, v, n, (int)p.ldz);
        });
    }
    template <typename C>
    static FBL_DEV void done(const Args& p, float*, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        const int lane = threadIdx.x & 63, g = lane >> 5, v0 = m0 + wm * C::TM * 32;
        head_dz(p, acc, v0, n0 + wn * C::TN * 32);
        const __amdgpu_buffer_rsrc_t rz = span(p.dz, p.dz_bytes);
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            const int m = n0 + (wn * C::TN + j) * 32 + (lane & 31);
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int v = v0 + 32 * i + 8 * q + 4 * g;
                    const uint32_t off = m < p.tokens && v < p.ldz ? (uint32_t)(((int64_t)m * p.ldz + v) * 4) : kNowhere;
                    const f32x4 x = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, x), rz, off, 0, 0);
                }
        }
    }
};

// dX over the pieces of the vocabulary: sums in fp32, scaled and rounded once with the last piece.  (And
// dW, of one piece.)
//
// The factor of a mean's or sum's gradient is the same for every row, so bf16 keeps it out of dz: dz's
// largest entries, -1 at the labels, are then exact, where g, a constant, rounded would be off by the same
// 2^-9 in every row (4096 x 1024 x 50257: error of dx 0.28% of its norm, 0.17% of
// which are the result's own rounding).  A factor of each row's own, and distillation's weights of the targets, are
// in dz and rounded with it: one rounding of an operand that the matrix instructions take in 16 bits (2048 x 2048 x
// 128256, 32 targets a row: 0.23%).
template <bool SPLIT>
struct SumPieces {
    using Args = SumArgs;
    static constexpr bool kByRows = true, kSplits = SPLIT;
    template <typename C>
    static FBL_DEV void done(const Args& p, uint32_t lds, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn) {
        const bool last = !SPLIT && p.last;
        const float scale = last ? *p.scale : 1.f;
        const __amdgpu_buffer_rsrc_t rc = span(p.c, p.c_bytes),
                                     rs = span(SPLIT ? p.sum + (int64_t)blockIdx.y * p.M * p.lds : p.sum, p.sum_bytes);
        struct Sums {
            f32x4 h[2];
        };
        const auto offset = [&](int m, int n) __attribute__((always_inline)) {
            return m < p.M && n < p.N ? (uint32_t)(((int64_t)m * p.lds + n) * 4) : kNowhere;
        };
        const auto ahead = [&](int m, int n) __attribute__((always_inline)) {
            Sums s;
            const uint32_t off = p.first ? kNowhere : offset(m, n);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                s.h[h] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 16 * h, 0));
            return s;
        };
        by_rows<C>(lds, acc, m0, n0, wm, wn, ahead, [&](int m, int n, float (&v)[8], const Sums& s) __attribute__((always_inline)) {
            const bool in = m < p.M && n < p.N;
            const uint32_t soff = offset(m, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += s.h[e / 4][e % 4];  // 0 with the first piece
            if (last) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= scale;
                store8(rc, in ? (uint32_t)(((int64_t)m * p.ldc + n) * 2) : kNowhere, v, n, p.N);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 s = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                    // the second four may be past the row (N a multiple of 4), where the next one begins
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, s), rs,
                                                           n + 4 * h < p.N ? soff + 16 * h : kNowhere, 0, 0);
                }
            }
        });
    }
    template <typename C>
    static FBL_DEV void done(const Args& p, float*, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int wm, int wn) {
        const int lane = threadIdx.x & 63, g = lane >> 5;
        const __amdgpu_buffer_rsrc_t rc =
            SPLIT ? span(p.sum + (int64_t)blockIdx.y * p.M * p.lds, p.sum_bytes) : span(p.c, p.c_bytes);
        const int64_t ld = SPLIT ? p.lds : p.ldc;
#pragma unroll
        for (int tm = 0; tm < C::TM; ++tm)
#pragma unroll
            for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int m = m0 + (wm * C::TM + tm) * 32 + acc_row(r, g), n = n0 + (wn * C::TN + tn) * 32 + (lane & 31);
                    const uint32_t off = m < p.M && n < p.N ? (uint32_t)(((int64_t)m * ld + n) * 4) : kNowhere;
                    float v = acc[tm][tn][r];
                    if (!p.first) v += __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rc, off, 0, 0));
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(v), rc, off, 0, 0);
                }
    }
};

// c = sum of the planes times *scale, in a fixed order.  A thread adds an element's planes; where there are many, SLICES
// threads take every SLICES-th each, for a chain of loads as much shorter, and their sums are added one after the
// other.
template <typename T, int SLICES>
__global__ __launch_bounds__(256) void sum_planes(const float* planes, int splits, int64_t M, int64_t N, const float* scale,
                                                  T* c, int64_t ldc) {
    constexpr int COLS = 256 / SLICES;
    __shared__ float part[SLICES][COLS];
    const int l = threadIdx.x % COLS, r = threadIdx.x / COLS;
    const int64_t n = (int64_t)blockIdx.x * COLS + l, at = n < N ? n : N - 1;
    const float f = scale ? *scale : 1.f;
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
        const auto plane = [&](int i) { return planes[((int64_t)i * M + m) * N + at]; };
        float s = 0.f;
        int i = r;
        for (; i + 3 * SLICES < splits; i += 4 * SLICES) {
            const float a = plane(i), b = plane(i + SLICES), d = plane(i + 2 * SLICES), e = plane(i + 3 * SLICES);
            s += a, s += b, s += d, s += e;
        }
        for (; i < splits; i += SLICES) s += plane(i);
        if constexpr (SLICES > 1) {
            __syncthreads();
            part[r][l] = s;
            __syncthreads();
            if (r > 0) continue;
#pragma unroll
            for (int k = 1; k < SLICES; ++k) s += part[k][l];
        }
        if (n < N) c[m * ldc + n] = (T)(s * f);
    }
}

template <typename EP>
hipError_t launch_head(int f32, int table, HeadArgs& p, hipStream_t s) {
    if (!f32) {  // C = X W: tokens are the rows
        switch (p.shape) {
            case 9: return table ? launch_gemm_bf16<9, false, true, EP>(p, s) : launch_gemm_bf16<9, false, false, EP>(p, s);
            case 16: return table ? launch_gemm_bf16<16, false, true, EP>(p, s) : launch_gemm_bf16<16, false, false, EP>(p, s);
            case 15: return table ? launch_gemm_bf16<15, false, true, EP>(p, s) : launch_gemm_bf16<15, false, false, EP>(p, s);
            case 6: return table ? launch_gemm_bf16<6, false, true, EP>(p, s) : launch_gemm_bf16<6, false, false, EP>(p, s);
            case 4: return table ? launch_gemm_bf16<4, false, true, EP>(p, s) : launch_gemm_bf16<4, false, false, EP>(p, s);
            default: return table ? launch_gemm_bf16<19, false, true, EP>(p, s) : launch_gemm_bf16<19, false, false, EP>(p, s);
        }
    }
    // C = W^T X^T: the vocabulary is the rows, so that tokens lie along the lanes here too
    std::swap(p.a, p.b), std::swap(p.lda, p.ldb), std::swap(p.a_bytes, p.b_bytes), std::swap(p.M, p.N);
    switch (p.shape) {
        case 2: return table ? launch_gemm_f32<2, false, true, EP>(p, s) : launch_gemm_f32<2, true, true, EP>(p, s);
        case 3: return table ? launch_gemm_f32<3, false, true, EP>(p, s) : launch_gemm_f32<3, true, true, EP>(p, s);
        case 4: return table ? launch_gemm_f32<4, false, true, EP>(p, s) : launch_gemm_f32<4, true, true, EP>(p, s);
        case 5: return table ? launch_gemm_f32<5, false, true, EP>(p, s) : launch_gemm_f32<5, true, true, EP>(p, s);
        default: return table ? launch_gemm_f32<0, false, true, EP>(p, s) : launch_gemm_f32<0, true, true, EP>(p, s);
    }
}

// The tile of a split product: as narrow as the few rows that split one.
constexpr int kSplitTileLarge = 19;
int split_tile(int64_t M) { return M <= 32 ? 15 : M <= 64 ? 6 : M <= 128 ? 4 : kSplitTileLarge; }
constexpr int kSplitTileF32 = 4;

}  // namespace

// bf16: of tiles of 32, 64, 128 and 256 tokens, the narrower two also with a contraction split among their wavefronts,
// the one of least modelled time (gemm_cost.hpp; 4 tokens x 3600 x 288 forward 25.2 us without the split ones, 17.0
// with, 16 x 8192 x 128 43.1 and 24.5, 300 x 4096 x 1000 28.0 and 19.8).  Two workgroups a CU, so that one's exponentials
// and stores run beside the other's products, do not pay for their narrower tiles: 4096 x 1024 x 50257 forward 451
// us with 256 x 256, 495 with 256 x 128 or 128 x 256 in steps of 32, 581 with 128 x 128; dz 141, 159, 156 and 171 a
// piece.
// fp32: 128 x 128 where that makes two workgroups for each CU; 64 x 64 with more than 320 of them (300 x 2000 x 5000
// forward 88.4 us, 91.1 with 64 x 32 on half a step a wavefront, 85.5 with 32 x 32 on a quarter, but 1000 x 700 x 4000
// 71, 85 and 84); 64 x 32 down to 160 (250 x 500 x 5003 30.6, 29.0 and 32.3); below, 32 x 32 on a quarter, or for 1024
// and more on an eighth (500 x 512 x 1000 22.4, 17.7, 16.6 and 17.5; 128 x 2048 x 1024 53, 35, 27 and 23).
int head_tile(int f32, int table, int64_t M, int64_t V, int64_t K) {
    if (f32) {
        const auto tiles = [&](int64_t n) { return ((M + n - 1) / n) * ((V + n - 1) / n); };
        return tiles(128) >= 512 ? 0 : tiles(64) > 320 ? 2 : tiles(64) > 160 ? 3 : K < 1024 ? 4 : 5;
    }
    int best = 19;
    for (int t : {4, 6, 15, 9, 16})
        if (gemm_cost(t, table, M, V, K) < gemm_cost(best, table, M, V, K)) best = t;
    return best;
}
int head_tile_width(int f32, int tile) { return f32 ? kF32Tiles[tile].bm : kGemmTiles[tile].bn; }

hipError_t launch_head_fwd(int f32, int table, HeadArgs p, hipStream_t s) { return launch_head<HeadFwd>(f32, table, p, s); }
hipError_t launch_head_grad(int f32, int table, HeadArgs p, hipStream_t s) { return launch_head<HeadGrad>(f32, table, p, s); }

// Products of few rows have few tiles for a long contraction (dX over a vocabulary, a layer's forward for a few
// tokens): where they do not fill the card, workgroups share them, two a CU in all with a contraction
// of 512 at least (fp32: four a CU of its small tiles, 256).  From 129 rows bf16 shares a contraction only where that
// lets 256 x 256 tiles fill the card in place of smaller ones and the model has it 5% below, the planes' 8 bytes
// at 4.5 TB/s included (2048 x 2048 from pieces of 32768 in four shares: 270 -> 245 us; 4096 x 1024 from 16384: 160 -> 143).
int sum_splits(int f32, int b_nmajor, int64_t M, int64_t N, int64_t kc, int tile) {
    if (!f32 && M > 128) {
        const int64_t tiles = ((M + 255) / 256) * ((N + 255) / 256), s = 256 / tiles;
        if (s < 2 || s > 8 || kc / s < 2048) return 1;
        const double shared = gemm_cost(kSplitTileLarge, b_nmajor, M * s, N, kc / s) + 8.0 * (double)(s * M * N) / 4.5e6;
        return shared < 0.95 * gemm_cost(tile, b_nmajor, M, N, kc) ? (int)s : 1;
    }
    const int t = split_tile(M), bm = f32 ? kF32Tiles[kSplitTileF32].bm : kGemmTiles[t].bm,
              bn = f32 ? kF32Tiles[kSplitTileF32].bn : kGemmTiles[t].bn;
    const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
    const int64_t want = f32 ? 1024 : 512;
    if (tiles > want / 2) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>((want + tiles / 2) / tiles, kc / (f32 ? 256 : 512)));
}

// A small weight gradient has few tiles and all tokens for its contraction.  Its shares are of 128 x 128 tiles, or 64 x
// 64 for a narrow layer (fp32: 64 x 64), up to two workgroups a CU in all, with 512 tokens each at least (fp32 256): bf16
// where the model has them 10% below, fp32 from 2048 tokens (alone and shared, us: bf16 32768 tokens 128 x 128 75 and
// 24, 8192 tokens 256 x 256 22.1 and 14.4, 8027 tokens 328 x 320 24.9 and 20.0; fp32 32768 tokens 128 x 128 199 and 28,
// 8192 tokens 256 x 256 52 and 18, 4096 tokens 512 x 1024 52 and 49, 2048 tokens 256 x 256 15.7 and 12.0).
static int weight_split_tile(int f32, int64_t K, int64_t N) { return f32 ? 2 : K <= 64 || N <= 64 ? 7 : 4; }

int weight_splits(int f32, int64_t M, int64_t K, int64_t N, int tile) {
    if (K * N > kWeightSplitMax) return 1;
    const int t = weight_split_tile(f32, K, N), bm = f32 ? kF32Tiles[t].bm : kGemmTiles[t].bm,
              bn = f32 ? kF32Tiles[t].bn : kGemmTiles[t].bn;
    const int64_t rows = (K + bm - 1) / bm, tiles = rows * ((N + bn - 1) / bn);
    const int64_t s = std::min<int64_t>(512 / tiles, M / (f32 ? 256 : 512));
    if (s < 2) return 1;
    if (f32) return M >= 2048 ? (int)s : 1;
    const double shared = gemm_cost(t, 2, rows * bm * s, N, M / s) + 3.0 + 8.0 * (double)(s * K * N) / 4.5e6;
    return shared < 0.9 * gemm_cost(tile, 2, K, N, M) ? (int)s : 1;
}

hipError_t launch_weight_shares(int f32, const SumArgs& p, hipStream_t s) {
    using EP = SumPieces<true>;
    const int t = weight_split_tile(f32, p.M, p.N);
    if (f32) return launch_gemm_f32<2, true, false, EP>(p, s, p.splits);
    return t == 4 ? launch_gemm_bf16<4, true, false, EP>(p, s, p.splits) : launch_gemm_bf16<7, true, false, EP>(p, s, p.splits);
}

hipError_t launch_sum_gemm(int a_kmajor, int b_nmajor, int tile, const SumArgs& p, hipStream_t s) {
    if (p.splits > 1) {
        const auto run = [&](auto bt_c) {
            constexpr bool BT = decltype(bt_c)::value;
            switch (split_tile(p.M)) {
                case 15: return launch_gemm_bf16<15, false, BT, SumPieces<true>>(p, s, p.splits);
                case 6: return launch_gemm_bf16<6, false, BT, SumPieces<true>>(p, s, p.splits);
                case 4: return launch_gemm_bf16<4, false, BT, SumPieces<true>>(p, s, p.splits);
                default: return launch_gemm_bf16<kSplitTileLarge, false, BT, SumPieces<true>>(p, s, p.splits);
            }
        };
        return b_nmajor ? run(std::true_type{}) : run(std::false_type{});
    }
    using EP = SumPieces<false>;
    if (a_kmajor) return launch_gemm_tile<true, false, EP>(tile, p, s);
    return b_nmajor ? launch_gemm_tile<false, true, EP>(tile, p, s) : launch_gemm_tile<false, false, EP>(tile, p, s);
}
hipError_t launch_sum_gemm_f32(int b_nmajor, const SumArgs& p, hipStream_t s) {
    if (p.splits > 1) {
        using EP = SumPieces<true>;
        return b_nmajor ? launch_gemm_f32<kSplitTileF32, false, true, EP>(p, s, p.splits)
                        : launch_gemm_f32<kSplitTileF32, false, false, EP>(p, s, p.splits);
    }
    using EP = SumPieces<false>;
    return b_nmajor ? launch_f32_tile<false, true, EP>(f32_tile(p), p, s) : launch_f32_tile<false, false, EP>(f32_tile(p), p, s);
}

hipError_t launch_sum_planes(int f32, const float* planes, int splits, int64_t M, int64_t N, const float* scale, void* c,
                             int64_t ldc, hipStream_t s) {
    const auto run = [&](auto kernel, int cols, auto* out) {
        const dim3 grid((unsigned)((N + cols - 1) / cols), (unsigned)std::min<int64_t>(M, 4096));
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, planes, splits, M, N, scale, out, ldc);
        return hipGetLastError();
    };
    const bool many = splits >= 16;
    if (f32) return many ? run(sum_planes<float, 8>, 32, (float*)c) : run(sum_planes<float, 1>, 256, (float*)c);
    return many ? run(sum_planes<bf16, 8>, 32, (bf16*)c) : run(sum_planes<bf16, 1>, 256, (bf16*)c);
}

}  // namespace fbl
