// gemm_bf16.hpp -- the kernel of the bf16 matrix products, gfx950: the projection
// products (proj_gemm.hip, whose head describes the products, the operand reads and
// the partial tiles) and the products with something fused behind them
// (linear_gemm.hpp, head_gemm.hip).
#pragma once

#include <array>
#include <type_traits>
#include <utility>

#include "cdna4.hpp"
#include "gemm_tiles.hpp"
#include "kernels.hpp"
#include "stage.hpp"

namespace fbl {

namespace {

// LDS tile of ROWS stored rows of COLS bf16 elements (swizzled as in stage.hpp),
// loaded by NW wavefronts.
template <int ROWS, int COLS, int NW>
struct GTile {
    using G = TileGeom<bf16, COLS>;
    using Dma = DmaPlan<bf16, COLS, ROWS, NW>;
    static constexpr int BYTES = ROWS * COLS * 2;
    // every wavefront issues the same number of loads, so one vmcnt count fits all
    static_assert(Dma::INSTS % NW == 0, "whole 1 KB loads per wavefront");
    // row read: stored row r (lane % 32 + 32 * tile), columns 16c + 8g .. +7
    static FBL_DEV uint32_t row_addr(int lane, int c) {
        return 2u * (uint32_t)G::off(lane & 31, 16 * c + 8 * (lane >> 5));
    }
    // transposed read, natural order: stored rows 8g + 4h + [0..3] (plus 16kc),
    // column 32t + lane % 32
    static FBL_DEV uint32_t tr_addr(int lane, int t, int h) {
        const int q = lane & 15;
        const int r = 8 * (lane >> 5) + 4 * h + (q >> 2);
        const int col = 32 * t + 16 * ((lane >> 4) & 1) + 4 * (q & 3);
        return 2u * (uint32_t)G::off(r, col);
    }
};

// AT: A stored k-major ([K, M] rows); BT: B stored n-major ([N, K] rows).
template <int BM_, int BN_, int BK, int NS, int WM_, int WN_, int WK, bool AT, bool BT>
struct GemmCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int NW = WM * WN * WK;
    using TA = GTile<AT ? BK : BM, AT ? BM : BK, NW>;
    using TB = GTile<BT ? BN : BK, BT ? BK : BN, NW>;
    static constexpr int TM = BM / (32 * WM), TN = BN / (32 * WN);  // 32x32 tiles per wavefront
    static constexpr int NKC = BK / 16;                              // 16-deep MFMA chunks per step
    static constexpr int KCW = NKC / WK;                             // chunks per wavefront per step
    static constexpr int SA = TA::BYTES, SB = TB::BYTES;
    static constexpr int STAGE = SA + SB;
    static constexpr int BYTES = gemm_lds_bytes(GemmTile{BM, BN, BK, NS, WM, WN, WK});
    static constexpr int LOADS = TA::Dma::PER_WAVE + TB::Dma::PER_WAVE;
    static constexpr int PART = TM * TN * 4096;  // bytes of one wavefront's partial sums
    static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "wavefront tiles of whole 32x32 blocks");
    static_assert(BK % 32 == 0 && NKC % WK == 0 && NS >= 2, "whole chunks per wavefront, at least double buffered");
    static_assert(NW == 4 || NW == 8, "4 or 8 wavefronts");
    // stage offsets are added at run time; the read immediates are tile offsets within a stage
    static_assert((TM - 1) * 32 * BK * 2 < 65536 && (TN - 1) * 32 * BK * 2 < 65536 &&
                      (KCW - 1) * 16 * (BM > BN ? BM : BN) * 2 + 128 < 65536,
                  "LDS read immediates fit 16 bits");
    static constexpr int ROWS_BYTES = WM * WN * 32 * (32 * TN + 4) * 4;  // of by_rows below
    static_assert(ROWS_BYTES <= 160 * 1024, "LDS");
    static_assert(BYTES <= 160 * 1024 && NS * STAGE <= BYTES && (WK - 1) * WM * WN * PART <= BYTES, "LDS");
    static_assert((NS - 1) * LOADS < 64, "vmcnt range");
    // wavefronts per SIMD the registers must allow: two workgroups per CU where LDS does
    static constexpr int OCC = BYTES <= 80 * 1024 ? NW / 2 : NW / 4;
};

// What becomes of an output tile.  EP::Args is GemmArgs or derived from it; PlainStore
// writes the tile as it is, any other EP gets it as
//   EP::done<Cfg>(args, lds, acc, m0, n0, wm, wn)
// on every wavefront that holds a share of it (all of them, or those of wk = 0 where
// the contraction is split): acc[tn][tm] is the C^T tile of rows m0 + (wm * TM + tm) *
// 32 + lane % 32 and columns n0 + (wn * TN + tn) * 32 + acc_row(register, lane / 32).
// The loads have all landed; LDS is free once the wavefronts have met at a barrier.
//
// EP::kPairs (where there is one, and true): the weight [K, 2F] holds two matrices side by side, and a tile's columns are
// 8 of the one, 8 of the other, 8 of the one ..: p.N is 2F, and tile column n is column n0 / 2 + 8 (n / 16) + n % 8 of
// matrix n / 8 % 2.  A 16-byte load is 8 columns, so only the loads' addresses know; and the accumulators of a column's pair are
// in one lane, four registers apart.
template <typename EP, typename = void>
struct PairsOf : std::false_type {};
template <typename EP>
struct PairsOf<EP, std::enable_if_t<EP::kPairs>> : std::true_type {};

struct PlainStore {
    using Args = GemmArgs;
    static constexpr bool kByRows = false;  // done uses by_rows
    static constexpr bool kSplits = false;  // gridDim.y workgroups share a tile's contraction (take_share)
};

template <int BM, int BN, int BK, int NS, int WM, int WN, int WK, bool AT, bool BT, typename EP>
__global__ __launch_bounds__(64 * WM * WN * WK, (GemmCfg<BM, BN, BK, NS, WM, WN, WK, AT, BT>::OCC)) void
proj_gemm_bf16(typename EP::Args p) {
    using C = GemmCfg<BM, BN, BK, NS, WM, WN, WK, AT, BT>;
    using TA = typename C::TA;
    using TB = typename C::TB;
    constexpr int TM = C::TM, TN = C::TN, KCW = C::KCW;
    constexpr bool PAIRS = PairsOf<EP>::value;
    static_assert(!PAIRS || !BT, "columns of pairs along B's stored rows");
    extern __shared__ __attribute__((aligned(1024))) unsigned char gemm_smem[];
    const uint32_t lds = lds_addr(gemm_smem);
    if constexpr (EP::kSplits) take_share<2, AT, BT>(p);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 5;
    // wavefront position: (wm, wn) in the tile grid, wk = its share of each step
    const int wm = wave % WM, wn = (wave / WM) % WN, wk = wave / (WM * WN);
    const int mt = (p.M + BM - 1) / BM, nt = (p.N + BN - 1) / BN;
    // consecutive ids share a column block of B (the weight) and land on one XCD
    const int logical = xcd_logical_id(blockIdx.x, mt * nt, gridDim.x);
    if (logical < 0) return;
    const int m0 = (logical % mt) * BM, n0 = (logical / mt) * BN;
    const int nk = (p.K + BK - 1) / BK;

    // ---- DMA: each stage holds the A and B tiles of one BK-deep step
    const Rsrc ra = make_rsrc(p.a, p.a_bytes), rb = make_rsrc(p.b, p.b_bytes);
    typename TA::Dma da;
    typename TB::Dma db;
    da.init((uint32_t)(p.lda * 2), wave, lane);
    if constexpr (PAIRS) {
        const uint32_t second = (uint32_t)p.N;  // bytes from one matrix to the other
        db.init((uint32_t)(p.ldb * 2), wave, lane,
                [&](int c) __attribute__((always_inline)) { return (uint32_t)(c >> 1) * 16u + (c & 1 ? second : 0u); });
    } else {
        db.init((uint32_t)(p.ldb * 2), wave, lane);
    }
    auto a_off = [&](int s) __attribute__((always_inline)) {
        const int k0 = s * BK;
        return (uint32_t)((AT ? (int64_t)k0 * p.lda + m0 : (int64_t)m0 * p.lda + k0) * 2);
    };
    auto b_off = [&](int s) __attribute__((always_inline)) {
        const int k0 = s * BK;
        return (uint32_t)((BT ? (int64_t)n0 * p.ldb + k0 : (int64_t)k0 * p.ldb + (PAIRS ? n0 / 2 : n0)) * 2);
    };
    auto issue = [&](int s, int buf) __attribute__((always_inline)) {
        da.issue(lds + buf * C::STAGE, ra, a_off(s), wave);
        db.issue(lds + buf * C::STAGE + C::SA, rb, b_off(s), wave);
    };

    // ---- per-lane LDS read addresses (stage 0, the wavefront's first chunk)
    const int kc0 = wk * KCW;
    uint32_t aaddr[AT ? TM : KCW][2], baddr[BT ? KCW : TN][2];
    if constexpr (AT) {
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                aaddr[tm][h] = lds + TA::tr_addr(lane, wm * TM + tm, h) + (uint32_t)(kc0 * 16 * BM * 2);
    } else {
#pragma unroll
        for (int j = 0; j < KCW; ++j) aaddr[j][0] = lds + TA::row_addr(lane, kc0 + j);
    }
    if constexpr (BT) {
#pragma unroll
        for (int j = 0; j < KCW; ++j) baddr[j][0] = lds + C::SA + TB::row_addr(lane, kc0 + j);
    } else {
#pragma unroll
        for (int tn = 0; tn < TN; ++tn)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                baddr[tn][h] = lds + C::SA + TB::tr_addr(lane, wn * TN + tn, h) + (uint32_t)(kc0 * 16 * BN * 2);
    }
    const uint32_t arow = (uint32_t)(wm * TM * 32 * BK * 2), brow = (uint32_t)(wn * TN * 32 * BK * 2);
    // fragment of A for m-tile tm, the wavefront's chunk j, from the stage at
    // byte offset `stage` (a run-time, wave-uniform value added to the address)
    auto frag_a = [&](uint32_t stage, int tm, int j) __attribute__((always_inline)) {
        Frag<bf16> f;
        if constexpr (AT) {
            const uint32_t off = j * 16 * BM * 2;
            const bf16x4 x = lds_tr(aaddr[tm][0] + stage, off), y = lds_tr(aaddr[tm][1] + stage, off);
            f.v = bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        } else {
            f.v = lds_b128(aaddr[j][0] + stage + arow, tm * 32 * BK * 2);
        }
        return f;
    };
    auto frag_b = [&](uint32_t stage, int tn, int j) __attribute__((always_inline)) {
        Frag<bf16> f;
        if constexpr (BT) {
            f.v = lds_b128(baddr[j][0] + stage + brow, tn * 32 * BK * 2);
        } else {
            const uint32_t off = j * 16 * BN * 2;
            const bf16x4 x = lds_tr(baddr[tn][0] + stage, off), y = lds_tr(baddr[tn][1] + stage, off);
            f.v = bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        }
        return f;
    };

    // C^T accumulators: acc[tn][tm] rows = n (acc_row), columns = m (lane)
    f32x16 acc[TN][TM];
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) acc[tn][tm] = f32x16{};

    // Step s: wait until step s has landed (the NS - 2 later steps may still
    // be in flight), meet, refill the stage step s-1 used with step s+NS-1,
    // then contract the wavefront's chunks of step s.
    auto wait_step = [&](int s) __attribute__((always_inline)) {
        const int later = min(NS - 2, nk - 1 - s);  // steps issued after step s
        if constexpr (NS >= 5) {
            if (later >= 3) { wait_vmcnt<(NS >= 5 ? 3 : 0) * C::LOADS>(); return; }
        }
        if constexpr (NS >= 4) {
            if (later == 2) { wait_vmcnt<(NS >= 4 ? 2 : 0) * C::LOADS>(); return; }
        }
        if constexpr (NS >= 3) {
            if (later == 1) { wait_vmcnt<C::LOADS>(); return; }
        }
        wait_vmcnt<0>();
    };
    static_assert(NS <= 5, "wait_step covers at most three steps in flight behind the awaited one");
    for (int s = 0; s < NS - 1 && s < nk; ++s) issue(s, s);
    // The last step may hold the end of the contraction (krem < BK elements
    // left, a multiple of 8).  Once its tiles have landed, the workgroup
    // zeroes their contraction positions krem .. BK-1 in LDS (whatever the
    // loads brought there: zeros past an operand's last row, or the next
    // row's elements past its width), so the products run unchanged.
    auto zero_tail = [&](uint32_t stage, int krem) __attribute__((always_inline)) {
        const int tid = threadIdx.x;
        constexpr int NT = 64 * C::NW;
        const f32x4 z = f32x4{};
        // operand tile with the contraction along its stored rows (AT / not BT): whole rows
        auto rows = [&](uint32_t tile, int cols) __attribute__((always_inline)) {
            const int n16 = (BK - krem) * cols / 8;  // 16-byte chunks past row krem
            for (int i = tid; i < n16; i += NT)
                *(FBL_LDS f32x4*)(uintptr_t)(tile + (uint32_t)(krem * cols * 2 + i * 16)) = z;
        };
        // operand tile with the contraction along its stored columns: chunks krem/8 .. of every row
        auto cols = [&](uint32_t tile, int nrows, auto geom) __attribute__((always_inline)) {
            using G = decltype(geom);
            const int per = (BK - krem) / 8;
            for (int i = tid; i < nrows * per; i += NT) {
                const int r = i / per, c = krem / 8 + i % per;
                *(FBL_LDS f32x4*)(uintptr_t)(tile + 2u * (uint32_t)G::off(r, 8 * c)) = z;
            }
        };
        const uint32_t ta = lds + stage, tb = lds + stage + C::SA;
        if constexpr (AT) rows(ta, BM);
        else cols(ta, BM, typename TA::G{});
        if constexpr (BT) cols(tb, BN, typename TB::G{});
        else rows(tb, BN);
    };
    int buf = 0;
    const int nfull = p.K / BK;  // steps wholly inside the contraction
    // One step.  MORE: a later step's loads are issued during it, a few after
    // every TM products: issued in one go (200 .. 400 cycles for 4 .. 8 of them)
    // they hold the wavefront's products up, between the products they cost
    // little.  With two stages they must land within this very step, so they go
    // into its first half; and where both operands take twice as many LDS reads
    // besides (AT, not BT) the late loads cost 2 .. 5% more than they save, so they
    // still go out in one go after the first reads.  In one go -> spread (us): dX 512
    // x 2048 from 8192 29.5 -> 25.7, Y 4096 x 3072 from 2048 56.8 -> 54.2, dW 2048 x
    // 3072 from 4096 65.0 -> 57.3, Y 1000 x 2304 from 768 9.2 -> 8.9; the tiles of one
    // workgroup per CU gain most (tile 5 dX 1.2x, 12 dX 1.15x, 17 .. 20 dX 1.1 .. 1.2x).
    // A step of two groups of products has nothing to spread them over (tile 16:
    // dX 3768 x 64 from 3648 11.0 -> 12.1), and one loop is the smaller kernel where
    // there is a single step (tile 3: U 512 x 2048 from 16 3.4 against 3.7).
    constexpr bool SPREAD = KCW * TN >= 4 && !(NS == 2 && AT && !BT);
    auto step = [&](auto more_c, int s) __attribute__((always_inline)) {
        constexpr bool MORE = decltype(more_c)::value;
        wait_step(s);
        __syncthreads();
        const uint32_t stage = (uint32_t)buf * C::STAGE;
        if (!(SPREAD && MORE) && s == nfull) {  // the partial last step (every load of it has landed: nothing is in flight)
            zero_tail(stage, p.K - s * BK);
            __syncthreads();
        }
        Frag<bf16> fa[2][TM], fb[2][TN];
        auto read = [&](auto j_c) __attribute__((always_inline)) {
            constexpr int J = decltype(j_c)::value;
#pragma unroll
            for (int tm = 0; tm < TM; ++tm) fa[J & 1][tm] = frag_a(stage, tm, J);
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) fb[J & 1][tn] = frag_b(stage, tn, J);
        };
        const int later = buf == 0 ? NS - 1 : buf - 1;  // the stage step s - 1 used
        const uint32_t sa = SPREAD && MORE ? a_off(s + NS - 1) : 0u, sb = SPREAD && MORE ? b_off(s + NS - 1) : 0u;
        const uint32_t into = lds + (uint32_t)later * C::STAGE;
        read(std::integral_constant<int, 0>{});
        if constexpr (!SPREAD) {
            if (s + NS - 1 < nk) issue(s + NS - 1, later);
        }
        unroll_steps(std::make_integer_sequence<int, KCW>{}, [&](auto j_c) __attribute__((always_inline)) {
            constexpr int J = decltype(j_c)::value;
            if constexpr (J + 1 < KCW) read(std::integral_constant<int, J + 1>{});
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) {
#pragma unroll
                for (int tm = 0; tm < TM; ++tm) mma(acc[tn][tm], fb[J & 1][tn], fa[J & 1][tm]);
                if constexpr (MORE && SPREAD) {
                    constexpr int GROUPS = NS == 2 ? (KCW * TN + 1) / 2 : KCW * TN, LA = TA::Dma::PER_WAVE;
                    const int gi = J * TN + tn;
                    if (gi < GROUPS) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int l = gi * C::LOADS / GROUPS; l < (gi + 1) * C::LOADS / GROUPS && l < C::LOADS; ++l) {
                        if (l < LA)
                            dma16<true>(ra, into + (uint32_t)(l * C::NW + wave) * 1024u, da.voff[l < LA ? l : 0], sa);
                        else
                            dma16<true>(rb, into + C::SA + (uint32_t)((l - LA) * C::NW + wave) * 1024u,
                                        db.voff[l < LA ? 0 : l - LA], sb);
                    }
                    if (gi < GROUPS) __builtin_amdgcn_sched_barrier(0);
                }
            }
        });
        buf = buf + 1 == NS ? 0 : buf + 1;
    };
    int s = 0;
    if constexpr (SPREAD)
        for (; s < nk - (NS - 1); ++s) step(std::true_type{}, s);
    for (; s < nk; ++s) step(std::false_type{}, s);

    if constexpr (WK > 1) {
        // Partial sums: wavefront (wm, wn, wk > 0) parks its accumulators in LDS
        // (the stages are free once every wavefront has passed the barrier
        // after its last step, whose loads it waited for in full); the wk = 0
        // wavefront of the tile adds them in the order wk = 1, 2, ... and stores.
        // Layout per wavefront: [tn][tm][quad][lane] x 16 bytes.
        __syncthreads();
        const uint32_t part0 = lds + (uint32_t)((wn * WM + wm) * C::PART);
        constexpr uint32_t kSlot = (uint32_t)(WM * WN * C::PART);
        if (wk > 0) {
            const uint32_t mine = part0 + (uint32_t)(wk - 1) * kSlot;
#pragma unroll
            for (int tn = 0; tn < TN; ++tn)
#pragma unroll
                for (int tm = 0; tm < TM; ++tm)
#pragma unroll
                    for (int qd = 0; qd < 4; ++qd) {
                        const uint32_t a = mine + (uint32_t)((((tn * TM + tm) * 4 + qd) * 64 + lane) * 16);
                        *(FBL_LDS f32x4*)(uintptr_t)a = f32x4{acc[tn][tm][4 * qd], acc[tn][tm][4 * qd + 1],
                                                              acc[tn][tm][4 * qd + 2], acc[tn][tm][4 * qd + 3]};
                    }
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int w = 1; w < WK; ++w) {
            const uint32_t theirs = part0 + (uint32_t)(w - 1) * kSlot;
#pragma unroll
            for (int tn = 0; tn < TN; ++tn)
#pragma unroll
                for (int tm = 0; tm < TM; ++tm)
#pragma unroll
                    for (int qd = 0; qd < 4; ++qd) {
                        const uint32_t a = theirs + (uint32_t)((((tn * TM + tm) * 4 + qd) * 64 + lane) * 16);
                        const f32x4 v = *(const FBL_LDS f32x4*)(uintptr_t)a;
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[tn][tm][4 * qd + e] += v[e];
                    }
        }
    }

    if constexpr (!std::is_same_v<EP, PlainStore>) {
        EP::template done<C>(p, lds, acc, m0, n0, wm, wn);
        return;
    }

    // C[m][n .. n+3]: lane <-> m, four consecutive n per store (N is a
    // multiple of 4, so a store is wholly inside or wholly outside).  Stores
    // outside the output go to an offset past the buffer's range, which the
    // hardware drops -- no divergent branches around the stores.
    using i32x2 = int __attribute__((ext_vector_type(2)));
    const __amdgpu_buffer_rsrc_t crs = __builtin_amdgcn_make_buffer_rsrc(p.c, 0, (int)p.c_bytes, 0x00020000);
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
        const int m = m0 + (wm * TM + tm) * 32 + (lane & 31);
#pragma unroll
        for (int tn = 0; tn < TN; ++tn)
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
                const int n = n0 + (wn * TN + tn) * 32 + 8 * rr + 4 * g;
                const uint32_t off = m < p.M && n < p.N ? (uint32_t)(((int64_t)m * p.ldc + n) * 2) : 0x80000000u;
                const bf16x4 v = bf16x4{(bf16)acc[tn][tm][4 * rr], (bf16)acc[tn][tm][4 * rr + 1],
                                        (bf16)acc[tn][tm][4 * rr + 2], (bf16)acc[tn][tm][4 * rr + 3]};
                __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(i32x2, v), crs, off, 0, 0);
            }
    }
}

// A wavefront's accumulators by rows: f(m, n, v, d) gets 8 consecutive columns n .. n+7 of row m and what
// d = ahead(m, n) has loaded for them, neighbouring lanes the next 8, so that whole 128-byte lines are
// loaded and stored beside them.  (As they stand a lane has 4 columns of a row and the lanes 32 rows: a layer
// that writes y and z that way and reads a residual spends as long on it as on a contraction of 1500.  4096 x
// 8192 from 2048, GELU: 208 us, 140 through here.)  Each 32 rows go through LDS, 32 x (32 TN + 4) floats of
// the wavefront's own; the pitch puts 16 rows' writes on different banks.  The loads beside 32 rows
// are all issued before the first store (no load is moved over a store to what might be the same memory).
struct Nothing {};
template <typename C, typename A, typename F>
FBL_DEV void by_rows(uint32_t lds, const f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int wm, int wn, A&& ahead, F&& f) {
    constexpr int PITCH = 32 * C::TN + 4, LANES = 4 * C::TN, ROWS = 64 / LANES;  // lanes a row, rows a turn
    const int lane = threadIdx.x & 63, g = lane >> 5;
    const uint32_t mine = lds + (uint32_t)((wn * C::WM + wm) * 32 * PITCH * 4);
    const uint32_t put = mine + (uint32_t)(((lane & 31) * PITCH + 4 * g) * 4);
    const uint32_t get = mine + (uint32_t)((lane / LANES * PITCH + lane % LANES * 8) * 4);
    __syncthreads();  // the stages have been read
    const int nl = n0 + wn * C::TN * 32 + lane % LANES * 8, ml = m0 + wm * C::TM * 32 + lane / LANES;
#pragma unroll
    for (int tm = 0; tm < C::TM; ++tm) {
        decltype(ahead(0, 0)) beside[32 / ROWS];
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) beside[i] = ahead(ml + 32 * tm + i * ROWS, nl);
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
            const f32x4 a = *(const FBL_LDS f32x4*)(uintptr_t)(get + i * ROWS * PITCH * 4);
            const f32x4 b = *(const FBL_LDS f32x4*)(uintptr_t)(get + i * ROWS * PITCH * 4 + 16);
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
            f(ml + 32 * tm + i * ROWS, nl, v, beside[i]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

using i32x2 = int __attribute__((ext_vector_type(2)));
using i32x4 = int __attribute__((ext_vector_type(4)));

FBL_DEV __amdgpu_buffer_rsrc_t span(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, p ? (int)bytes : 0, 0x00020000);
}
constexpr uint32_t kNowhere = 0x80000000u;  // past every span: loads give 0, stores are dropped

// 8 elements of a row, from a column that is a multiple of 8 on
FBL_DEV bf16x8 load8(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}
// ... stored where columns n .. of a row of N (a multiple of 4) have room for them
FBL_DEV void store8(__amdgpu_buffer_rsrc_t r, uint32_t off, const float (&v)[8], int n, int N) {
    bf16x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (bf16)v[e];
    const i32x4 w = __builtin_bit_cast(i32x4, x);
    __builtin_amdgcn_raw_buffer_store_b128(w, r, n + 8 <= N ? off : kNowhere, 0, 0);
    if (N & 4) __builtin_amdgcn_raw_buffer_store_b64(i32x2{w[0], w[1]}, r, n + 4 == N ? off : kNowhere, 0, 0);
}

// Launch of tile I of kGemmTiles.
template <int I, bool AT, bool BT, typename EP>
hipError_t launch_gemm_bf16(const typename EP::Args& p, hipStream_t stream, int splits = 1) {
    constexpr GemmTile t = kGemmTiles[I];
    using C = GemmCfg<t.bm, t.bn, t.bk, t.ns, t.wm, t.wn, t.wk, AT, BT>;
    constexpr auto kernel = &proj_gemm_bf16<t.bm, t.bn, t.bk, t.ns, t.wm, t.wn, t.wk, AT, BT, EP>;
    constexpr int bytes = EP::kByRows && C::ROWS_BYTES > C::BYTES ? C::ROWS_BYTES : C::BYTES;
    const hipError_t once = ensure_dynamic_lds<kernel>(bytes);
    if (once != hipSuccess) return once;
    const int tiles = ((p.M + t.bm - 1) / t.bm) * ((p.N + t.bn - 1) / t.bn);
    hipLaunchKernelGGL(kernel, dim3((tiles + 7) / 8 * 8, splits), dim3(64 * C::NW), bytes, stream, p);
    return hipGetLastError();
}

template <typename EP>
using GemmLauncher = hipError_t (*)(const typename EP::Args&, hipStream_t, int splits);

template <bool AT, bool BT, typename EP, int... I>
constexpr std::array<GemmLauncher<EP>, sizeof...(I)> gemm_launchers(std::integer_sequence<int, I...>) {
    return {&launch_gemm_bf16<I, AT, BT, EP>...};
}

template <bool AT, bool BT, typename EP>
hipError_t launch_gemm_tile(int tile, const typename EP::Args& p, hipStream_t stream) {
    static constexpr auto table = gemm_launchers<AT, BT, EP>(std::make_integer_sequence<int, kGemmTileCount>{});
    return table[tile](p, stream, 1);
}

}  // namespace

}  // namespace fbl
