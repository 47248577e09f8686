// kernels.hpp -- launchers of the attention kernels (host-callable).
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "attn_tiles.hpp"
#include "gemm_tiles.hpp"
#include "tokmap.hpp"

namespace fbl {

// Raise a kernel's dynamic-LDS limit before its first launch on each device
// (the attribute is held per device).  One flag word per kernel; devices 64
// and up set the attribute on every launch.
template <auto Kernel>
hipError_t ensure_dynamic_lds(int bytes) {
    static std::atomic<uint64_t> done{0};  // bit d: set on device d
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t(1) << dev) : 0;
    if (bit && (done.load(std::memory_order_acquire) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && bit) done.fetch_or(bit, std::memory_order_release);
    return e;
}

typedef __bf16 bf16;

// Forward, 32 queries per workgroup: O and LSE from Q, K, V; D in {32, 64, 128}.
template <typename T, int D>
hipError_t launch_attn_fwd_streams(const FwdArgs& a, hipStream_t stream);

// Forward for bf16 storage with forward tile `tile` of kAttnTiles.
template <int D>
hipError_t launch_attn_fwd_bf16(const FwdArgs& a, int tile, hipStream_t stream);

// Backward: per-row statistics (LSE * log2(e), D = rowsum(dO * O)), then the
// key/value-major pass (dK, dV) and the query-major pass (dQ).
// `phases`: bit 0 statistics, bit 1 kv pass, bit 2 q pass.
template <typename T, int D>
hipError_t launch_attn_bwd(const BwdArgs& a, unsigned phases, hipStream_t stream);

// The whole backward in one launch, 32 keys or 32 queries per workgroup: dK and
// dV, and dQ (recomputing S and dP), each with its row statistics.
template <typename T, int D>
hipError_t launch_attn_bwd_streams(const BwdArgs& a, hipStream_t stream);

// The same for key/value sequences of at most 128 tokens, one workgroup per
// (batch, kv head); fp32 at D = 32 and 64 only.
template <typename T, int D>
hipError_t launch_attn_bwd_fused(const BwdArgs& a, hipStream_t stream);

// Backward passes for fp32 storage: dK and dV, and dQ (recomputing S and dP).
template <int D>
hipError_t launch_attn_bwd_kv_f32(const BwdArgs& a, hipStream_t stream);
template <int D>
hipError_t launch_attn_bwd_q_f32(const BwdArgs& a, hipStream_t stream);

// fp32 passes in 128-row workgroups for short walks (attn_rows_f32.hip), the forward at
// d = 64 and 128 and the backward's passes at d = 128, and whether they are the faster ones.
bool f32_rows_fwd(const FwdArgs& a, int D);
bool f32_rows_kv(const BwdArgs& a);
bool f32_rows_q(const BwdArgs& a);
template <int D>
hipError_t launch_attn_fwd_rows_f32(const FwdArgs& a, hipStream_t stream);
hipError_t launch_attn_bwd_kv_rows_f32(const BwdArgs& a, hipStream_t stream);
hipError_t launch_attn_bwd_q_rows_f32(const BwdArgs& a, hipStream_t stream);

// Key/value-major backward pass for bf16 storage (software-pipelined kernel)
// with kv tile `tile` of kAttnTiles (its split is a.kv_split).
template <int D>
hipError_t launch_attn_bwd_kv_bf16(const BwdArgs& a, int tile, hipStream_t stream);

// Query-major backward pass (dQ) for bf16 storage (software-pipelined kernel),
// recomputing S and dP.
template <int D>
hipError_t launch_attn_bwd_q_bf16(const BwdArgs& a, hipStream_t stream);

// dQ for bf16 storage from the dS blocks the key/value-major pass stored in
// the workspace (a.ds != nullptr), with dQ tile `tile` of kAttnTiles.
template <int D>
hipError_t launch_attn_bwd_dq_bf16(const BwdArgs& a, int tile, hipStream_t stream);

// Projection matrix products (proj_gemm.hip).  Output tile shapes:
// `tile` indexes kGemmTiles (gemm_tiles.hpp).
// a_kmajor: A stored [K, M]; b_nmajor: B stored [N, K].
hipError_t launch_proj_gemm(int a_kmajor, int b_nmajor, int tile, const GemmArgs& p, hipStream_t stream);
// The same products for fp32 storage (proj_gemm_f32.hip); the tile follows from the shape.
hipError_t launch_proj_gemm_f32(int a_kmajor, int b_nmajor, const GemmArgs& p, hipStream_t stream);
// That tile (bm, bn, bk, wavefronts, wk) and the workgroups it takes, for an M x N output.
void proj_gemm_f32_info(const GemmArgs& p, int32_t* info);

// Layer norm (layer_norm.hip); f32: fp32 storage, else bf16.  N up to kNormMaxWidth.  The
// backward ends with launch_column_sums where a.part is given.
constexpr int kNormMaxWidth = 16384;
hipError_t launch_layer_norm_fwd(int f32, const NormArgs& a, hipStream_t stream);
hipError_t launch_layer_norm_bwd(int f32, const NormArgs& a, hipStream_t stream);
// Rows of N values that one workgroup holds at a time.
int layer_norm_slots(int f32, int N);
bool layer_norm_wide(int f32, int N);  // a row takes 16 wavefronts

// out0[n], out1[n] (K = 1 or 2 of them, each may be nullptr) = sums over `groups` of part [groups][K][N].
hipError_t launch_column_sums(int f32, const float* part, int groups, int K, int N, void* out0, void* out1,
                              hipStream_t stream);

// Norms of queries and keys and their rotation (qk_norm_rotary.hip), D 32, 64 or 128; forward, or with `bwd` the
// gradients.  rotary_rows: heads that a wavefront has room for in a step.
int rotary_rows(int f32, int D);
hipError_t launch_qk_norm_rotary(int f32, int D, int neighbours, int norm, int bwd, const RotaryArgs& p, hipStream_t stream);

// Products with a linear layer's epilogue (linear_gemm.hpp), ACT of act.hpp: the forward, or with
// `grad` the data gradient times act'.  bf16 with `tile` of kGemmTiles; fp32 with its own choice.
template <int ACT>
hipError_t launch_linear_gemm(int grad, int tile, const LinearArgs& p, hipStream_t stream);
hipError_t launch_weight_gemm(int tile, const LinearArgs& p, hipStream_t stream);  // A stored k-major, no epilogue
template <int ACT>
hipError_t launch_linear_gemm_f32(int grad, const LinearArgs& p, hipStream_t stream);
// Rows of LinearArgs::sums that a data gradient with p's extents writes, one for each wavefront's rows of a tile
// (tile: of the launch, bf16), at most M / 32 + 4.
int64_t linear_grad_groups(int f32, int tile, const GemmArgs& p);
// y and z of a forward product, or with `grad` dx of a data gradient, from its planes (launch_sum_gemm), for few rows
// (linear_finish.hip); p.sums: M rows.
hipError_t launch_linear_finish(int f32, int act, int grad, const LinearArgs& p, const float* planes, int splits,
                                hipStream_t stream);
// The gated layer's products: the forward (gated_gemm.hpp) and the data gradient (gated_grad.hip).
template <int ACT>
hipError_t launch_gated_gemm(int tile, const GatedArgs& p, hipStream_t stream);
template <int ACT>
hipError_t launch_gated_gemm_f32(const GatedArgs& p, hipStream_t stream);
hipError_t launch_gated_grad(int f32, int tile, const GatedArgs& p, hipStream_t stream);
// The same from a product's planes [splits][M][2F], or of the data gradient [splits][M][F] (gated_finish.hip); p.sums: M
// rows.
hipError_t launch_gated_finish(int f32, int act, const GatedArgs& p, const float* planes, int splits, hipStream_t stream);
hipError_t launch_gated_grad_finish(int f32, const GatedArgs& p, const float* planes, int splits, hipStream_t stream);
hipError_t launch_linear_act_bwd(int f32, int act, const LinearActArgs& a, hipStream_t stream);

// Sums of squares of a list's tensors, one for each workgroup; the norm from n of them; out = g min(1, limit / (norm +
// 1e-6)), the norm being that of n sums, which is then written where norm is not nullptr, or, sums nullptr, norm's.
hipError_t launch_grad_squares(const GradList& a, double* sums, int workgroups, hipStream_t stream);
hipError_t launch_grad_norm(const double* sums, int n, float* norm, hipStream_t stream);
hipError_t launch_grad_scale(const GradList& a, const double* sums, int n, float* norm, float limit, int workgroups,
                             hipStream_t stream);

// Softmax losses of a linear head (head_gemm.hip, head_rows.hip); table: the weight is stored
// [V, K], else [K, V].
constexpr int kHeadMaxTop = 1024;
// The tile (HeadArgs::shape) for M tokens and V entries, and the entries it spans.
int head_tile(int f32, int table, int64_t M, int64_t V, int64_t K);
int head_tile_width(int f32, int tile);
hipError_t launch_head_fwd(int f32, int table, HeadArgs p, hipStream_t stream);
hipError_t launch_head_grad(int f32, int table, HeadArgs p, hipStream_t stream);
// bf16 with `tile` of kGemmTiles where it is not split.
hipError_t launch_sum_gemm(int a_kmajor, int b_nmajor, int tile, const SumArgs& p, hipStream_t stream);
hipError_t launch_sum_gemm_f32(int b_nmajor, const SumArgs& p, hipStream_t stream);
// Workgroups that should share the contraction kc of an M x N product's tiles, which alone would run with `tile` (bf16).
int sum_splits(int f32, int b_nmajor, int64_t M, int64_t N, int64_t kc, int tile);
// The same for a weight gradient of K x N over M tokens (bf16: alone with `tile`), and its launch for p.splits > 1.
constexpr int64_t kWeightSplitMax = (int64_t)1 << 19;  // K N
int weight_splits(int f32, int64_t M, int64_t K, int64_t N, int tile);
hipError_t launch_weight_shares(int f32, const SumArgs& p, hipStream_t stream);
// C [M][ldc] = scale * the sum of the planes [splits][M][N] (scale nullptr: 1).
hipError_t launch_sum_planes(int f32, const float* planes, int splits, int64_t M, int64_t N, const float* scale, void* c,
                             int64_t ldc, hipStream_t stream);
hipError_t launch_head_targets(const HeadRowArgs& a, hipStream_t stream);       // forward: targets, probabilities
hipError_t launch_head_join(const HeadRowArgs& a, hipStream_t stream);          // parts -> loss, lse, sums
hipError_t launch_head_grad_rows(const HeadRowArgs& a, hipStream_t stream);     // backward: targets, factors

// The tile of kGemmTiles that FBL_GEMM_TILE_AUTO names for a projection product (api.cpp).
int proj_auto_tile(uint32_t op, int64_t M, int64_t K, int64_t N);
// The same for a weight gradient whose tiles are written by rows.
int weight_tile(int64_t M, int64_t K, int64_t N);
// Both as they are without fbl_proj_tune: functions of the shape, by which workspaces are laid out.
int proj_untuned_tile(uint32_t op, int64_t M, int64_t K, int64_t N);
int weight_untuned_tile(int64_t M, int64_t K, int64_t N);

// Diagnostic: offsets of a token-major tensor computed by the device index map.
hipError_t launch_layout_map(const TokMap& m, int B, int H, int S, int D, int64_t* out, hipStream_t stream);

}  // namespace fbl
