// tokmap.hpp -- the device side of the token-major index map.
//
// The reshape (B,S,D) -> (B,S,H,HD) and transpose -> (B,H,S,HD) of the
// multi-head attention chain (paper section 4.3.1) only move whole head-dim
// rows, so their composition (section 4.3.2, f3 o f2 o f1) is one affine map
//   offset(b, h, s, i) = b*sb + s*ss + h*sh + i        (sd == 1)
// evaluated once per tile origin; rows of a staged tile then sit ss elements
// apart.  The strides arrive as kernel arguments, already validated on the
// host (sd == 1, head-aligned tiles, 16-byte aligned rows).
#pragma once

#include <stdint.h>

#include "cdna4.hpp"

namespace fbl {

struct TokMap {
    int64_t sb, ss, sh;

    __device__ __host__ __forceinline__ int64_t head_base(int b, int h) const {
        return (int64_t)b * sb + (int64_t)h * sh;
    }
    __device__ __host__ __forceinline__ int64_t offset(int b, int h, int s, int i) const {
        return (int64_t)b * sb + (int64_t)s * ss + (int64_t)h * sh + i;
    }
};

struct MaskArgs {
    int causal;             // key j allowed only for query i >= j
    const int32_t* kv_len;  // nullptr, or device [B]: key j allowed only if j < kv_len[b]
};

struct FwdArgs {
    const void* q;
    const void* k;
    const void* v;
    void* o;
    float* lse;
    TokMap mq, mk, mv, mo;
    int B, S, Hq, Hkv;  // S: query tokens
    int Skv;            // key/value tokens (S for self-attention)
    float scale_log2;  // softmax scale times log2(e)
    MaskArgs mask;
};

struct BwdArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* o;
    const void* dout;
    const float* lse;
    void* dq;
    void* dk;
    void* dv;
    float* stats;      // workspace [B, Hq, 2, S]: rows LSE * log2(e) and sum_k dO*O per query
    void* ds;          // nullptr, or workspace [B, Hq, nk32, nq32] blocks of 32x32 bf16 dS
    int nq32, nk32;    // ceil(S / 32), ceil(Skv / 32)
    TokMap mq, mk, mv, mo, mdo, mdq, mdk, mdv;
    int B, S, Hq, Hkv;  // S: query tokens
    int Skv;            // key/value tokens (S for self-attention)
    float scale;       // softmax scale
    float scale_log2;  // scale * log2(e)
    MaskArgs mask;
    // Key/value pass split: each key block's query iterations are shared by
    // kv_split workgroups, which write fp32 partial dK (times scale) and dV to
    // dkv_part, [2][kv_split][B, Skv, Hkv, D] (dK planes, then dV); a reduction
    // adds them in split order.  1: no split, dK and dV written directly.
    float* dkv_part = nullptr;
    int kv_split = 1;
    // tile ids (attn_tiles.hpp) of the bf16 key/value and dQ passes
    int kv_tile = 5;
    int dq_tile = 7;
};

// Norms of queries and keys for each head and their rotation (qk_norm_rotary.hip).  Of what a call does
// not have the pointers are nullptr: keys (Hkv 0), weights, x in a backward without norm.
struct RotaryArgs {
    const void *q, *k;    // x
    const void *gq, *gk;  // backward: dy
    void *oq, *ok;        // y, or dx
    TokMap mq, mk, mgq, mgk, moq, mok;
    const void *wq, *wk;
    float eps;
    int B, S, Hq, Hkv;
    // dims (0: no rotation) of a head's values turn; turns [dims / 2], 2^64 a turn a position; positions [axis][b][s]
    // by strides, nullptr: s; axes: 2 bits for each pair
    int dims, num_axes;
    const uint64_t* turns;
    const int64_t* pos;
    int64_t pos_axis, pos_batch, pos_token;
    uint64_t axes[2];
    // a wavefront's step is `heads` heads (a power of two) of as many tokens as its rows have room for, a group; a
    // group's heads are `parts` items of `per` steps
    int heads, per, parts;
    int64_t groups;
    int workgroups;
    float* sums;  // backward: [workgroups][2][D] partial sums of the weights' gradients, or nullptr
};

// Matrix product C[M, N] = sum_k A(m, k) B(k, n), bf16 operands, row-major
// storage with leading dimensions in elements.  A is stored [M, K] (or [K, M]
// when read k-major), B [K, N] (or [N, K] when read n-major); a_bytes/b_bytes
// bound the bytes the buffer resources may touch.
struct GemmArgs {
    const void* a;
    const void* b;
    void* c;
    int64_t lda, ldb, ldc;
    int M, N, K;
    uint32_t a_bytes, b_bytes, c_bytes;  // spans of the operands and the result (< 2 GiB)
};

// Layer norm over M rows of N values (strides in elements).  w, b, mean, rstd
// (forward), dx, dw and db may be nullptr.
struct NormArgs {
    const void* x;
    const void* dy;
    const void* w;
    const void* b;
    void* y;
    void* dx;
    void* dw;
    void* db;
    float* mean;
    float* rstd;
    float* part;  // backward: [groups][2][N] partial sums of dw and db, or nullptr
    int64_t ldx, lddy, ldy, lddx;
    int64_t M;
    int N;
    int groups;  // backward: workgroups
    float eps;
};

// A product with a linear layer's epilogue.  Forward: C = act(A B + bias) + res, and the
// pre-activation to z where given; data gradient: C = (A B) act'(z).  bias, res and the
// forward's z may be nullptr; z and res have C's extents.
struct LinearArgs : GemmArgs {
    const void* bias;
    const void* res;
    void* z;
    int64_t ldr, ldz;
    uint32_t res_bytes, z_bytes;
    float* sums;  // data gradient: [groups][N] sums of c down blocks of rows (linear_grad_groups), or nullptr
};

// A gated layer's products with their epilogues.  Forward (gated_gemm.hpp): N is 2F, C is h = act(gate) up of (gate, up) = A B
// + bias, and the factors [M][2F] (up act'(gate), act(gate)) are stored where given.  Data gradient (gated_grad.hip): N is
// F, the product is the gradient of h, C [M][2F] its products with the given factors.
struct GatedArgs : GemmArgs {
    const void* bias;
    void* factors;
    int64_t ldf;
    uint32_t f_bytes;
    float* sums;  // data gradient: [groups][2F] sums of C down blocks of rows (linear_grad_groups), or nullptr
};

// Tensors of one launch over a list of gradients (grad_clip.hip), by value in its arguments: `first` chunks of kGradChunk
// bytes come before each, and first[count] = chunks.
constexpr int kGradChunk = 16384;
constexpr int kGradTensors = 112;
struct GradList {
    struct {
        const void* p;
        void* out;
        int64_t n : 62, f32 : 2;
    } t[kGradTensors];
    int first[kGradTensors + 1];
    int count, chunks;
    int in_place;  // every tensor's output is itself
};
static_assert(sizeof(GradList) <= 3584, "a launch's arguments end at 4 KB");

// dz = dy act'(z) over M x N; part, where not nullptr, gets [groups][N] sums down blocks of `rows` rows.
struct LinearActArgs {
    const void* dy;
    const void* z;
    void* dz;
    float* part;
    int64_t lddy, ldz, lddz;
    int64_t M, rows;
    int N, groups;
};

// Softmax of a linear head over one piece of the vocabulary: the product is X W for the piece's
// columns (bf16: tokens are the rows; fp32: the vocabulary is).  Targets are [top][tokens].
struct HeadArgs : GemmArgs {
    int tokens;
    int shape;          // tile: id of kGemmTiles, or of the fp32 tiles
    int first, width;   // the piece: vocabulary entries first .. first + width - 1
    int top;
    float unit;         // log2(e) / temperature
    const int* index;   // vocabulary entries of the targets, -1: none
    // forward: (maximum, sum of exp2 relative to it) of each tile's columns, both in units of unit times the
    // logit: [tile0 + tile][tokens]; logits of the targets
    float2* part;
    int tile0;
    float* target;
    // backward: dz = row.x (exp2(unit z - row.y) - sum of the targets' weights there), 0 where row.x is
    const float2* row;
    const float* weight;  // of the targets, nullptr: 1
    void* dz;             // [tokens][ldz]; columns width .. ldz - 1 become 0
    int64_t ldz;
    uint32_t dz_bytes;
};

// A product added up over the pieces of its contraction, each perhaps shared by `splits` workgroups a tile:
// sum (fp32, one plane [M][N] a share) is overwritten (first) or added to.  A bf16 product that
// is not split is scaled by *scale and rounded to C with the last piece, and an fp32 one is summed in C.
struct SumArgs : GemmArgs {
    float* sum;
    const float* scale;
    int64_t lds;
    uint32_t sum_bytes;  // of a plane
    int first, last;
    int share, splits;
};

// The small steps around a head's loss, one row (token) of M each.
struct HeadRowArgs {
    int64_t M;
    int V, top;
    const int64_t* labels;  // cross entropy: one target a row
    int64_t ignore;
    const int64_t* given;  // distillation: targets [M][ldi], negative: absent
    int64_t ldi;
    const void* logits;  // the teacher's [M][ldl]
    int64_t ldl;
    int logits_f32;
    float T;
    // rows -> targets
    int* index;     // [top][M]
    float* prob;    // [M][top], weights of the targets (forward: written, backward: read)
    float* weight;  // [top][M], the same for the backward's tiles
    float* entropy; // [M] sum of p log p; nan: a target outside the vocabulary
    float* counted; // [M] 1 or 0
    // backward: factors of the rows
    const float* dloss;
    int64_t dloss_stride;
    const float* total;
    const float* lse_in;
    float2* row;
    float* scale;  // bf16: what dx and dw are multiplied by -- the factor, where it is the same for all rows, and row.x 1 or 0
    // the tiles' parts -> loss
    const float2* part;
    int parts;
    const float* target;  // [top][M]
    float* loss;
    float* lse;
    float* sums;  // [2]: losses, rows counted
    float* mean;  // their quotient (0 where no row counts)
};

}  // namespace fbl
