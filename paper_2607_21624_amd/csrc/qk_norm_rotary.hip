// qk_norm_rotary.hip -- norms of queries and keys for each head and their rotation by
// position, forward and backward, gfx950.
//
//   h = x r w,  r = 1 / sqrt(mean(x^2) + eps)          over a head's D values, or h = x
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t)   for each of dims / 2 pairs of h, t = position * frequency
// and back: g = the same by -t of dy,  dw = sum over tokens and heads of g x r,
//   dx = r (g w - x r mean(g w x r))
//
// Bound by memory: x is read and y written once, dy and (for the norm) x read and dx written.  A head's row is
// shared by D / 2V lanes that hold two 16-byte chunks of V values each, which are the two members of the lane's V pairs
// (halves), or V / 2 pairs each (neighbours): a pair never leaves its lane, and a lane keeps the same pairs for all heads
// and tokens.  So the angle's cosine and sine are made once a token, and w stays in registers.  A wavefront takes
// whole tokens, queries and keys in one sequence of heads; few tokens are shared by heads instead, and few heads leave
// room for several tokens.
//
// The angle is in turns of 64-bit fixed point: frequency / 2 pi times 2^64, so that the wrapped product with any 64-bit
// position is the angle without its whole turns, off by position * 2^-65 turns.  The cosine and sine of its upper 32 bits
// come from the hardware for bf16 (good to 2^-19 or so, against 2^-9 of the storage) and from polynomials for fp32.
//
// The weights' gradients stay in registers over all tokens of a wavefront, are added across the lanes
// that hold the same columns and the wavefronts, and go out as one row of partial sums a workgroup, which
// column_sums adds in a fixed order.
#include "kernels.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

// Sum over groups of LANES (2 .. 16) consecutive lanes.
template <int LANES>
FBL_DEV float group_sum(float x) {
    x += dpp<0xB1>(x);                               // quad_perm 1 0 3 2
    if constexpr (LANES >= 4) x += dpp<0x4E>(x);     // quad_perm 2 3 0 1
    if constexpr (LANES >= 8) x += dpp<0x141>(x);    // row_half_mirror
    if constexpr (LANES >= 16) x += dpp<0x140>(x);   // row_mirror
    return x;
}

// Cosine and sine of f / 2^32 turns.
template <bool FAST>
FBL_DEV void turned(int32_t f, float& c, float& s) {
    if constexpr (FAST) {
        const float t = (float)f * 0x1p-32f;
        c = __builtin_amdgcn_cosf(t);
        s = __builtin_amdgcn_sinf(t);
    } else {
        // the nearest quarter turn apart, the rest at most pi / 4: Taylor's series, good to 2e-9 and 3e-10 there
        const uint32_t q = ((uint32_t)f + 0x20000000u) >> 30;
        const float y = (float)(int32_t)((uint32_t)f - (q << 30)) * (float)(6.283185307179586 / 4294967296.0), z = y * y;
        float sn = __builtin_fmaf(z, 2.7557319e-6f, -1.98412698e-4f);
        sn = __builtin_fmaf(z, sn, 8.3333333e-3f);
        sn = __builtin_fmaf(z, sn, -1.66666667e-1f);
        sn = __builtin_fmaf(z * y, sn, y);
        float cs = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
        cs = __builtin_fmaf(z, cs, -1.38888889e-3f);
        cs = __builtin_fmaf(z, cs, 4.16666667e-2f);
        cs = __builtin_fmaf(z, cs, -0.5f);
        cs = __builtin_fmaf(z, cs, 1.f);
        const float u = q & 1 ? sn : cs, v = q & 1 ? cs : sn;
        c = (q + 1) & 2 ? -u : u;
        s = q & 2 ? -v : v;
    }
}

template <typename T>
struct Chunk {
    static constexpr int V = 16 / (int)sizeof(T);
    T v[V] __attribute__((aligned(16)));
};

template <typename T, int D, bool NEIGHBOURS>
struct HeadRow {
    static constexpr int V = Chunk<T>::V, LANES = D / (2 * V), ROWS = 64 / LANES;  // lanes a head, heads a wavefront
    // Elements of a lane's two chunks within the head, where its pairs p .. p + V - 1 are.  (Past the rotated
    // dims the values are pairs of angle 0, halves of what is left.)
    static FBL_DEV int first(int p, int dims) {
        if constexpr (NEIGHBOURS) return 2 * p;
        return p < dims / 2 ? p : dims / 2 + p;
    }
    static FBL_DEV int second(int p, int dims) {
        if constexpr (NEIGHBOURS) return 2 * p + V;
        return p < dims / 2 ? dims / 2 + p : D / 2 + p;
    }
    // The pair members' place among the lane's 2V values: (a, b) of pair i
    static constexpr int a(int i) { return NEIGHBOURS ? 2 * i : i; }
    static constexpr int b(int i) { return NEIGHBOURS ? 2 * i + 1 : V + i; }
};

template <typename T>
FBL_DEV void load2(float (&x)[2 * Chunk<T>::V], const T* p, int c0, int c1) {
    using C = Chunk<T>;
    const C u = *reinterpret_cast<const C*>(p + c0), v = *reinterpret_cast<const C*>(p + c1);
#pragma unroll
    for (int e = 0; e < C::V; ++e) x[e] = (float)u.v[e], x[C::V + e] = (float)v.v[e];
}
template <typename T>
FBL_DEV void store2(const float (&x)[2 * Chunk<T>::V], T* p, int c0, int c1) {
    using C = Chunk<T>;
    C u, v;
#pragma unroll
    for (int e = 0; e < C::V; ++e) u.v[e] = (T)x[e], v.v[e] = (T)x[C::V + e];
    *reinterpret_cast<C*>(p + c0) = u;
    *reinterpret_cast<C*>(p + c1) = v;
}

// (a, b) by the angle, or BACK by its negative
template <typename H, bool BACK, int V>
FBL_DEV void rotate(float (&x)[2 * V], const float (&c)[V], const float (&s)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float a = x[H::a(i)], b = x[H::b(i)], t = BACK ? -s[i] : s[i];
        x[H::a(i)] = __builtin_fmaf(a, c[i], -(b * t));
        x[H::b(i)] = __builtin_fmaf(b, c[i], a * t);
    }
}

template <typename T, int D, bool NEIGHBOURS, bool NORM, bool BWD>
__global__ __launch_bounds__(256) void qk_norm_rotary(RotaryArgs p) {
    using H = HeadRow<T, D, NEIGHBOURS>;
    constexpr int V = H::V, LANES = H::LANES, ROWS = H::ROWS;
    constexpr bool SUMS = NORM && BWD;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int pair = lane % LANES * V, sub = lane / LANES;
    const int c0 = H::first(pair, p.dims), c1 = H::second(pair, p.dims);
    const bool turns = 2 * pair < p.dims;  // the lane's pairs, all or none (dims are whole lanes)
    const int hsub = sub & (p.heads - 1), tsub = sub / p.heads;  // heads: a power of two, up to ROWS
    const int H_all = p.Hq + p.Hkv;
    const int64_t tokens = (int64_t)p.B * p.S;

    // weights of the lane's columns
    float w[2][2 * V];
    float sum[2][2 * V];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const T* wp = static_cast<const T*>(k ? p.wk : p.wq);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) w[k][e] = 1.f, sum[k][e] = 0.f;
        if (NORM && wp) {
#pragma unroll
            for (int e = 0; e < V; ++e) w[k][e] = (float)wp[c0 + e], w[k][V + e] = (float)wp[c1 + e];
        }
    }
    uint64_t freq[V];
    int axis[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        freq[i] = turns ? p.turns[pair + i] : 0;
        axis[i] = (int)(p.axes[(pair + i) / 32] >> (pair + i) % 32 * 2) & 3;
    }

    // a wavefront's items: blocks of `per` steps of heads of a group of tokens
    const int64_t items = p.groups * p.parts;
    for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < items; item += (int64_t)gridDim.x * 4) {
        const int64_t group = item / p.parts;
        const int part = (int)(item - group * p.parts);
        const int64_t token = group * (ROWS / p.heads) + tsub;
        const bool there = token < tokens;
        const int64_t b = there ? token / p.S : 0, s = there ? token - b * p.S : 0;
        float cs[V], sn[V];
        if (p.dims) {
            int64_t at[4] = {s, s, s, s};
            if (p.pos) {
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    if (a < p.num_axes) at[a] = p.pos[a * p.pos_axis + b * p.pos_batch + s * p.pos_token];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                int64_t n = at[0];
                if (p.num_axes > 1) n = axis[i] == 0 ? at[0] : axis[i] == 1 ? at[1] : axis[i] == 2 ? at[2] : at[3];
                turned<sizeof(T) == 2>((int32_t)((uint64_t)n * freq[i] >> 32), cs[i], sn[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) cs[i] = 1.f, sn[i] = 0.f;
        }
        const int h1 = min(H_all, (part + 1) * p.per * p.heads);
        for (int h0 = part * p.per * p.heads; h0 < h1; h0 += p.heads) {
            const int h = h0 + hsub;
            const bool live = there && h < H_all, key = h >= p.Hq;
            const int hk = key ? h - p.Hq : h;
            float x[2 * V], g[2 * V];
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) x[e] = g[e] = 0.f;
            if (live) {
                if (!BWD || NORM)
                    load2<T>(x, static_cast<const T*>(key ? p.k : p.q) + (key ? p.mk : p.mq).offset((int)b, hk, (int)s, 0), c0, c1);
                if (BWD)
                    load2<T>(g, static_cast<const T*>(key ? p.gk : p.gq) + (key ? p.mgk : p.mgq).offset((int)b, hk, (int)s, 0), c0, c1);
            }
            float r = 1.f;
            if constexpr (NORM) {
                float q = 0.f;
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) q = __builtin_fmaf(x[e], x[e], q);
                r = 1.f / sqrtf(group_sum<LANES>(q) * (1.f / D) + p.eps);
                if (!live) r = 0.f;  // (eps may be 0)
            }
            if constexpr (!BWD) {
                if constexpr (NORM) {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) x[e] *= r * (key ? w[1][e] : w[0][e]);
                }
                if (turns) rotate<H, false, V>(x, cs, sn);  // (an infinite value that does not turn stays alone)
            } else {
                if (turns) rotate<H, true, V>(g, cs, sn);
                if constexpr (NORM) {
                    float m = 0.f;
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) {
                        const float xh = x[e] * r, t = g[e] * xh;
                        sum[0][e] += key ? 0.f : t;
                        sum[1][e] += key ? t : 0.f;
                        g[e] *= key ? w[1][e] : w[0][e];
                        m = __builtin_fmaf(g[e], xh, m);
                        x[e] = xh;
                    }
                    m = group_sum<LANES>(m) * (1.f / D);
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) x[e] = r * (g[e] - x[e] * m);
                } else {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) x[e] = g[e];
                }
            }
            if (live)
                store2<T>(x, static_cast<T*>(key ? p.ok : p.oq) + (key ? p.mok : p.moq).offset((int)b, hk, (int)s, 0), c0, c1);
        }
    }

    if constexpr (SUMS) {
        if (!p.sums) return;
        __shared__ float part[4][2][D];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) sum[k][e] += __shfl_xor(sum[k][e], d);
                if (lane < LANES) part[wave][k][(e < V ? c0 : c1) + e % V] = sum[k][e];
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * D; i += 256) {
            const int k = i / D, c = i % D;
            p.sums[(int64_t)blockIdx.x * 2 * D + i] = (part[0][k][c] + part[1][k][c]) + (part[2][k][c] + part[3][k][c]);
        }
    }
}

template <typename T, int D, bool NEIGHBOURS>
hipError_t launch(int norm, int bwd, const RotaryArgs& p, hipStream_t s) {
    const dim3 grid((unsigned)p.workgroups), block(256);
    if (norm && bwd) hipLaunchKernelGGL((qk_norm_rotary<T, D, NEIGHBOURS, true, true>), grid, block, 0, s, p);
    else if (norm) hipLaunchKernelGGL((qk_norm_rotary<T, D, NEIGHBOURS, true, false>), grid, block, 0, s, p);
    else if (bwd) hipLaunchKernelGGL((qk_norm_rotary<T, D, NEIGHBOURS, false, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((qk_norm_rotary<T, D, NEIGHBOURS, false, false>), grid, block, 0, s, p);
    return hipGetLastError();
}

template <typename T>
hipError_t for_dim(int D, int neighbours, int norm, int bwd, const RotaryArgs& p, hipStream_t s) {
    switch (D) {
        case 32: return neighbours ? launch<T, 32, true>(norm, bwd, p, s) : launch<T, 32, false>(norm, bwd, p, s);
        case 64: return neighbours ? launch<T, 64, true>(norm, bwd, p, s) : launch<T, 64, false>(norm, bwd, p, s);
        default: return neighbours ? launch<T, 128, true>(norm, bwd, p, s) : launch<T, 128, false>(norm, bwd, p, s);
    }
}

}  // namespace

int rotary_rows(int f32, int D) { return 64 / (D / (f32 ? 8 : 16)); }

hipError_t launch_qk_norm_rotary(int f32, int D, int neighbours, int norm, int bwd, const RotaryArgs& p, hipStream_t s) {
    return f32 ? for_dim<float>(D, neighbours, norm, bwd, p, s) : for_dim<bf16>(D, neighbours, norm, bwd, p, s);
}

}  // namespace fbl
