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
// position is the angle without its whole turns, off by the position times what the kept frequency is off (2^-62 turns at most).
// Its upper 32 bits go to fp32, whose rounding is 2^-26 turns at most (a quarter turn at a time, for fp32, 2^-28); cosine and
// sine come from the hardware for bf16 (good to 2^-19 or so, against 2^-9 of the storage) and from polynomials for fp32.
//
// The weights' gradients stay in registers over all tokens of a wavefront, are added across the lanes
// that hold the same columns and the wavefronts, and go out as one row of partial sums a workgroup, which
// column_sums adds in a fixed order.
//
// bf16 with norms and weights, forward / backward without column_sums: 4096 tokens of 32 + 32 heads of 128 23.2 us (5.8 TB/s) and
// 35.8 (5.6), of 32 + 8 heads of 64 10.9 and 16.5 (3.9 and 3.8: a launch's start and end are a fifth, and of three steps of 16
// heads for 40 the last one's second half repeats work).  16 tokens, the rotation alone, 3.5.  fp32, with column_sums: 4096 tokens of
// 32 + 32 heads of 128 43 (6.2 TB/s) and 83 (4.8), of 32 + 8 heads of 64 14.8 and 25.6.
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

// Sum over the lanes of a wavefront that have the same place in groups of LANES, the same value in each: rotations
// within 16 lanes, then the row swaps.
template <int LANES>
FBL_DEV float place_sum(float x) {
    if constexpr (LANES <= 2) x += dpp<0x122>(x);  // row_ror 2
    if constexpr (LANES <= 4) x += dpp<0x124>(x);  // row_ror 4
    if constexpr (LANES <= 8) x += dpp<0x128>(x);  // row_ror 8
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
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

// A lane's two chunks of a head's row as they are stored, and as numbers.
template <typename T>
struct Two {
    static constexpr int V = Chunk<T>::V;
    Chunk<T> c[2];
    FBL_DEV void load(const T* p, int c0, int c1) {
        c[0] = *reinterpret_cast<const Chunk<T>*>(p + c0);
        c[1] = *reinterpret_cast<const Chunk<T>*>(p + c1);
    }
    FBL_DEV void store(T* p, int c0, int c1) const {
        *reinterpret_cast<Chunk<T>*>(p + c0) = c[0];
        *reinterpret_cast<Chunk<T>*>(p + c1) = c[1];
    }
    FBL_DEV float operator[](int e) const { return (float)c[e / V].v[e % V]; }
    FBL_DEV void set(int e, float x) { c[e / V].v[e % V] = (T)x; }
};
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
__global__ __launch_bounds__(256, (NORM && BWD ? 3 : 5)) void qk_norm_rotary(RotaryArgs p) {
    using H = HeadRow<T, D, NEIGHBOURS>;
    constexpr int V = H::V, LANES = H::LANES, ROWS = H::ROWS;
    constexpr bool SUMS = NORM && BWD;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pair = lane % LANES * V, sub = lane / LANES;
    const int c0 = H::first(pair, p.dims), c1 = H::second(pair, p.dims);
    const bool turns = 2 * pair < p.dims;  // the lane's pairs, all or none (dims are whole lanes)
    const int hsub = sub & (p.heads - 1), tsub = sub / p.heads;  // heads: a power of two, up to ROWS
    const int H_all = p.Hq + p.Hkv;
    const uint32_t tokens = (uint32_t)p.B * (uint32_t)p.S, per_group = ROWS / p.heads;

    // A wavefront's items: blocks of `per` steps of heads of a group of tokens.  While one step is computed the next one's
    // rows, and its tokens' positions, are on the way.
    struct Step {
        uint32_t group, part;  // (the next item is found by adding: a division by parts in every step took a tenth of the time)
        int h0;
        int b, s;   // of the lane's token
        bool there;
    };
    const uint32_t groups = (uint32_t)p.groups, parts = (uint32_t)p.parts, waves = gridDim.x * 4;
    const uint32_t group_step = waves / parts, part_step = waves % parts;
    Two<T> nx, ng;
    // A group's angles, PAIRS of each of its tokens, are made once, 64 of them at a time, a lane each, and go to the lanes
    // that hold the pairs through LDS: made by every lane for itself they were a sixth of the time.
    constexpr int PAIRS = D / 2;
    const int angles = (int)per_group * PAIRS;
    const auto token_at = [&](uint32_t token, int& b, int& s) __attribute__((always_inline)) {
        const uint32_t t = min(token, tokens - 1);
        b = (int)(t / (uint32_t)p.S);
        s = (int)(t - (uint32_t)b * (uint32_t)p.S);
        return token < tokens;
    };
    const int mine = lane % PAIRS, axis = (int)((mine < 32 ? p.axes[0] : p.axes[1]) >> mine % 32 * 2) & 3;
    const int64_t* const positions = p.pos ? p.pos + axis * p.pos_axis : nullptr;
    struct Position {
        int64_t given;
        int s;
        FBL_DEV int64_t of(const int64_t* given_there) const { return given_there ? given : (int64_t)s; }
    };
    const auto position = [&](Position& x, uint32_t group, int i) __attribute__((always_inline)) {  // of this lane's i-th angle
        int b;
        token_at(group * per_group + (uint32_t)(i * 64 + lane) / PAIRS, b, x.s);
        if (p.pos) x.given = positions[b * p.pos_batch + x.s * p.pos_token];
    };
    Position at;
    const auto enter = [&](Step& k) __attribute__((always_inline)) {
        k.there = token_at(k.group * per_group + tsub, k.b, k.s);
        k.h0 = (int)k.part * p.per * p.heads;
        if (p.dims) position(at, k.group, 0);
    };
    // A tensor's address and strides in bytes, in scalar registers.  (The compiler would choose between the addresses of the
    // arguments for queries and for keys, lane by lane, and load from there in every step, behind the rows on the way, which the
    // stores then wait for: 4096 tokens of 32 + 32 heads of 128 53.9 us backward instead of 36.9.)
    using Bytes = __attribute__((address_space(1))) char*;
    struct Side {
        Bytes p;
        int64_t sb, ss, sh;
    };
    const auto side = [](const void* ptr, const TokMap& m) __attribute__((always_inline)) {
        constexpr int64_t es = sizeof(T);
        Side t{(Bytes)ptr, m.sb * es, m.ss * es, m.sh * es};
        asm("" : "+s"(t.p), "+s"(t.sb), "+s"(t.ss), "+s"(t.sh));
        return t;
    };
    const Side xq = side(p.q, p.mq), xk = side(p.k, p.mk), gq = side(p.gq, p.mgq), gk = side(p.gk, p.mgk), oq = side(p.oq, p.moq),
               ok = side(p.ok, p.mok);
    const auto row = [&](const Side& q, const Side& k, const Step& at) __attribute__((always_inline)) {
        const auto address = [&](const Side& t, int h) __attribute__((always_inline)) {
            return t.p + (at.b * t.sb + at.s * t.ss + h * t.sh);
        };
        const bool keys = at.h0 >= p.Hq;  // the same for the wavefront, as are all its heads but in one step of a token
        const Side t{keys ? k.p : q.p, keys ? k.sb : q.sb, keys ? k.ss : q.ss, keys ? k.sh : q.sh};
        const int h = min(at.h0 + hsub, H_all - 1);
        Bytes a = address(t, keys ? h - p.Hq : h);
        if (!keys && h >= p.Hq) a = address(k, h - p.Hq);
        return (T*)a;
    };
    const auto fetch = [&](const Step& k) __attribute__((always_inline)) {
        if (!BWD || NORM) nx.load(row(xq, xk, k), c0, c1);
        if (BWD) ng.load(row(gq, gk, k), c0, c1);
    };
    Step cur{}, next{};
    const uint32_t first_item = blockIdx.x * 4 + (uint32_t)wave;
    next.group = first_item / parts, next.part = first_item % parts;
    if (next.group < groups) {
        enter(next);
        fetch(next);
    }

    // weights and frequencies in LDS: in registers, unpacked for every step, they are what keeps a third wavefront out
    __shared__ T lw[2][D] __attribute__((aligned(16)));
    __shared__ uint64_t lfreq[PAIRS] __attribute__((aligned(16)));
    if (NORM && threadIdx.x < 2 * D) {
        const int k = threadIdx.x / D, c = threadIdx.x % D;
        const T* const wp = static_cast<const T*>(k ? p.wk : p.wq);
        lw[k][c] = wp ? wp[c] : (T)1.f;
    }
    __shared__ float langle[4][2][V * 64] __attribute__((aligned(16)));  // [wavefront][cosine, sine][token of the group][pair]
    if (threadIdx.x < PAIRS) lfreq[threadIdx.x] = 2 * (int)threadIdx.x < p.dims ? p.turns[threadIdx.x] : 0;
    __syncthreads();
    float sum[2][2 * V];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) sum[k][e] = 0.f;
    float cs[V], sn[V];
    bool entered = true;
    // the first rows are there before the loop: else the compiler waits in every step as the first one has to, for all stores
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)

    while (next.group < groups) {
        cur = next;
        Two<T> x = nx, g = ng;
        if (entered && p.dims) {
            float* const lc = langle[wave][0];
            float* const ls = langle[wave][1];
            for (int i = 0; i * 64 < angles; ++i) {
                const int k = i * 64 + lane;
                float c, n;
                // (a group of more than 128 / D tokens, of a few heads, waits for the positions behind them)
                Position where = at;
                if (i > 0) {
                    position(where, cur.group, i);
                    __builtin_amdgcn_s_waitcnt(0x0f70);
                }
                turned<sizeof(T) == 2>((int32_t)((uint64_t)where.of(p.pos) * lfreq[mine] >> 32), c, n);
                if (k < angles) lc[k] = c, ls[k] = n;
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int i = 0; i < V; ++i) cs[i] = lc[tsub * PAIRS + pair + i], sn[i] = ls[tsub * PAIRS + pair + i];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        next.h0 += p.heads;
        entered = next.h0 >= min(H_all, ((int)cur.part + 1) * p.per * p.heads);
        if (entered) {
            next.group += group_step, next.part += part_step;
            if (next.part >= parts) next.part -= parts, ++next.group;
            if (next.group < groups) enter(next);
        }
        if (next.group < groups) fetch(next);

        // Lanes behind the last head or token do that one's work over again and store the same: a store that some lanes leave
        // out is one that the next step's loads cannot be told apart from, and waits for.
        const int h = min(cur.h0 + hsub, H_all - 1);
        const bool live = cur.there && cur.h0 + hsub < H_all, key = h >= p.Hq;
        float r = 1.f;
        if constexpr (NORM) {
            float q = 0.f;
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) q = __builtin_fmaf(x[e], x[e], q);
            r = 1.f / sqrtf(group_sum<LANES>(q) * (1.f / D) + p.eps);
        }
        float y[2 * V];
        if constexpr (!BWD) {
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) y[e] = x[e];
            if constexpr (NORM) {
                Two<T> wh;
                wh.load(lw[key], c0, c1);
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) y[e] *= r * wh[e];
            }
            if (turns) rotate<H, false, V>(y, cs, sn);  // (an infinite value that does not turn stays alone)
        } else {
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) y[e] = g[e];
            if (turns) rotate<H, true, V>(y, cs, sn);
            if constexpr (NORM) {
                Two<T> wh;
                wh.load(lw[key], c0, c1);
                const int first = cur.h0, last = min(H_all, cur.h0 + p.heads) - 1;
                const bool all_q = last < p.Hq, all_k = first >= p.Hq;  // the same for the wavefront
                float m = 0.f, t[2 * V];
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    t[e] = y[e] * (x[e] * r);
                    m = __builtin_fmaf(t[e], wh[e], m);
                }
                // (chosen, not multiplied: 0 times an infinite value that its own lane adds would make the sum nan)
                const auto add = [&](int k) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) sum[k][e] += live ? t[e] : 0.f;
                };
                if (all_q) add(0);
                else if (all_k) add(1);
                else {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) sum[0][e] += live && !key ? t[e] : 0.f, sum[1][e] += live && key ? t[e] : 0.f;
                }
                m = group_sum<LANES>(m) * (1.f / D);
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) y[e] = r * (y[e] * wh[e] - x[e] * r * m);
            }
        }
        Two<T> o;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) o.set(e, y[e]);
        o.store(row(oq, ok, cur), c0, c1);
    }

    if constexpr (SUMS) {
        if (!p.sums) return;
        __shared__ float part[4][2][D];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) {
                sum[k][e] = place_sum<LANES>(sum[k][e]);
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
