// head_rows.hip -- softmax losses of a linear head: the small steps around the
// products of head_gemm.hip, gfx950.
//
//   targets    the teacher's probabilities p = softmax(t / T) over a row's entries and
//              sum p log p; targets laid out [top][M], as the tiles read them
//   join       the tiles' (maximum, sum) pairs -> lse, and the row's loss
//                T^2 (sum p log p + lse - sum p z / T)     (cross entropy: one p of 1, T = 1)
//              then the sum of the losses and the rows counted
//   grad rows  the rows' factors and targets for the backward's tiles
//
// All of them move a few bytes a row or (join) 8 bytes a row and tile, and are bound by
// the latency of their loads.
#include "kernels.hpp"
#include "rows.hpp"

namespace fbl {

namespace {

FBL_DEV float wave_max(float x) {
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    x = fmaxf(x, dpp<0x140>(x));
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
FBL_DEV float quiet_nan() { return __int_as_float(0x7fc00000); }

// A label's place in the vocabulary: counted unless it is `ignore`, nowhere (and then the loss is nan)
// outside 0 .. V-1.
struct Label {
    bool counted, good;
    int at;
};
FBL_DEV Label label_of(const HeadRowArgs& a, int64_t m) {
    const int64_t v = a.labels[m];
    const bool on = v != a.ignore, good = v >= 0 && v < a.V;
    return {on, good, on && good ? (int)v : -1};
}

__global__ __launch_bounds__(256) void head_labels(HeadRowArgs a) {
    const int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (m >= a.M) return;
    const Label l = label_of(a, m);
    a.index[m] = l.at;
    a.entropy[m] = l.counted && !l.good ? quiet_nan() : 0.f;
    a.counted[m] = l.counted ? 1.f : 0.f;
}

template <typename T>
__global__ __launch_bounds__(256) void head_teacher(HeadRowArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= a.M) return;
    const int64_t* given = a.given + m * a.ldi;
    const T* logits = static_cast<const T*>(a.logits) + m * a.ldl;
    const auto entry = [&](int j) { return j < a.top && given[j] >= 0 ? (float)logits[j] / a.T : -INFINITY; };
    float top = -INFINITY;
    bool bad = false;
    for (int j = lane; j < a.top; j += 64) {
        top = fmaxf(top, entry(j));
        bad |= given[j] >= a.V;
        a.index[(int64_t)j * a.M + m] = given[j] >= 0 && given[j] < a.V ? (int)given[j] : -1;
    }
    top = wave_max(top);
    float sum = 0.f;
    for (int j = lane; j < a.top; j += 64) {
        const float t = entry(j);
        sum += t == -INFINITY ? 0.f : expf(t - top);
    }
    sum = lane_sum<64>(sum);
    const float lg = logf(sum);
    float ent = 0.f;
    for (int j = lane; j < a.top; j += 64) {
        const float t = entry(j), p = t == -INFINITY ? 0.f : expf(t - top) / sum;
        a.prob[m * a.top + j] = p;
        ent += p == 0.f ? 0.f : p * (t - top - lg);
    }
    ent = lane_sum<64>(ent);
    const bool any_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (lane == 0) {
        a.entropy[m] = any_bad ? quiet_nan() : sum == 0.f ? 0.f : ent;
        a.counted[m] = sum == 0.f && !any_bad ? 0.f : 1.f;
    }
}

// 16 rows a workgroup: 64 threads each walk a row's parts (16 rows side by side: 128-byte lines), then a
// wavefront joins them and sums over the targets.
__global__ __launch_bounds__(1024) void head_join(HeadRowArgs a) {
    __shared__ float2 s[16][65];
    const int64_t m0 = (int64_t)blockIdx.x * 16;
    {
        const int r = threadIdx.x & 15, l = threadIdx.x >> 4;
        const int64_t m = m0 + r;
        float top = -INFINITY, sum = 0.f;
        if (m < a.M)
            for (int p = l; p < a.parts; p += 64) {
                const float2 o = a.part[(int64_t)p * a.M + m];
                const float t = fmaxf(top, o.x), ref = t == -INFINITY ? 0.f : t;
                sum = sum * fast_exp2(top - ref) + o.y * fast_exp2(o.x - ref);
                top = t;
            }
        s[r][l] = make_float2(top, sum);
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, r = threadIdx.x >> 6;
    const int64_t m = m0 + r;
    if (m >= a.M) return;
    const float2 o = s[r][lane];
    const float top = wave_max(o.x), ref = top == -INFINITY ? 0.f : top;
    const float sum = lane_sum<64>(o.y * fast_exp2(o.x - ref));
    const float lse = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
    float pz = 0.f;
    for (int j = lane; j < a.top; j += 64) {
        const float p = a.index[(int64_t)j * a.M + m] < 0 ? 0.f : a.prob ? a.prob[m * a.top + j] : 1.f;
        if (p != 0.f) pz += p * a.target[(int64_t)j * a.M + m];
    }
    pz = lane_sum<64>(pz);
    if (lane == 0) {
        a.lse[m] = lse;
        a.loss[m] = a.counted[m] == 0.f ? 0.f : a.T * a.T * (a.entropy[m] + (lse - pz / a.T));
    }
}

// Sum of the losses and of the rows counted, in a fixed order.
__global__ __launch_bounds__(1024) void head_sums(HeadRowArgs a) {
    __shared__ float s[2][16];
    float l = 0.f, c = 0.f;
    for (int64_t m = threadIdx.x; m < a.M; m += 1024) l += a.loss[m], c += a.counted[m];
    l = lane_sum<64>(l), c = lane_sum<64>(c);
    if ((threadIdx.x & 63) == 0) s[0][threadIdx.x >> 6] = l, s[1][threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        l = c = 0.f;
        for (int i = 0; i < 16; ++i) l += s[0][i], c += s[1][i];
        a.sums[0] = l;
        a.sums[1] = c;
        if (a.mean) *a.mean = l / fmaxf(c, 1.f);
    }
}

// The factor of a row's dz: its loss' gradient (a mean's over the rows counted), 0 for a row that does not
// count, nan for one with a target outside the vocabulary; and its lse in units of log2(e).
FBL_DEV float2 row_factor(const HeadRowArgs& a, int64_t m, bool counted, bool bad) {
    float g = a.dloss[m * a.dloss_stride] * a.T;
    if (a.total) g /= fmaxf(a.total[1], 1.f);
    if (a.scale) {
        const bool one = a.dloss_stride == 0;  // one factor for all rows
        if (m == 0) *a.scale = one ? g : 1.f;
        if (one) g = 1.f;
    }
    return make_float2(!counted ? 0.f : bad ? quiet_nan() : g, a.lse_in[m] * kLog2e);
}

__global__ __launch_bounds__(256) void head_grad_labels(HeadRowArgs a) {
    const int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (m >= a.M) return;
    const Label l = label_of(a, m);
    a.index[m] = l.at;
    a.row[m] = row_factor(a, m, l.counted, !l.good);
}

__global__ __launch_bounds__(256) void head_grad_teacher(HeadRowArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= a.M) return;
    const int64_t* given = a.given + m * a.ldi;
    float sum = 0.f;
    bool bad = false;
    for (int j = lane; j < a.top; j += 64) {
        const float p = a.prob[m * a.top + j];
        sum += p;
        bad |= given[j] >= a.V;
        a.index[(int64_t)j * a.M + m] = given[j] >= 0 && given[j] < a.V && p != 0.f ? (int)given[j] : -1;
        a.weight[(int64_t)j * a.M + m] = p;
    }
    sum = lane_sum<64>(sum);
    const bool any_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (lane == 0) a.row[m] = row_factor(a, m, sum != 0.f || any_bad, any_bad);
}

unsigned blocks(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

}  // namespace

hipError_t launch_head_targets(const HeadRowArgs& a, hipStream_t s) {
    if (a.labels) hipLaunchKernelGGL(head_labels, dim3(blocks(a.M, 256)), dim3(256), 0, s, a);
    else if (a.logits_f32) hipLaunchKernelGGL(head_teacher<float>, dim3(blocks(a.M, 4)), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(head_teacher<bf16>, dim3(blocks(a.M, 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_head_join(const HeadRowArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(head_join, dim3(blocks(a.M, 16)), dim3(1024), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.sums) return e;
    hipLaunchKernelGGL(head_sums, dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_head_grad_rows(const HeadRowArgs& a, hipStream_t s) {
    if (a.labels) hipLaunchKernelGGL(head_grad_labels, dim3(blocks(a.M, 256)), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(head_grad_teacher, dim3(blocks(a.M, 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace fbl
