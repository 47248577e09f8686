// rows.hpp -- building blocks of the kernels that work on rows of values: 16-byte
// accesses at any element alignment, and sums over the lanes that share a row.
#pragma once

#include "cdna4.hpp"

namespace fbl {

// 16 bytes of elements, aligned as one element is: a row may start anywhere (an odd
// width, a column view), and the hardware takes unaligned global accesses.
template <typename T>
struct Pack {
    static constexpr int N = 16 / (int)sizeof(T);
    struct __attribute__((packed, aligned(sizeof(T)))) Raw {
        T v[N];
    };
    Raw raw;
    // Elements col .. of a row of n at `row`, those past its end zeros, in two steps: fetch has no branch
    // and waits for nothing, so that several can be on the way, and settle puts the chunk right that would cross the
    // row's end (fetch reads it from where it fits).  Rows shorter than a chunk: SHORT, read one by one.
    template <bool SHORT = false>
    FBL_DEV void fetch(const T* row, int col, int n) {
        if constexpr (SHORT) {
#pragma unroll
            for (int e = 0; e < N; ++e) raw.v[e] = col + e < n ? row[col + e] : (T)0.f;
        } else {
            raw = *reinterpret_cast<const Raw*>(row + (col < n - N ? col : n - N));
        }
    }
    template <bool SHORT = false>
    FBL_DEV void settle(int col, int n) {
        if constexpr (!SHORT) {
            const int past = col - (n - N);  // elements of the chunk beyond the row
            if (past > 0) {
                unsigned __int128 x = __builtin_bit_cast(unsigned __int128, raw);
                x = past < N ? x >> (past * 8 * (int)sizeof(T)) : 0;
                raw = __builtin_bit_cast(Raw, x);
            }
        }
    }
    FBL_DEV void load(const T* row, int col, int n) {
        if (n < N) {
            fetch<true>(row, col, n);
        } else {
            fetch(row, col, n);
            settle(col, n);
        }
    }
    FBL_DEV void store(T* row, int col, int n) const {
        if (col + N <= n) {
            *reinterpret_cast<Raw*>(row + col) = raw;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (col + e < n) row[col + e] = raw.v[e];
        }
    }
    FBL_DEV float operator[](int e) const { return (float)raw.v[e]; }
    FBL_DEV void set(int e, float x) { raw.v[e] = (T)x; }
};

template <int CTRL>
FBL_DEV float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// Sum over groups of LANES (16 or 64) consecutive lanes, the same value in each: within 16
// by DPP (swaps of neighbours, pairs, halves mirrored), across them by the row swaps of the wavefront.
template <int LANES>
FBL_DEV float lane_sum(float x) {
    static_assert(LANES == 16 || LANES == 64, "a row of 16 lanes or a wavefront");
    x += dpp<0xB1>(x);   // quad_perm 1 0 3 2
    x += dpp<0x4E>(x);   // quad_perm 2 3 0 1
    x += dpp<0x141>(x);  // row_half_mirror
    x += dpp<0x140>(x);  // row_mirror
    if constexpr (LANES == 64) {
        auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return x;
}

}  // namespace fbl
