// factors.hpp -- the factors of a gated layer's gradient as they are kept in bf16's two bytes a value, gfx950.
//
// Eight consecutive ones of a row share an exponent E, the biased one of their largest: each is f 2^(126 - E), which is below
// 1, in fp16, and bit 14 of an fp16 of at most 1 is clear: the eight hold E's bits there (value 2q bit q, value 2q + 1 bit
// 4 + q).  So a factor within 2^13 of the largest is good to 2^-11 of itself and every other to 2^-24 of the largest, in
// bf16's range.  bf16 would be good to 2^-8: a rounding as large as dz's own and the result's (0.17% of a norm each), which two
// products carry on to every gradient of the layer.  Packing them costs the forward's epilogue about 30 operations for eight
// (4096 tokens 2048 -> 8192 259 -> 264 us, 4096 -> 11008 716 -> 720), unpacking them nothing that shows.
// A value that is not finite sets all bits of its eight, which read as infinities.
#pragma once

#include "kernels.hpp"
#include "stage.hpp"

namespace fbl {

using FactorWords = int __attribute__((ext_vector_type(4)));

constexpr uint32_t kShared = 0x40004000u;  // bit 14 of both halves of a word

// Cache policy of their stores and loads (nt).  A tile's factors are read once, long after they were written; passed through the caches like
// others they push out h, which the next product reads, and dz, which the next two do (us a step, stores alone / loads too: 8192
// tokens 1024 -> 4096 736 -> 713 / 698 -> 678 on another card, 16384 tokens 512 -> 2048 loads 505 -> 475, 4096 tokens 2048 -> 8192
// 1216 -> 1207 / 1183 -> 1179, 4096 -> 11008 the same, 2048 tokens 1024 -> 2816 178 -> 181).
constexpr int kOnce = 2;

FBL_DEV float with_exponent(_Float16 h, int e) { return __builtin_amdgcn_ldexpf((float)h, e - 126); }

FBL_DEV FactorWords pack_factors(const float (&f)[8]) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    float m = __builtin_fabsf(f[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __builtin_fmaxf(m, __builtin_fabsf(f[i]));
    const uint32_t e = __float_as_uint(m) >> 23, bits = (e & 15) << 11 | (e >> 4) << 27;
    uint32_t w[4], any = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f16x2 h = {(_Float16)__builtin_amdgcn_ldexpf(f[2 * q], 126 - (int)e),
                         (_Float16)__builtin_amdgcn_ldexpf(f[2 * q + 1], 126 - (int)e)};
        w[q] = __builtin_bit_cast(uint32_t, h);
        any |= w[q];
    }
    const bool finite = !(any & kShared);
    FactorWords out;
#pragma unroll
    for (int q = 0; q < 4; ++q) out[q] = finite ? (int)(w[q] | (bits << (3 - q) & kShared)) : -1;
    return out;
}

FBL_DEV void unpack_factors(const FactorWords& w, float (&f)[8]) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    uint32_t bits = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) bits |= ((uint32_t)w[q] & kShared) >> (3 - q);
    const int e = (int)((bits >> 11 & 0xf) | (bits >> 23 & 0xf0));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f16x2 h = __builtin_bit_cast(f16x2, (uint32_t)w[q] & ~kShared);
        f[2 * q] = with_exponent(h[0], e), f[2 * q + 1] = with_exponent(h[1], e);
    }
}

// The same where eight lanes hold one value each, in order.
FBL_DEV uint32_t of_eight(bool x) { return (uint32_t)(__ballot(x) >> (threadIdx.x & 56)) & 0xff; }

FBL_DEV uint16_t pack_factor(float f) {
    float m = __builtin_fabsf(f);
#pragma unroll
    for (int d = 1; d < 8; d *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, d));
    const uint32_t e = __float_as_uint(m) >> 23;
    const uint16_t h = __builtin_bit_cast(uint16_t, (_Float16)__builtin_amdgcn_ldexpf(f, 126 - (int)e));
    const uint32_t i = threadIdx.x & 7, bit = e >> (i / 2 + (i & 1) * 4) & 1;
    return of_eight(h & 0x4000) ? 0xffff : (uint16_t)(h | bit << 14);
}

FBL_DEV float unpack_factor(uint16_t h) {
    const uint32_t b = of_eight(h & 0x4000);
    uint32_t e = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) e |= (b >> 2 * q & 1) << q | (b >> (2 * q + 1) & 1) << (4 + q);
    return with_exponent(__builtin_bit_cast(_Float16, (uint16_t)(h & 0xbfff)), (int)e);
}

}  // namespace fbl
