// The 4-bit format of the packed cache (see "The cache in 4 bits" in rheo.h): codes of
// two elements a byte (e2m1), an exponent for every 32 elements of an entry.
#pragma once

#include <type_traits>

#include "cache_state.h"
#include "half_types.h"

namespace rheo {

// Exponents (+ 127) between which every code's value is exact in T, whatever the value:
// beyond them the smallest or the largest would not be numbers of the type.
template <typename T>
constexpr int kScaleLow = std::is_same<T, __bf16>::value ? 2 : 104;
template <typename T>
constexpr int kScaleHigh = std::is_same<T, __bf16>::value ? 252 : 140;

// Byte j of a word as the power of two that it stands for.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
template <int J>
__device__ __forceinline__ float scale_at(uint32_t w) {
    const uint32_t m = 0x7F800000u;
    return __uint_as_float(J == 3 ? w >> 1 & m : w << (23 - 8 * J) & m);
}

// The values of byte J of `codes` (two elements), as a word of two.  Exact: a code has two
// bits of fraction.
template <typename T, int J>
__device__ __forceinline__ uint32_t pair_of(uint32_t codes, float scale) {
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, J));
    else
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, J));
}

// The code byte J of a word from two elements, to nearest even, 6 at most.
template <typename T, int J>
__device__ __forceinline__ uint32_t put_pair(uint32_t codes, uint32_t w, float scale) {
    typedef typename Pack<T>::v2 v2;
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(v2, w), scale, J);
    else
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(v2, w), scale, J);
}

// Eight elements of a block to a word of codes; the block's four lanes (next to each
// other) call it together.  `scale` becomes the block's exponent byte; whether an element
// was no finite number.
//
// With the largest magnitude m 2^E, exponents E - 2 and E - 1 put it at 4 m and 2 m: the first
// has half the step and, up to m = 1.75, is off by 1 of it at most (7 held as 6); above,
// the second is (3.5 to 4 held as 4).  The carry of m's fraction + 0.25 into the exponent is
// that choice.
template <typename T>
__device__ __forceinline__ bool pack_block(uint4 x, uint32_t* codes, uint32_t* scale) {
    constexpr uint32_t E = Pack<T>::kExp, kMost = E - 1;     // the largest finite
    uint32_t* w = &x.x;
    bool bad = false;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t lo = w[i] & 0x7FFFu, hi = w[i] >> 16 & 0x7FFFu;
        if (lo >= E || hi >= E) {                      // rare
            bad = true;
            if (lo >= E) w[i] = (w[i] & 0xFFFF0000u) | (lo > E ? 0 : (w[i] & 0x8000u) | kMost);
            if (hi >= E) w[i] = (w[i] & 0xFFFFu) | (hi > E ? 0 : (w[i] & 0x80000000u) | kMost << 16);
            if (lo >= E) lo = 0;
            if (hi >= E) hi = 0;
        }
        most = max(most, max(lo, hi));
    }
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    const uint32_t bits = __float_as_uint(lo_f32<T>(most));
    const int e = min(max((int)((bits + 0x200000u) >> 23) - 2, kScaleLow<T>), kScaleHigh<T>);
    const float f = scale_of(e);
    uint32_t c = put_pair<T, 0>(0u, w[0], f);
    c = put_pair<T, 1>(c, w[1], f);
    c = put_pair<T, 2>(c, w[2], f);
    *codes = put_pair<T, 3>(c, w[3], f);
    *scale = e;
    return bad;
}

}  // namespace rheo
