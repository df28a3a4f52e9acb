// The reference of a softmax's exponents, as the attention kernels keep it.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

namespace rheo {

constexpr float kLog2e = 1.4426950408889634f;

// The exponents' reference stands at most kSlack<T> below a row's largest score so far (in
// units of log2), and kRise<T> lower still.  For bf16, which has fp32's exponents, that is
// 2^8 at most for a probability, and no rise.  fp16 ends at 65504 and has full accuracy
// from 2^-14 on, so its probabilities take all of the upper range, to 2^15: those down to
// 2^-24 (16.6 nats) of the largest are rounded to 11 bits, and 2^-35 of it is the most
// that smaller ones are off by.  (With the largest at 1, keys 17 nats below a sink lost 44 %
// of their weight to the smallest step.)  A slack of 4 and a rise of 11: more rescaling,
// 395 us for 385 with 244 rows of 256 elements over 32 times 4096 entries; 6 and 9: 379;
// at other head sizes the three are alike.
template <typename T>
constexpr float kSlack = std::is_same<T, __bf16>::value ? 8.0f : 5.0f;
template <typename T>
constexpr float kRise = std::is_same<T, __bf16>::value ? 0.0f : 10.0f;

// The reference as the exponents have it, rounded; any where a row has no score yet.
template <typename T>
__device__ __forceinline__ float ref_of(float m, float to2) {
    return m == -INFINITY ? 0.0f : m * to2 - kRise<T>;
}
// ln of a sum relative to it
template <typename T>
__device__ __forceinline__ float lse_of(float m, float l, float scale) {
    constexpr float down = std::is_same<T, __bf16>::value ? 1.0f : 0x1p-10f;    // 2^-kRise, exact
    return m * scale + logf(l * down);
}

}  // namespace rheo
