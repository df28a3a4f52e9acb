// The 16-bit types of the cache operators: bf16 (__bf16) and fp16 (_Float16).
// All roundings are to nearest even.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rheo {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Pack;
template <>
struct Pack<__bf16> {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExp = 0x7F80;       // exponent bits of one element
};
template <>
struct Pack<_Float16> {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExp = 0x7C00;
};

template <typename T>
__device__ __forceinline__ float lo_f32(uint32_t w);
template <typename T>
__device__ __forceinline__ float hi_f32(uint32_t w);
template <>
__device__ __forceinline__ float lo_f32<__bf16>(uint32_t w) { return __uint_as_float(w << 16); }
template <>
__device__ __forceinline__ float hi_f32<__bf16>(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
template <>
__device__ __forceinline__ float lo_f32<_Float16>(uint32_t w) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
}
template <>
__device__ __forceinline__ float hi_f32<_Float16>(uint32_t w) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
}

// Two floats rounded into one word, the first in its low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, typename Pack<T>::v2));
}

// Eight elements of a 16-byte vector to floats, and back.
template <typename T>
__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = lo_f32<T>(w[i]);
        f[2 * i + 1] = hi_f32<T>(w[i]);
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* f) {
    return make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]),
                      pack2<T>(f[6], f[7]));
}

}  // namespace rheo
