// Attention over 4-bit pages: the launch by head size (see packed_kernels.h).
#include <type_traits>

#include "cache_state.h"

namespace rheo {

// (as packed_kernels.h defines it; that is compiled in the sources packed_heads_*)
template <int NB>
struct PackedHeads {
    static hipError_t prepare(int dtype);
    static size_t workspace(int units);
    static hipError_t launch(const CacheDev& c, const PackedDev& d, const rheo_packed_attention_args& a,
                             int* desc, hipStream_t s);
};

namespace {

// f(a constant: the blocks of 32 elements of a head, 1 to 8)
template <typename F>
auto by_blocks(int nb, F f) {
    switch (nb) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    case 4: return f(std::integral_constant<int, 4>());
    case 5: return f(std::integral_constant<int, 5>());
    case 6: return f(std::integral_constant<int, 6>());
    case 7: return f(std::integral_constant<int, 7>());
    default: return f(std::integral_constant<int, 8>());
    }
}

constexpr size_t kDescs = 2 * 8;         // words a compute unit: two workgroups' joins

}  // namespace

hipError_t prepare_packed(const CacheDev& c) {
    return by_blocks((c.D + 31) / 32, [&](auto nb) { return PackedHeads<nb>::prepare(c.dtype); });
}

size_t packed_workspace(const CacheDev& c) {
    return by_blocks((c.D + 31) / 32, [&](auto nb) { return PackedHeads<nb>::workspace(c.slots); }) +
           c.slots * kDescs;
}

hipError_t launch_packed_attention(const CacheDev& c, const PackedDev& d,
                                   const rheo_packed_attention_args& a, hipStream_t s) {
    int* desc = (int*)(c.part + packed_workspace(c) - c.slots * kDescs);
    return by_blocks(d.nb, [&](auto nb) { return PackedHeads<nb>::launch(c, d, a, desc, s); });
}

}  // namespace rheo
