// Attention over 4-bit pages by head size: each has sources of its own (packed_heads_*), so that
// they are compiled side by side.
#pragma once

#include "cache_state.h"

namespace rheo {

// The calls for heads of a number of blocks of 32 elements.
struct PackedHeads {
    hipError_t (*prepare)(int dtype);        // once for the current device
    size_t (*workspace)(int units);          // floats of partial results, without the joins' words
    hipError_t (*launch)(const CacheDev& c, const PackedDev& d, const rheo_packed_attention_args& a,
                         int* desc, hipStream_t s);
};

PackedHeads packed_heads_1();
PackedHeads packed_heads_2();
PackedHeads packed_heads_3();
PackedHeads packed_heads_4();
PackedHeads packed_heads_5();
PackedHeads packed_heads_6();
PackedHeads packed_heads_7();
PackedHeads packed_heads_8();

}  // namespace rheo
