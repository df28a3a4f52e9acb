// Attention over 4-bit pages: the launch by head size (see packed_kernels.h).
#include "packed_heads.h"

namespace rheo {

namespace {

PackedHeads heads_of(const CacheDev& c) {
    switch ((c.D + 31) / 32) {
    case 1: return packed_heads_1();
    case 2: return packed_heads_2();
    case 3: return packed_heads_3();
    case 4: return packed_heads_4();
    case 5: return packed_heads_5();
    case 6: return packed_heads_6();
    case 7: return packed_heads_7();
    default: return packed_heads_8();
    }
}

constexpr size_t kDescs = 2 * 8;         // words a compute unit: two workgroups' joins

}  // namespace

hipError_t prepare_packed(const CacheDev& c) { return heads_of(c).prepare(c.dtype); }

size_t packed_workspace(const CacheDev& c) {
    return heads_of(c).workspace(c.slots) + c.slots * kDescs;
}

hipError_t launch_packed_attention(const CacheDev& c, const PackedDev& d,
                                   const rheo_packed_attention_args& a, hipStream_t s) {
    int* desc = (int*)(c.part + packed_workspace(c) - c.slots * kDescs);
    return heads_of(c).launch(c, d, a, desc, s);
}

}  // namespace rheo
