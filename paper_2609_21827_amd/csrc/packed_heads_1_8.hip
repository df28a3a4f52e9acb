// Attention over 4-bit pages, heads of 1 and of 8 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

PackedHeads packed_heads_1() { return packed_heads<1>(); }
PackedHeads packed_heads_8() { return packed_heads<8>(); }

}  // namespace rheo
