// Attention over 4-bit pages, heads of 2 and of 7 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

PackedHeads packed_heads_2() { return packed_heads<2>(); }
PackedHeads packed_heads_7() { return packed_heads<7>(); }

}  // namespace rheo
