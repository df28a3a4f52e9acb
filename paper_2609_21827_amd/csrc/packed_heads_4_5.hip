// Attention over 4-bit pages, heads of 4 and of 5 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

PackedHeads packed_heads_4() { return packed_heads<4>(); }
PackedHeads packed_heads_5() { return packed_heads<5>(); }

}  // namespace rheo
