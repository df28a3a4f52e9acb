// Attention over 4-bit pages, heads of 3 and of 6 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

PackedHeads packed_heads_3() { return packed_heads<3>(); }
PackedHeads packed_heads_6() { return packed_heads<6>(); }

}  // namespace rheo
