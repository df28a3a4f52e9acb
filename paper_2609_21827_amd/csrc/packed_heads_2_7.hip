// Attention over 4-bit pages, heads of 2 and of 7 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

template struct PackedHeads<2>;
template struct PackedHeads<7>;

}  // namespace rheo
