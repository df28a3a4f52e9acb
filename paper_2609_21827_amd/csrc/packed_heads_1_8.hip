// Attention over 4-bit pages, heads of 1 and of 8 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

template struct PackedHeads<1>;
template struct PackedHeads<8>;

}  // namespace rheo
