// Attention over 4-bit pages, heads of 4 and of 5 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

template struct PackedHeads<4>;
template struct PackedHeads<5>;

}  // namespace rheo
