// Attention over 4-bit pages, heads of 3 and of 6 blocks of 32 elements.
#include "packed_kernels.h"

namespace rheo {

template struct PackedHeads<3>;
template struct PackedHeads<6>;

}  // namespace rheo
