// Tiles of 8-bit products: X in e5m2, scales in powers of two, Y in fp32.
#include "linear8_tile.hpp"

namespace rmm {
template void launch_linear8_tiles<F8_E5M2, SCALE_E8M0, float>(const Linear8Args &, bool, hipStream_t);
}  // namespace rmm
