// Tiles of 8-bit products: X in e5m2, scales in fp32, Y in bf16.
#include "linear8_tile.hpp"

namespace rmm {
template void launch_linear8_tiles<F8_E5M2, SCALE_F32, bf16_t>(const Linear8Args &, bool, hipStream_t);
}  // namespace rmm
