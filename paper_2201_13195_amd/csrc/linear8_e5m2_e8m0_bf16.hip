// Products of 8-bit operands: X in e5m2, scales in powers of two, Y in bf16.
#include "linear8_launch.hpp"

namespace rmm {
template void launch_linear8_by<F8_E5M2, SCALE_E8M0, bf16_t>(int, const Linear8Args &, hipStream_t);
}  // namespace rmm
