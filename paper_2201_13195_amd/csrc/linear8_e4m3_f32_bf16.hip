// Products of 8-bit operands: X in e4m3, scales in fp32, Y in bf16.
#include "linear8_launch.hpp"

namespace rmm {
template void launch_linear8_by<F8_E4M3, SCALE_F32, bf16_t>(int, const Linear8Args &, hipStream_t);
}  // namespace rmm
