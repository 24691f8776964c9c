// Loads from memory straight into LDS, and the waits around them, shared by the kernels whose operands take that way
// (mfma_kernels.hpp, linear8_tile.hpp).
#pragma once
#include "mfma_frag.hpp"

namespace rmm {

namespace {

// One wave's load of 1 KB into LDS from byte `to` on, 16 bytes from `off` + `soff` per lane.  The compiler does
// not see that it writes LDS (it would wait for it before every LDS read): the explicit waits and barriers order them.
__device__ __forceinline__ void load_to_lds(u32x4_t rsrc, uint32_t to, uint32_t off, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(rsrc), "s"(soff) : "m0");
}
// The same from `off`.
__device__ __forceinline__ void load_to_lds(u32x4_t rsrc, uint32_t to, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(rsrc) : "m0");
}
// Waits until at most N of this wave's loads are outstanding.
template <int N>
__device__ __forceinline__ void wait_for_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The wait states between a vector instruction that writes a scalar register (a readfirstlane, a spilled one that comes back) and a
// load that reads it: the compiler does not look for them in front of load_to_lds.  What a step of a K-contiguous operand writes (the range
// of its descriptor, the offset along its rows) is scalar instructions, which need none, and is not settled: twenty clocks a step and
// operand, 64 x 64 tiles of Y 5 % (1024 x 1024 -> 512 5.8 and 6.1 us).  That the compiler brings none of it back from a vector register too
// close to a load is looked for in the built library (tests/test_load_hazards.py).
__device__ __forceinline__ void settle(u32x4_t &descriptor) { asm volatile("s_nop 4" : "+s"(descriptor)); }

}  // namespace

}  // namespace rmm
