// What the kernels of 8-bit products share: fragments, the matrix instructions on them, scales.
//
// The 8-bit matrix instructions add products of eight neighbouring contraction elements at once, cut (towards zero) to 2^-13 of
// the largest one's power of two (measured: 1 beside 2^13 counts, beside 2^14 it does not), before they reach the fp32
// accumulator: 1.5e-5 of the result for normal data.  Far below the rounding of a bf16 result (1.7e-3), and that is where they are
// used.  An fp32 result takes the exact way: both operands as bf16 numbers, which hold every 8-bit one, at half the rate.
#pragma once
#include "mfma_frag.hpp"
#include "quant8.hpp"

namespace rmm {

struct Linear8Args {
    Mat8 x, w;
    const void *bias;
    void *Y;
    int64_t n, d_in, d_out;
};

// The product by the kernel that linear8_plan() names (linear8_<X>_<scales>_<Y>.hip, an instance each).
template <int F8, int SCALE, typename T>
void launch_linear8_by(int kernel, const Linear8Args &g, hipStream_t stream);

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// The product of two powers of two 2^(x - 127) and 2^(w - 127) (255: no number), whose exponents reach from -254 to 254, as s 2^(rest - 127)
// with s among fp32's normal numbers.  `rest` goes to X's data, in front of the sum of a block: 127 nearly always, and what it is more or
// less than that counts up to 64, as sums of a block (0, or 2^-25 to 2^32) times s are then infinite or nothing anyway.
struct PowerProduct {
    float s;
    uint32_t rest;
};
__device__ __forceinline__ PowerProduct power_product(uint32_t x, uint32_t w) {
    const int e = (int)(x + w) - 127, normal = min(max(e, 1), 254);
    return {__uint_as_float(max(x, w) == 255u ? 0x7FC00000u : (uint32_t)normal << 23), (uint32_t)(min(max(e - normal, -64), 64) + 127)};
}

// The first `valid` bytes of 16, the others zero.
__device__ __forceinline__ uint4 first_bytes(uint4 q, int64_t valid) {
    uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t left = valid - 4 * i;
        v[i] = left >= 4 ? v[i] : left <= 0 ? 0u : v[i] & ((1u << (8 * left)) - 1u);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Bytes 8 q .. 8 q + 7 of a fragment, times a power of two, as bf16 numbers.
template <int F8>
__device__ __forceinline__ bf16x8_t widened(const i32x8_t &f, int q, float by = 1.0f) {
    union {
        bf16x8_t v;
        bf16x2_t p[4];
    } o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t u = (uint32_t)f[2 * q + i];
        if constexpr (F8 == F8_E4M3) {
            o.p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, by, false), o.p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, by, true);
        } else {
            o.p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(u, by, false), o.p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(u, by, true);
        }
    }
    return o.v;
}
// The products of one block of 128: W's fragment times X's (of format F8), without the block's scales.
template <int F8>
__device__ __forceinline__ f32x4_t block_products(const i32x8_t &w, const i32x8_t &x) {
    const f32x4_t zero = {0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, F8, 0, 0, 0, 0);
}
// The same with X times 2^(rest - 127).
template <int F8>
__device__ __forceinline__ f32x4_t block_products(const i32x8_t &w, const i32x8_t &x, uint32_t rest) {
    const f32x4_t zero = {0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, F8, 0, 127, 0, (int)rest);
}
__device__ __forceinline__ f32x4_t block_products(const bf16x8_t (&w)[4], const bf16x8_t (&x)[4]) {
    f32x4_t part = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[q], x[q], part, 0, 0, 0);
    return part;
}
// acc += the products times both scales: powers of two, byte J of the lane's `xs` and the lowest byte of `ws`.  Written as assembly
// because the compiler never gives the scaled instruction the same registers for the sum that goes in and the one that comes out: twice
// the accumulators, and copies.  (The two wait states are for an operand that a vector instruction has just written, which the
// compiler does not look for in front of assembly; results are read behind settle_sums.)
template <int F8, int J>
__device__ __forceinline__ void add_scaled_products(const i32x8_t &w, const i32x8_t &x, f32x4_t &acc, uint32_t ws, uint32_t xs) {
#define RMM_SCALED(SEL)                                                                                                            \
    if constexpr (F8 == F8_E4M3)                                                                                                   \
        asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 " SEL                                  \
                     : "+v"(acc)                                                                                                   \
                     : "v"(w), "v"(x), "v"(ws), "v"(xs)                                                                            \
                     : "memory");                                                                                                  \
    else                                                                                                                           \
        asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 " SEL " blgp:1"                        \
                     : "+v"(acc)                                                                                                   \
                     : "v"(w), "v"(x), "v"(ws), "v"(xs)                                                                            \
                     : "memory");
    if constexpr (J == 0) {
        RMM_SCALED("op_sel_hi:[0,0,0]")
    } else if constexpr (J == 1) {
        RMM_SCALED("op_sel:[0,1,0] op_sel_hi:[0,0,0]")
    } else if constexpr (J == 2) {
        RMM_SCALED("op_sel_hi:[0,1,0]")
    } else {
        RMM_SCALED("op_sel:[0,1,0] op_sel_hi:[0,1,0]")
    }
#undef RMM_SCALED
}
// Keeps the making of a value, and the memory accesses around it, in their places.
__device__ __forceinline__ void pin(f32x4_t &v) { asm volatile("" : "+v"(v) : : "memory"); }
// Between the last of these and the first use of their sums (19 wait states would do for the longest of matrix instructions).
template <int TU, int TJ>
__device__ __forceinline__ void settle_sums(f32x4_t (&acc)[TU][TJ]) {
    asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
    for (int u = 0; u < TU; ++u)
#pragma unroll
        for (int j = 0; j < TJ; ++j) asm volatile("" : "+v"(acc[u][j]));
}

// Four consecutive outputs o .. o + 3 of a row, of which `valid` exist.
typedef uint32_t u32x2a_t __attribute__((ext_vector_type(2), aligned(2)));
template <typename T>
__device__ __forceinline__ void store4(T *p, int64_t valid, const f32x4_t &v) {
    if (valid >= 4) {
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<u32x2a_t *>(p) = (u32x2a_t){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else
            *reinterpret_cast<f32x4a_t *>(p) = (f32x4a_t){v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < valid) store_f32<T>(p + i, v[i]);
    }
}

}  // namespace

}  // namespace rmm
