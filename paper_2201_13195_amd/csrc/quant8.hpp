// 8-bit operands: rows and weights in OCP e4m3 / e5m2 with a scale for each block, and what the kernels that make
// them (quant8.hip, norm.hip) and read them (linear8.hip) share.
//
// A block of amax = max |x| has the scale s = amax / top (top: the format's largest number), no less than 2^-126 so
// that it is normal, or the next power of two; its data are x / s in the nearest number of the format.  |x / s| <= top
// up to one rounding, far from where the format's next number would begin: nothing saturates.
#pragma once
#include "common.hpp"

namespace rmm {

// An 8-bit matrix as the kernels see it (rmm_mat8_t).
struct Mat8 {
    uint8_t *data;
    int64_t ld;
    void *scales;
    int64_t ld_scales;
};

enum { F8_E4M3 = 0, F8_E5M2 = 1 };
enum { SCALE_F32 = 0, SCALE_E8M0 = 1 };
constexpr int kBlock8 = 128;  // columns (and rows, of weights) of a block

// Launchers (quant8.hip, norm.hip, linear8.hip).  T: bf16_t or float.
template <typename T>
hipError_t launch_quantize_rows8(const T *A, int64_t n, int64_t d, int f8, int scale, const Mat8 &out, hipStream_t stream);
// (`out_t`: the transposed matrix too, if not null)
template <typename T>
hipError_t launch_quantize_weight8(const T *W, int64_t rows, int64_t cols, int f8, int scale, const Mat8 &out, const Mat8 *out_t,
                                   hipStream_t stream);
template <typename T>
hipError_t launch_linear8(const Mat8 &X, const Mat8 &W, const T *bias, T *Y, int64_t n, int64_t d_in, int64_t d_out, int f8, int scale,
                          hipStream_t stream);
// (residual, H, Y, Y8 and rstd may be null)
template <typename T>
hipError_t launch_rms_norm(const T *X, const T *residual, const T *weight, T *H, T *Y, const Mat8 *Y8, int f8, int scale, float *rstd,
                           int64_t n, int64_t d, float eps, hipStream_t stream);
size_t norm_backward_partials(int64_t n, int64_t d);  // fp32 numbers of scratch for dweight
template <typename T>
hipError_t launch_rms_norm_backward(const T *dY, const T *dH, const T *H, const T *weight, const float *rstd, T *dX, T *dweight,
                                    float *part, int64_t n, int64_t d, hipStream_t stream);

namespace {

typedef float f32x2v_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));

// Rounds to T's numbers, two at a time.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    union {
        bf16x2v_t v;
        uint32_t u;
    } o;
    o.v = __builtin_convertvector((f32x2v_t){a, b}, bf16x2v_t);  // nearest even
    return o.u;
}
template <typename T>
__device__ __forceinline__ float rounded(float v) {
    if constexpr (sizeof(T) == 2)
        return __uint_as_float(pack_bf16(v, v) << 16);
    else
        return v;
}

// Eight columns of a row, as they are in memory: the loads of several runs, and of the row that is next, are in flight before the
// first is waited for.  So no load stands behind a branch (with one, the compiler waits for each load where the branches meet:
// 768 x 768 weights to 8 bits 11.1 us, without 7.9), and what a run's end asks for happens when it is used.  Rows by their width:
//   EVEN    a multiple of eight: a run exists whole or not at all
//   RAGGED  eight and more: the run that the row ends in is loaded from eight before the end and shifted down (element by element
//           behind a branch: norm backward of 16384 x 4095 bf16 214 us, like this 129)
//   TINY    fewer: element by element
// Rows start anywhere: the hardware takes 16-byte loads at any element's address.
enum { ROWS_EVEN = 0, ROWS_RAGGED = 1, ROWS_TINY = 2 };
inline int rows_mode(int64_t d) { return d % 8 == 0 ? ROWS_EVEN : d >= 8 ? ROWS_RAGGED : ROWS_TINY; }
typedef uint32_t u32x4a_t __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4a_t __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct Run8 {
    uint32_t q[2 * sizeof(T)];
};
// (also of columns that the row does not have)
template <typename T, int MODE>
__device__ __forceinline__ Run8<T> load_run(const T *row, int64_t col, int64_t d) {
    Run8<T> r;
    if constexpr (MODE != ROWS_TINY) {
        const T *p = row + (MODE == ROWS_EVEN ? (col < d ? col : 0) : min(col, d - 8));
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            const u32x4a_t a = *reinterpret_cast<const u32x4a_t *>(p + 16 / sizeof(T) * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) r.q[4 * h + i] = a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t e = col + i < d ? __float_as_uint(load_f32<T>(row + col + i)) : 0u;
            if constexpr (sizeof(T) == 2)
                r.q[i / 2] = i % 2 ? r.q[i / 2] | e : e >> 16;
            else
                r.q[i] = e;
        }
    }
    return r;
}
// Its values as fp32; zeros where the row has no columns.
template <typename T, int MODE>
__device__ __forceinline__ void values(const Run8<T> &run, int64_t col, int64_t d, float (&v)[8]) {
    constexpr int N = 2 * sizeof(T), A = N / 2;  // dwords, and those of four elements
    uint32_t q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = run.q[i];
    if constexpr (MODE == ROWS_EVEN) {
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = col < d ? q[i] : 0u;
    } else if constexpr (MODE == ROWS_RAGGED) {
        const int by = (int)max((int64_t)0, min(col - (d - 8), (int64_t)8));  // elements
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = by & 4 ? (i + A < N ? q[i + A < N ? i + A : 0] : 0u) : q[i];
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = by & 2 ? (i + A / 2 < N ? q[i + A / 2 < N ? i + A / 2 : 0] : 0u) : q[i];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t above = i + 1 < N ? q[i + 1 < N ? i + 1 : 0] : 0u;
            q[i] = by & 8 ? 0u : by & 1 ? (sizeof(T) == 2 ? q[i] >> 16 | above << 16 : above) : q[i];
        }
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(q[i] << 16), v[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(q[i]);
    }
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t valid, float (&v)[8]) {
    if (valid >= 8)
        values<T, ROWS_EVEN>(load_run<T, ROWS_EVEN>(p, 0, 8), 0, 8, v);
    else
        values<T, ROWS_TINY>(load_run<T, ROWS_TINY>(p, 0, valid), 0, valid, v);
}
template <typename T>
__device__ __forceinline__ void store8(T *p, int64_t valid, const float (&v)[8]) {
    if (valid >= 8) {
        if constexpr (sizeof(T) == 2) {
            u32x4a_t q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<u32x4a_t *>(p) = q;
        } else {
            *reinterpret_cast<f32x4a_t *>(p) = (f32x4a_t){v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4a_t *>(p + 4) = (f32x4a_t){v[4], v[5], v[6], v[7]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) store_f32<T>(p + i, v[i]);
    }
}
template <typename T, int MODE>
__device__ __forceinline__ void store_run(T *row, int64_t col, int64_t d, const float (&v)[8]) {
    if constexpr (MODE == ROWS_EVEN) {
        if (col < d) store8<T>(row + col, 8, v);
    } else {
        store8<T>(row + (col < d ? col : 0), d - col, v);
    }
}
// Eight data bytes to p (8-byte aligned), of which the first `valid` belong to the matrix.
__device__ __forceinline__ void store8_bytes(uint8_t *p, int64_t valid, uint2 q) {
    if (valid >= 8) {
        *reinterpret_cast<uint2 *>(p) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (uint8_t)((i < 4 ? q.x : q.y) >> (i % 4 * 8));
    }
}

// Largest magnitude, as its bits: they are ordered as the magnitudes are, with infinity and NaN on top.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t amax8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
    return m;
}

// The scale of a block, as the divisor and as it is stored.
struct BlockScale {
    float s, inv;  // inv = 1 / s, rounded; meaningful where !slow
    uint32_t stored;
    bool slow;
};
template <int F8>
__device__ __forceinline__ constexpr float top_of() { return F8 == F8_E4M3 ? 448.0f : 57344.0f; }
// (`q`: amax / top)
template <int F8, int SCALE>
__device__ __forceinline__ BlockScale block_scale(float q) {
    const float s = q < 0x1p-126f ? 0x1p-126f : q;  // (NaN stays)
    BlockScale b;
    if constexpr (SCALE == SCALE_F32) {
        b.s = s, b.stored = __float_as_uint(s);
    } else {
        const uint32_t e = (__float_as_uint(s) + 0x7FFFFFu) >> 23;  // s is normal: its exponent, one more if it is no power of two
        b.stored = e < 255u ? e : 255u;
        b.s = e < 255u ? __uint_as_float(e << 23) : __uint_as_float(0x7FC00000u);
    }
    b.inv = 1.0f / b.s;
    // (then the remainder below would not be exact, or s is no number)
    b.slow = !(b.s > 0x1p-90f && b.s < 0x1p125f);
    return b;
}

template <int F8, int SCALE>
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits) {
    return block_scale<F8, SCALE>(__uint_as_float(amax_bits) / top_of<F8>());
}

// v / s, correctly rounded.  A power of two: the product with its inverse is exact.  Else from q = v inv, which is a unit
// or so off, and the remainder v - q s, which is exact in one fused operation: three instructions where the division
// written out is ten (the norm's kernel would be bound by them).  (With s of 2^-90 and less the remainder could be below the
// numbers of fp32, and an s that is no number has none: `slow`.)  With a v that is known to more than fp32, as v + low, the
// remainder takes what fp32 does not hold.
template <int SCALE>
__device__ __forceinline__ float over_scale(float v, const BlockScale &b) {
    const float q = v * b.inv;
    if constexpr (SCALE == SCALE_E8M0) return q;
    return fmaf(fmaf(-q, b.s, v), b.inv, q);
}
template <int SCALE>
__device__ __forceinline__ float over_scale(float v, float low, const BlockScale &b) {
    const float q = v * b.inv;
    if constexpr (SCALE == SCALE_E8M0) return q;
    return fmaf(fmaf(-q, b.s, v) + low, b.inv, q);
}
template <int F8>
__device__ __forceinline__ uint32_t pack4_f8(float a, float b, float c, float d) {
    int r;
    if constexpr (F8 == F8_E4M3)
        r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    else
        r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
    return (uint32_t)r;
}
template <int F8, int SCALE>
__device__ __forceinline__ uint2 to_f8(const float (&v)[8], const float (&low)[8], const BlockScale &b) {
    float q[8];
    if (b.slow) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = v[i] / b.s;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = over_scale<SCALE>(v[i], low[i], b);
    }
    return make_uint2(pack4_f8<F8>(q[0], q[1], q[2], q[3]), pack4_f8<F8>(q[4], q[5], q[6], q[7]));
}
template <int F8, int SCALE>
__device__ __forceinline__ uint2 to_f8(const float (&v)[8], const BlockScale &b) {
    float q[8];
    if (b.slow) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = v[i] / b.s;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = over_scale<SCALE>(v[i], b);
    }
    return make_uint2(pack4_f8<F8>(q[0], q[1], q[2], q[3]), pack4_f8<F8>(q[4], q[5], q[6], q[7]));
}
template <int SCALE>
__device__ __forceinline__ void store_scale(void *scales, int64_t at, const BlockScale &b) {
    if constexpr (SCALE == SCALE_F32)
        reinterpret_cast<uint32_t *>(scales)[at] = b.stored;
    else
        reinterpret_cast<uint8_t *>(scales)[at] = (uint8_t)b.stored;
}

// Exchanges within rows of 16 lanes, in the vector unit: with neighbours at distance 1 and 2, then across the halves of eight and
// of 16 (mirrored, which is the same once the lanes of a half agree).
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
enum { LANE_XOR1 = 0xB1, LANE_XOR2 = 0x4E, LANE_MIRROR8 = 0x141, LANE_MIRROR16 = 0x140 };
// Largest over the 16 lanes that hold a block of 128 columns, eight each.
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
    m = max(m, from_lane<LANE_XOR1>(m)), m = max(m, from_lane<LANE_XOR2>(m));
    m = max(m, from_lane<LANE_MIRROR8>(m));
    return max(m, from_lane<LANE_MIRROR16>(m));
}
__device__ __forceinline__ float max_of_16(float v) {
    auto with = [&](uint32_t other) { v = fmaxf(v, __uint_as_float(other)); };
    with(from_lane<LANE_XOR1>(__float_as_uint(v))), with(from_lane<LANE_XOR2>(__float_as_uint(v)));
    with(from_lane<LANE_MIRROR8>(__float_as_uint(v))), with(from_lane<LANE_MIRROR16>(__float_as_uint(v)));
    return v;
}
template <int CTRL>
__device__ __forceinline__ float plus_lane(float v) {
    return v + __uint_as_float(from_lane<CTRL>(__float_as_uint(v)));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); }
template <int CTRL>
__device__ __forceinline__ double plus_lane(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    return v + __longlong_as_double((long long)(from_lane<CTRL>((uint32_t)u) | (uint64_t)from_lane<CTRL>((uint32_t)(u >> 32)) << 32));
}
__device__ __forceinline__ double lane_value(double v, int lane) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane) |
                                            (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane) << 32));
}
// Sum over the 64 lanes, the same in all.
template <typename F>
__device__ __forceinline__ F sum_of_64(F v) {
    v = plus_lane<LANE_MIRROR16>(plus_lane<LANE_MIRROR8>(plus_lane<LANE_XOR2>(plus_lane<LANE_XOR1>(v))));
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

}  // namespace

}  // namespace rmm
