// Y = X W^T (+ bias) with 8-bit operands: Y(i, o) = sum over blocks b of 128 contraction elements of
// sx(b, i) sw(o / 128, b) * (sum over the block of X W), in fp32.
//
// The 8-bit matrix instructions add products of eight neighbouring contraction elements at once, cut (towards zero) to 2^-13 of
// the largest one's power of two (measured: 1 beside 2^13 counts, beside 2^14 it does not), before they reach the fp32
// accumulator: 1.5e-5 of the result for normal data.  Far below the rounding of a bf16 result (1.7e-3), and that is where they are
// used.  An fp32 result takes the exact way: both operands as bf16 numbers, which hold every 8-bit one, at half the rate.
#include "quant8.hpp"

namespace rmm {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

struct Linear8Args {
    Mat8 x, w;
    const void *bias;
    void *Y;
    int64_t n, d_in, d_out;
};

template <int SCALE>
__device__ __forceinline__ float scale_at(const void *scales, int64_t at) {
    if constexpr (SCALE == SCALE_F32) {
        return reinterpret_cast<const float *>(scales)[at];
    } else {
        const uint32_t e = reinterpret_cast<const uint8_t *>(scales)[at];
        return __uint_as_float(e == 255u ? 0x7FC00000u : e == 0u ? 0x00400000u : e << 23);
    }
}

// 16 bytes of a row from column c on; what lies behind the row's d columns counts as zero.
__device__ __forceinline__ uint4 chunk16(const uint8_t *row, int64_t c, int64_t d) {
    uint4 q = make_uint4(0, 0, 0, 0);
    if (c < d) q = *reinterpret_cast<const uint4 *>(row + c);
    const int64_t valid = d - c;
    if (valid < 16) {
        uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t left = valid - 4 * i;
            v[i] = left >= 4 ? v[i] : left <= 0 ? 0u : v[i] & ((1u << (8 * left)) - 1u);
        }
        q = make_uint4(v[0], v[1], v[2], v[3]);
    }
    return q;
}
// A fragment of v_mfma_f32_16x16x128: lane l holds row l % 16.  Which 32 contraction elements a lane holds does not matter as long
// as both operands agree: chunks l / 16 and l / 16 + 4 of the block's eight.
__device__ __forceinline__ i32x8_t fragment(const uint8_t *row, int64_t c, int64_t d) {
    union {
        i32x8_t v;
        uint4 q[2];
    } f;
    f.q[0] = chunk16(row, c, d), f.q[1] = chunk16(row, c + 64, d);
    return f.v;
}

// Bytes 8 q .. 8 q + 7 of a fragment as bf16 numbers.
template <int F8>
__device__ __forceinline__ bf16x8_t widened(const i32x8_t &f, int q) {
    union {
        bf16x8_t v;
        bf16x2_t p[4];
    } o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t u = (uint32_t)f[2 * q + i];
        if constexpr (F8 == F8_E4M3) {
            o.p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, false), o.p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, true);
        } else {
            o.p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(u, 1.0f, false), o.p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(u, 1.0f, true);
        }
    }
    return o.v;
}
// The products of one block of 128: W's fragment times X's.
template <int F8, bool EXACT>
__device__ __forceinline__ f32x4_t times(const i32x8_t &w, const i32x8_t &x) {
    f32x4_t part = {0, 0, 0, 0};
    if constexpr (EXACT) {
#pragma unroll
        for (int q = 0; q < 4; ++q) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened<F8_E4M3>(w, q), widened<F8>(x, q), part, 0, 0, 0);
    } else {
        part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, part, 0, F8, 0, 0, 0, 0);
    }
    return part;
}

// Simplest form: a wave for each 16 x 16 outputs, operands from memory.  W is the first operand of the MFMA, so that a
// lane holds four outputs o .. o + 3 of one token.
template <typename T, int F8, int SCALE>
__global__ void __launch_bounds__(256) linear8_simple_kernel(Linear8Args g) {
    const int lane = threadIdx.x & 63;
    const int64_t tiles_o = (g.d_out + 15) / 16, tiles = tiles_o * ((g.n + 15) / 16);
    for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < tiles; tile += (int64_t)gridDim.x * 4) {
        const int64_t o0 = tile % tiles_o * 16, t0 = tile / tiles_o * 16;
        const int64_t o = min(o0 + (lane & 15), g.d_out - 1), t = min(t0 + (lane & 15), g.n - 1);
        const uint8_t *wr = g.w.data + o * g.w.ld, *xr = g.x.data + t * g.x.ld;
        f32x4_t acc = {0, 0, 0, 0};
        for (int64_t c = 0, b = 0; c < g.d_in; c += kBlock8, ++b) {
            const int64_t at = c + (lane >> 4) * 16;
            const f32x4_t part = times<F8, sizeof(T) == 4>(fragment(wr, at, g.d_in), fragment(xr, at, g.d_in));
            const float s = scale_at<SCALE>(g.x.scales, b * g.x.ld_scales + t) *
                            scale_at<SCALE>(g.w.scales, o0 / kBlock8 * g.w.ld_scales + b);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r] = fmaf(part[r], s, acc[r]);
        }
        if (t0 + (lane & 15) < g.n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t oo = o0 + 4 * (lane >> 4) + r;
                if (oo < g.d_out)
                    store_f32<T>((T *)g.Y + t * g.d_out + oo, g.bias != nullptr ? acc[r] + load_f32<T>((const T *)g.bias + oo) : acc[r]);
            }
    }
}

}  // namespace

template <typename T>
hipError_t launch_linear8(const Mat8 &X, const Mat8 &W, const T *bias, T *Y, int64_t n, int64_t d_in, int64_t d_out, int f8, int scale,
                          hipStream_t stream) {
    const Linear8Args g = {X, W, bias, Y, n, d_in, d_out};
    const int64_t groups = ((d_out + 15) / 16 * ((n + 15) / 16) + 3) / 4;
    const unsigned grid = (unsigned)(groups < (1 << 20) ? groups : (1 << 20));
    if (f8 == F8_E4M3) {
        if (scale == SCALE_F32)
            linear8_simple_kernel<T, F8_E4M3, SCALE_F32><<<grid, 256, 0, stream>>>(g);
        else
            linear8_simple_kernel<T, F8_E4M3, SCALE_E8M0><<<grid, 256, 0, stream>>>(g);
    } else {
        if (scale == SCALE_F32)
            linear8_simple_kernel<T, F8_E5M2, SCALE_F32><<<grid, 256, 0, stream>>>(g);
        else
            linear8_simple_kernel<T, F8_E5M2, SCALE_E8M0><<<grid, 256, 0, stream>>>(g);
    }
    return hipGetLastError();
}

template hipError_t launch_linear8<bf16_t>(const Mat8 &, const Mat8 &, const bf16_t *, bf16_t *, int64_t, int64_t, int64_t, int, int, hipStream_t);
template hipError_t launch_linear8<float>(const Mat8 &, const Mat8 &, const float *, float *, int64_t, int64_t, int64_t, int, int, hipStream_t);

}  // namespace rmm
