// Y = X W^T (+ bias) with 8-bit operands: Y(i, o) = sum over blocks b of 128 contraction elements of
// sx(b, i) sw(o / 128, b) * (sum over the block of X W), in fp32.  Host side, and the kernel without tiles.
#include "linear8_frag.hpp"

namespace rmm {

namespace {

// 16 bytes of a row from column c on; what lies behind the row's d columns counts as zero.
__device__ __forceinline__ uint4 chunk16(const uint8_t *row, int64_t c, int64_t d) {
    if (c >= d) return make_uint4(0, 0, 0, 0);
    const uint4 q = *reinterpret_cast<const uint4 *>(row + c);
    return d - c < 16 ? first_bytes(q, d - c) : q;
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
            const i32x8_t wf = fragment(wr, at, g.d_in), xf = fragment(xr, at, g.d_in);
            f32x4_t part;
            if constexpr (sizeof(T) == 4) {
                bf16x8_t ww[4], xw[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) ww[q] = widened<F8_E4M3>(wf, q), xw[q] = widened<F8>(xf, q);
                part = block_products(ww, xw);
            } else {
                part = block_products<F8>(wf, xf);
            }
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

template <int F8, int SCALE, typename T>
void launch_by_size(const Linear8Args &g, hipStream_t stream) {
    const int64_t large = (g.n + 255) / 256 * ((g.d_out + 255) / 256), mid = (g.n + 127) / 128 * ((g.d_out + 127) / 128);
    if (g.x.ld < (1 << 23) && g.w.ld < (1 << 23) && g.n > 64 && mid < (1 << 23)) {  // (offsets within a tile, and the grid, in 32 bits)
        return launch_linear8_tiles<F8, SCALE, T>(g, large >= 192, stream);
    }
    const int64_t groups = ((g.d_out + 15) / 16 * ((g.n + 15) / 16) + 3) / 4;
    linear8_simple_kernel<T, F8, SCALE><<<(unsigned)(groups < (1 << 20) ? groups : (1 << 20)), 256, 0, stream>>>(g);
}

}  // namespace

template <typename T>
hipError_t launch_linear8(const Mat8 &X, const Mat8 &W, const T *bias, T *Y, int64_t n, int64_t d_in, int64_t d_out, int f8, int scale,
                          hipStream_t stream) {
    const Linear8Args g = {X, W, bias, Y, n, d_in, d_out};
    if (f8 == F8_E4M3)
        scale == SCALE_F32 ? launch_by_size<F8_E4M3, SCALE_F32, T>(g, stream) : launch_by_size<F8_E4M3, SCALE_E8M0, T>(g, stream);
    else
        scale == SCALE_F32 ? launch_by_size<F8_E5M2, SCALE_F32, T>(g, stream) : launch_by_size<F8_E5M2, SCALE_E8M0, T>(g, stream);
    return hipGetLastError();
}

template hipError_t launch_linear8<bf16_t>(const Mat8 &, const Mat8 &, const bf16_t *, bf16_t *, int64_t, int64_t, int64_t, int, int, hipStream_t);
template hipError_t launch_linear8<float>(const Mat8 &, const Mat8 &, const float *, float *, int64_t, int64_t, int64_t, int, int, hipStream_t);

}  // namespace rmm
