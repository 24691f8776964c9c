// Y = X W^T with 8-bit operands where there are few outputs: a single token to a few hundred.
//
// What bounds these is the time to the first operand and how much is in flight, not the matrix unit: a work-group has 16 TU
// outputs of 16 TT tokens, its waves take the blocks of 128 contraction elements in turns, and each loads its fragments from
// memory as the matrix instruction wants them, the next block's under this one's products.  No LDS, no barrier, until the waves'
// sums are added at the end, in the order of the waves.
#pragma once
#include "linear8_frag.hpp"

namespace rmm {

namespace {

// What a wave holds of a block.
template <int TT, int TU, int SCALE>
struct FewBlock {
    i32x8_t x[TT], w[TU];
    uint32_t xs[TT], ws[TU];  // scales as stored
};

// 32 bytes of a row's block: chunks g4 and g4 + 4 (which of them a lane holds does not matter as long as both operands agree).
__device__ __forceinline__ i32x8_t few_fragment(const uint8_t *row, int64_t c, int64_t d) {
    union {
        i32x8_t v;
        uint4 q[2];
    } f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t at = c + 64 * h;
        f.q[h] = at < d ? *reinterpret_cast<const uint4 *>(row + at) : make_uint4(0, 0, 0, 0);
        if (at < d && d - at < 16) f.q[h] = first_bytes(f.q[h], d - at);
    }
    return f.v;
}

template <typename T, int F8, int SCALE, int TT, int TU, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) linear8_few_kernel(Linear8Args g) {
    constexpr bool EXACT = sizeof(T) == 4;
    __shared__ f32x4_t sums[WAVES][TT * TU][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), i16 = lane & 15, g4 = lane >> 4;
    const int64_t tiles_o = (g.d_out + 16 * TU - 1) / (16 * TU), tiles = tiles_o * ((g.n + 16 * TT - 1) / (16 * TT));
    const int64_t blocks = (g.d_in + kBlock8 - 1) / kBlock8, whole = g.d_in / kBlock8;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t o0 = tile % tiles_o * (16 * TU), t0 = tile / tiles_o * (16 * TT);
        const uint8_t *xr[TT], *wr[TU];
        int64_t xs_at[TT], ws_at[TU];
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const int64_t t = min(t0 + 16 * j + i16, g.n - 1);
            xr[j] = g.x.data + t * g.x.ld + g4 * 16, xs_at[j] = t;
        }
#pragma unroll
        for (int u = 0; u < TU; ++u) {
            wr[u] = g.w.data + min(o0 + 16 * u + i16, g.d_out - 1) * g.w.ld + g4 * 16;
            ws_at[u] = min(o0 + 16 * u, g.d_out - 1) / kBlock8 * g.w.ld_scales;  // (16 outputs lie in one block)
        }
        auto stored = [](const void *scales, int64_t at) -> uint32_t {
            if constexpr (SCALE == SCALE_F32)
                return reinterpret_cast<const uint32_t *>(scales)[at];
            else
                return reinterpret_cast<const uint8_t *>(scales)[at];
        };
        auto take = [&](FewBlock<TT, TU, SCALE> &f, int64_t b) __attribute__((always_inline)) {
            const int64_t c = b * kBlock8;
            if (b < whole) {
#pragma unroll
                for (int u = 0; u < TU; ++u) {
                    reinterpret_cast<uint4 *>(&f.w[u])[0] = *reinterpret_cast<const uint4 *>(wr[u] + c);
                    reinterpret_cast<uint4 *>(&f.w[u])[1] = *reinterpret_cast<const uint4 *>(wr[u] + c + 64);
                }
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    reinterpret_cast<uint4 *>(&f.x[j])[0] = *reinterpret_cast<const uint4 *>(xr[j] + c);
                    reinterpret_cast<uint4 *>(&f.x[j])[1] = *reinterpret_cast<const uint4 *>(xr[j] + c + 64);
                }
            } else {
#pragma unroll
                for (int u = 0; u < TU; ++u) f.w[u] = few_fragment(wr[u] - g4 * 16, c + g4 * 16, g.d_in);
#pragma unroll
                for (int j = 0; j < TT; ++j) f.x[j] = few_fragment(xr[j] - g4 * 16, c + g4 * 16, g.d_in);
            }
#pragma unroll
            for (int j = 0; j < TT; ++j) f.xs[j] = stored(g.x.scales, b * g.x.ld_scales + xs_at[j]);
#pragma unroll
            for (int u = 0; u < TU; ++u) f.ws[u] = stored(g.w.scales, ws_at[u] + b);
        };
        f32x4_t acc[TU][TT];
#pragma unroll
        for (int u = 0; u < TU; ++u)
#pragma unroll
            for (int j = 0; j < TT; ++j) acc[u][j] = (f32x4_t){0, 0, 0, 0};
        auto value = [](uint32_t s) { return SCALE == SCALE_F32 ? __uint_as_float(s) : e8m0_to_f32(s); };
        auto multiply = [&](const FewBlock<TT, TU, SCALE> &f) __attribute__((always_inline)) {
            [[maybe_unused]] bf16x8_t xw[EXACT ? TT : 1][4];
            if constexpr (EXACT) {
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) xw[j][q] = widened<F8>(f.x[j], q);
            }
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                [[maybe_unused]] bf16x8_t ww[4];
                if constexpr (EXACT) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) ww[q] = widened<F8_E4M3>(f.w[u], q);
                }
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    f32x4_t part;
                    if constexpr (EXACT)
                        part = block_products(ww, xw[j]);
                    else
                        part = block_products<F8>(f.w[u], f.x[j]);
                    const float s = value(f.xs[j]) * value(f.ws[u]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[u][j][r] = fmaf(part[r], s, acc[u][j][r]);
                }
            }
        };
        FewBlock<TT, TU, SCALE> now, next;
        if (wave < blocks) take(now, wave);
        for (int64_t b = wave; b < blocks; b += 2 * WAVES) {
            if (b + WAVES < blocks) take(next, b + WAVES);
            multiply(now);
            if (b + 2 * WAVES < blocks) take(now, b + 2 * WAVES);
            if (b + WAVES < blocks) multiply(next);
        }
        __syncthreads();  // (the tile before has been read)
#pragma unroll
        for (int u = 0; u < TU; ++u)
#pragma unroll
            for (int j = 0; j < TT; ++j) sums[wave][u * TT + j][lane] = acc[u][j];
        __syncthreads();
        for (int p = wave; p < TU * TT; p += WAVES) {
            f32x4_t y = sums[0][p][lane];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) y += sums[k][p][lane];
            const int64_t o = o0 + p / TT * 16 + 4 * g4, t = t0 + p % TT * 16 + i16, valid = g.d_out - o;
            if (t < g.n && valid > 0) {
                if (g.bias != nullptr)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (r < valid) y[r] += load_f32<T>((const T *)g.bias + o + r);
                store4<T>((T *)g.Y + t * g.d_out + o, valid, y);
            }
        }
    }
}

template <typename T, int F8, int SCALE, int TT, int TU, int WAVES>
void launch_few(const Linear8Args &g, hipStream_t stream) {
    const int64_t tiles = (g.n + 16 * TT - 1) / (16 * TT) * ((g.d_out + 16 * TU - 1) / (16 * TU));
    linear8_few_kernel<T, F8, SCALE, TT, TU, WAVES><<<(unsigned)(tiles < (1 << 22) ? tiles : (1 << 22)), 64 * WAVES, 0, stream>>>(g);
}

}  // namespace

}  // namespace rmm
