// Y = X W^T with 8-bit operands where there are few outputs: a single token to a few hundred.
//
// What bounds these is the time to the first operand and how much is in flight, not the matrix unit: a work-group has 16 TU
// outputs of 16 TT tokens, and its waves take the blocks of 128 contraction elements in turns, each through LDS of its own: whole lines go
// there straight from memory, the next block's as soon as this one's fragments are in registers.  No barrier until the waves'
// sums are added at the end, in the order of the waves.
//   fragments loaded from memory as the matrix instruction wants them (a quarter of a wave's addresses in 16 lines): 1 x 4096 -> 4096
//   5.1 us, 24 x 4096 -> 1024 6.2, 64 x 4096 -> 4096 10.4, 128 x 4096 -> 4096 14.7; like this 4.5, 4.2, 7.0, 8.0
//   two and three blocks of a wave on their way: 1 x 4096 -> 4096 4.5 and 4.7 us (one: 4.6), 24 x 4096 -> 1024 4.4 and 4.6 (4.2),
//   1 x 1024 -> 4096 3.6 (3.3): more code, and LDS holds fewer work-groups
#pragma once
#include "lds_loads.hpp"
#include "linear8_frag.hpp"

namespace rmm {

namespace {

// One wave's load of 64 dwords, or of 1 KB, into LDS from byte `to` on, a dword or 16 bytes from each lane's address (as load_to_lds).
__device__ __forceinline__ void load_dwords_from(uint64_t p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(p) : "m0", "memory");
}
__device__ __forceinline__ void load_chunks_from(uint64_t p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(p) : "m0", "memory");
}

// What of a fragment's 32 bytes, chunks g4 and g4 + 4 of a block, lies in the row; the others become zero.
__device__ __forceinline__ void cut_fragment(i32x8_t &f, int64_t left) {
    union {
        i32x8_t v;
        uint4 q[2];
    } o;
    o.v = f;
    o.q[0] = first_bytes(o.q[0], left), o.q[1] = first_bytes(o.q[1], left - 64);
    f = o.v;
}

// TT x TU tiles of 16 tokens and 16 outputs, WAVES waves.
template <int SCALE, int TT_, int TU_, int WAVES_>
struct Few8 {
    static constexpr int TT = TT_, TU = TU_, WAVES = WAVES_, SIZE = SCALE == SCALE_F32 ? 4 : 1;
    static constexpr int XS = TT * 16 * SIZE / 4, SCALE_LOADS = XS + 1 <= 64 ? 1 : 2;  // dwords of X's scales, one of W's behind them
    static constexpr int TILES = (TT + TU) * 2048, BLOCK = TILES + SCALE_LOADS * 256;  // of a wave
    static constexpr int SUMS = WAVES * TT * TU * 1024, LDS_BYTES = WAVES * BLOCK > SUMS ? WAVES * BLOCK : SUMS;
    static_assert(XS <= 64 && LDS_BYTES <= 160 * 1024, "one load of X's scales");
};

template <typename T, int F8, int SCALE, typename S>
__global__ void __launch_bounds__(64 * S::WAVES, 2) linear8_few_kernel(Linear8Args g) {
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int TT = S::TT, TU = S::TU, WAVES = S::WAVES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), i16 = lane & 15, g4 = lane >> 4;
    const int64_t tiles_o = (g.d_out + 16 * TU - 1) / (16 * TU), tiles = tiles_o * ((g.n + 16 * TT - 1) / (16 * TT));
    const int64_t blocks = (g.d_in + kBlock8 - 1) / kBlock8, whole = g.d_in / kBlock8;
    unsigned char *const mine = lds + wave * S::BLOCK;
    typedef __attribute__((address_space(3))) unsigned char *lds_ptr_t;
    const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_ptr_t)mine);
    // A load fills eight rows of 128 bytes, chunk c of row r at position c ^ (r / 2 % 8) (as in linear8_tile.hpp): lane l brings position
    // l % 8 of row l / 8.
    const int row8 = lane >> 3, chunk[2] = {(lane & 7) ^ (lane >> 4), (lane & 7) ^ (4 + (lane >> 4))};
    const uint32_t at0 = (uint32_t)(i16 * 128 + ((g4 ^ ((i16 >> 1) & 7)) << 4)), at1 = at0 ^ 64u;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t o0 = tile % tiles_o * (16 * TU), t0 = tile / tiles_o * (16 * TT);
        uint64_t row[TT + TU][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < TT; ++j) row[j][h] = reinterpret_cast<uint64_t>(g.x.data) + (uint64_t)(min(t0 + 16 * j + 8 * h + row8, g.n - 1) * g.x.ld);
#pragma unroll
            for (int u = 0; u < TU; ++u) row[TT + u][h] = reinterpret_cast<uint64_t>(g.w.data) + (uint64_t)(min(o0 + 16 * u + 8 * h + row8, g.d_out - 1) * g.w.ld);
        }
        // Scales: the dwords of X's from token t0 on (those that do not exist: the last one's), W's around its one (16 TU outputs lie in one block).
        const int64_t x_dword = min((int64_t)lane * (4 / S::SIZE), (g.n - 1 - t0) / (4 / S::SIZE) * (4 / S::SIZE));
        const uint64_t x_scale = reinterpret_cast<uint64_t>(g.x.scales) + (uint64_t)((t0 + x_dword) * S::SIZE);
        const uint64_t w_scale = reinterpret_cast<uint64_t>(g.w.scales) + (uint64_t)(o0 / kBlock8 * g.w.ld_scales * S::SIZE);
        auto request = [&](int64_t b) __attribute__((always_inline)) {
            const int64_t c = b * kBlock8;
            const uint64_t xs = x_scale + (uint64_t)(b * g.x.ld_scales * S::SIZE), ws = (w_scale + (uint64_t)(b * S::SIZE)) & ~(uint64_t)3;
            if constexpr (S::SCALE_LOADS == 1) {
                load_dwords_from(lane < S::XS ? xs : ws, lds0 + S::TILES);
            } else {
                load_dwords_from(xs, lds0 + S::TILES);
                load_dwords_from(ws, lds0 + S::TILES + 256);
            }
            uint64_t at[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) at[h] = (uint64_t)(c + (c + chunk[h] * 16 < g.d_in ? chunk[h] * 16 : 0));  // (what is behind the end is cut off later)
#pragma unroll
            for (int k = 0; k < TT + TU; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) load_chunks_from(row[k][h] + at[h], lds0 + (uint32_t)(k * 2048 + h * 1024));
        };
        f32x4_t acc[TU][TT];
#pragma unroll
        for (int u = 0; u < TU; ++u)
#pragma unroll
            for (int j = 0; j < TT; ++j) acc[u][j] = (f32x4_t){0, 0, 0, 0};
        auto stored = [&](int i) -> uint32_t {
            if constexpr (SCALE == SCALE_F32)
                return reinterpret_cast<const uint32_t *>(mine + S::TILES)[i];
            else
                return (mine + S::TILES)[i];
        };
        auto fragment = [&](int tile) {
            union {
                i32x8_t v;
                uint4 q[2];
            } f;
            f.q[0] = *reinterpret_cast<const uint4 *>(mine + tile * 2048 + at0), f.q[1] = *reinterpret_cast<const uint4 *>(mine + tile * 2048 + at1);
            return f.v;
        };
        if (wave < blocks) request(wave);
        for (int64_t b = wave; b < blocks; b += WAVES) {
            i32x8_t x[TT], w[TU];
            float s[TT];
            [[maybe_unused]] uint32_t rest[SCALE == SCALE_F32 ? 1 : TT];
            wait_for_loads<0>();
#pragma unroll
            for (int u = 0; u < TU; ++u) w[u] = fragment(TT + u);
#pragma unroll
            for (int j = 0; j < TT; ++j) x[j] = fragment(j);
            if constexpr (SCALE == SCALE_F32) {
                const float ws = __uint_as_float(stored(S::XS));
#pragma unroll
                for (int j = 0; j < TT; ++j) s[j] = __uint_as_float(stored(16 * j + i16)) * ws;
            } else {
                const uint32_t ws = stored(S::XS * 4 + (int)((uint32_t)(w_scale + (uint64_t)b) & 3u));
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    const PowerProduct p = power_product(stored(16 * j + i16), ws);
                    s[j] = p.s, rest[j] = p.rest;
                }
            }
            if (b + WAVES < blocks) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the block has been read)
                request(b + WAVES);
            }
            if (b >= whole) {
                const int64_t left = g.d_in - b * kBlock8 - g4 * 16;
#pragma unroll
                for (int u = 0; u < TU; ++u) cut_fragment(w[u], left);
#pragma unroll
                for (int j = 0; j < TT; ++j) cut_fragment(x[j], left);
            }
            [[maybe_unused]] bf16x8_t xw[EXACT ? TT : 1][4];
            if constexpr (EXACT) {
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) xw[j][q] = widened<F8>(x[j], q, SCALE == SCALE_F32 ? 1.0f : __uint_as_float(rest[SCALE == SCALE_F32 ? 0 : j] << 23));
            }
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                [[maybe_unused]] bf16x8_t ww[4];
                if constexpr (EXACT) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) ww[q] = widened<F8_E4M3>(w[u], q);
                }
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    f32x4_t part;
                    if constexpr (EXACT)
                        part = block_products(ww, xw[j]);
                    else if constexpr (SCALE == SCALE_F32)
                        part = block_products<F8>(w[u], x[j]);
                    else
                        part = block_products<F8>(w[u], x[j], rest[j]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[u][j][r] = fmaf(part[r], s[j], acc[u][j][r]);
                }
            }
        }
        __syncthreads();  // (the sums take the place of the blocks)
        f32x4_t *const sums = reinterpret_cast<f32x4_t *>(lds) + lane;
#pragma unroll
        for (int u = 0; u < TU; ++u)
#pragma unroll
            for (int j = 0; j < TT; ++j) sums[(wave * TU * TT + u * TT + j) * 64] = acc[u][j];
        __syncthreads();
        for (int p = wave; p < TU * TT; p += WAVES) {
            f32x4_t y = sums[p * 64];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) y += sums[(k * TU * TT + p) * 64];
            const int64_t o = o0 + p / TT * 16 + 4 * g4, t = t0 + p % TT * 16 + i16, valid = g.d_out - o;
            if (t < g.n && valid > 0) {
                if (g.bias != nullptr)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (r < valid) y[r] += load_f32<T>((const T *)g.bias + o + r);
                store4<T>((T *)g.Y + t * g.d_out + o, valid, y);
            }
        }
        if (tile + gridDim.x < tiles) __syncthreads();  // (the blocks of the next tile take the place of the sums)
    }
}

template <typename T, int F8, int SCALE, int TT, int TU, int WAVES>
void launch_few(const Linear8Args &g, hipStream_t stream) {
    typedef Few8<SCALE, TT, TU, WAVES> S;
    const int64_t tiles = (g.n + 16 * TT - 1) / (16 * TT) * ((g.d_out + 16 * TU - 1) / (16 * TU));
    linear8_few_kernel<T, F8, SCALE, S><<<(unsigned)(tiles < (1 << 22) ? tiles : (1 << 22)), 64 * WAVES, S::LDS_BYTES, stream>>>(g);
}

}  // namespace

}  // namespace rmm
