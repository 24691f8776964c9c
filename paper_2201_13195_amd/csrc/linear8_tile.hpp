// Y = X W^T with 8-bit operands on tiles of BT tokens x BO outputs.
//
// The contraction goes in steps of 128 elements, one block of the scales and one v_mfma_f32_16x16x128 deep.  Both operands go
// from memory straight into LDS (rows of 128 bytes, whole lines; chunk c of row r at position c ^ (r / 2 % 8), so that 16 rows
// are read without bank conflicts), in two stages, the step's scales behind them.  W is the first operand of the MFMA: a lane then
// holds outputs of one token, one scale of X a token tile is enough, and the scale of W is the same for the whole wave.
//   powers of two      the matrix instruction multiplies by both scales itself
//   fp32 scales        it starts from zero, and four fused multiply-adds add its result times the product of the scales
//   fp32 result        (exact) both operands widened to bf16, four MFMAs of 32, then as fp32 scales
//
// Which row of a wave's part goes to which LDS row is free, as the loads take it from any address:
//   tokens    LDS row 16 j + i holds token TJ i + j: the scales of a lane's TJ tokens are consecutive
//   outputs   LDS row 32 v + 16 h + 4 a + r holds output 32 v + 8 a + 4 h + r: a lane's results of two neighbouring tiles are eight
//             consecutive outputs, its 16 neighbours' the next
#pragma once
#include "lds_loads.hpp"
#include "linear8_frag.hpp"

#include <utility>

namespace rmm {

namespace {

// f(0), f(1), .. f(N - 1) with constants.
template <typename F, int... I>
__device__ __forceinline__ void for_each_of(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void for_each(F f) {
    for_each_of(std::make_integer_sequence<int, N>(), f);
}

// BT x BO outputs on NT x NO waves; PD fragments of W are read ahead, so that one barrier a step stands PD fragments before its
// end; the loads of a step are spread over SPAN MFMAs behind it.
template <int BT_, int BO_, int NT_, int NO_, int PD_, int SPAN_, int PER_SIMD_>
struct Tile8 {
    static constexpr int BT = BT_, BO = BO_, NT = NT_, NO = NO_, PD = PD_, SPAN = SPAN_, PER_SIMD = PER_SIMD_;
    static constexpr int WAVES = NT * NO, THREADS = 64 * WAVES;
    static constexpr int WT = BT / NT, WO = BO / NO, TJ = WT / 16, TU = WO / 16;  // of a wave: rows, 16-row tiles
    static constexpr int JX = BT / 8 / WAVES, JW = BO / 8 / WAVES, LOADS = JX + JW + 1;  // 1 KB loads of a wave and step, one of scales
    static constexpr int X_BYTES = BT * 128, W_BYTES = BO * 128, STAGE = X_BYTES + W_BYTES;
    static constexpr int XS_BYTES = BT * 4, SCALES = XS_BYTES + 256;  // of a stage: X's, W's
    static constexpr int LDS_BYTES = 2 * STAGE + 2 * SCALES + 256;  // (the last 256: of waves without a share of the scales)
    static constexpr int MFMAS = TU * TJ;
    static_assert(BT % (8 * WAVES) == 0 && BO % (8 * WAVES) == 0 && WT % 64 == 0 && WO % 64 == 0 && 128 % WO == 0, "shares of a wave");
    static_assert(PD == 3 && TU % 4 == 0 && SPAN <= MFMAS && LDS_BYTES <= 160 * 1024, "ring of four fragments");
};

// One row-major operand on its way into LDS, J loads of a wave: 32-bit offsets from the tile's first row.
template <int J>
struct Loads8 {
    u32x4_t rsrc;
    uint32_t off[J], beyond[2], to, range;
    // `row_of`: which row (of the tile) LDS row r holds
    template <typename F>
    __device__ __forceinline__ void init(const uint8_t *first, int64_t ld, int64_t rows, int64_t d, uint32_t lds, int wave, int lane, F row_of) {
        const uint64_t at = reinterpret_cast<uint64_t>(first);
        range = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(rows * ld));
        rsrc = (u32x4_t){(uint32_t)__builtin_amdgcn_readfirstlane((int)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)), range, 0x00020000u};
        to = lds + (uint32_t)(wave * J * 1024);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = (wave * J + j) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            const int64_t from = row_of(row);
            off[j] = from < rows ? (uint32_t)(from * ld) + (uint32_t)chunk * 16u : 0x80000000u;
            if (j < 2) beyond[j] = chunk * 16 < (int)((d - 1) % 128) + 1 ? 0u : 0x80000000u;  // in the last step
        }
        settle(rsrc);
    }
    // Load j of the step at byte `soff` of the rows into stage byte `stage`.
    __device__ __forceinline__ void load(int j, uint32_t stage, uint32_t soff, uint32_t last) const {
        load_to_lds(rsrc, to + stage + (uint32_t)j * 1024u, off[j] | (last & beyond[j & 1]), soff);
    }
};

// One wave's load of a dword a lane into 256 bytes of LDS.
__device__ __forceinline__ void load_dwords_to_lds(u32x4_t rsrc, uint32_t to, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(rsrc) : "m0");
}

// The wave's share of a step's scales: 64 dwords of X's, W's, or none (zeros to where nobody reads).  No branches: what differs
// between the shares are numbers.  A scale of W in one byte comes as the dword around it.
template <typename S, int SCALE>
struct ScaleLoads8 {
    static constexpr int SIZE = SCALE == SCALE_F32 ? 4 : 1, XL = S::BT * SIZE <= 256 ? 1 : S::BT * SIZE / 256;
    static_assert(XL + 1 <= S::WAVES, "a wave loads at most one share of the scales");
    uint64_t base, base_step;  // X: from step to step
    uint32_t off, off_step, range, to, stage_bytes;
    __device__ __forceinline__ void init(const Linear8Args &g, int64_t t0, int64_t o0, uint32_t lds, uint32_t idle, int wave, int lane) {
        if (wave < XL) {
            const int64_t first = t0 + wave * (256 / SIZE), left = g.n - first;
            base = reinterpret_cast<uint64_t>(g.x.scales) + (uint64_t)first * SIZE, base_step = (uint64_t)g.x.ld_scales * SIZE;
            range = left > 0 ? (uint32_t)((min((int64_t)(256 / SIZE), left) * SIZE + 3) & ~(int64_t)3) : 0u;
            off = lane * 4, off_step = 0, to = lds + wave * 256, stage_bytes = S::SCALES;
        } else if (wave == XL) {
            const int64_t blocks = (g.d_out + kBlock8 - 1) / kBlock8 - o0 / kBlock8;
            const uint64_t first = reinterpret_cast<uint64_t>(g.w.scales) + (uint64_t)(o0 / kBlock8 * g.w.ld_scales) * SIZE;
            base = first & ~(uint64_t)3, base_step = 0, range = 0x7FFFFFFFu;
            off = lane < S::BO / kBlock8 && lane < blocks ? (uint32_t)(first & 3) + (uint32_t)(lane * g.w.ld_scales) * SIZE : 0x80000000u;
            off_step = SIZE, to = lds + S::XS_BYTES, stage_bytes = S::SCALES;
        } else {
            base = reinterpret_cast<uint64_t>(g.x.scales), base_step = 0, range = 0, off = 0x80000000u, off_step = 0, to = idle, stage_bytes = 0;
        }
        // (the same in every lane; saying so keeps them in scalar registers)
        base = scalar((uint32_t)base) | (uint64_t)scalar((uint32_t)(base >> 32)) << 32, base_step = scalar((uint32_t)base_step) | (uint64_t)scalar((uint32_t)(base_step >> 32)) << 32;
        range = scalar(range), to = scalar(to), off_step = scalar(off_step), stage_bytes = scalar(stage_bytes);
        asm volatile("s_nop 4" : "+s"(base), "+s"(range), "+s"(to));  // (as settle)
    }
    static __device__ __forceinline__ uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
    __device__ __forceinline__ void load(int stage, bool live) {
        const u32x4_t rsrc = {(uint32_t)base, (uint32_t)(base >> 32), live ? range : 0u, 0x00020000u};
        load_dwords_to_lds(rsrc, to + (uint32_t)stage * stage_bytes, off & ~3u);
        base += base_step, off += off_step;
    }
};

// CUT: the contraction is no multiple of 16.
template <typename S, int F8, int SCALE, typename T, bool CUT>
__global__ void __launch_bounds__(S::THREADS, S::PER_SIMD) linear8_tile_kernel(Linear8Args g) {
    constexpr bool EXACT = sizeof(T) == 4, IN_MFMA = SCALE == SCALE_E8M0 && !EXACT;
    constexpr int TJ = S::TJ, TU = S::TU, PD = S::PD, BT = S::BT, BO = S::BO;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::LDS_BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave / S::NO, wo = wave % S::NO, i16 = lane & 15, g4 = lane >> 4;
    // Work-groups are dealt round-robin to the 8 XCDs, each with an L2 of its own: one XCD gets a run of consecutive positions, and
    // positions go through bands of eight tile rows (tokens), column by column, so that what runs on an XCD shares rows of both.
    const uint32_t tiles_t = (uint32_t)((g.n + BT - 1) / BT), tiles_o = (uint32_t)((g.d_out + BO - 1) / BO);
    int64_t t0, o0;
    {
        const uint32_t blocks = gridDim.x, per = blocks / 8, rem = blocks % 8, x = blockIdx.x % 8, r = blockIdx.x / 8;
        const uint32_t tile = x * per + (x < rem ? x : rem) + r, band = tile / (8 * tiles_o), in = tile - band * 8 * tiles_o;
        const uint32_t rows = min(8u, tiles_t - band * 8), col = in / rows;
        t0 = (int64_t)(band * 8 + in - col * rows) * BT, o0 = (int64_t)col * BO;
    }
    const int steps = (int)((g.d_in + kBlock8 - 1) / kBlock8);

    typedef __attribute__((address_space(3))) unsigned char *lds_ptr_t;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    Loads8<S::JX> lx;
    Loads8<S::JW> lw;
    ScaleLoads8<S, SCALE> ls;
    lx.init(g.x.data + t0 * g.x.ld, g.x.ld, min((int64_t)BT, g.n - t0), g.d_in, lds0, wave, lane,
            [](int r) { return (int64_t)(r / S::WT * S::WT + r % 16 * TJ + r % S::WT / 16); });
    lw.init(g.w.data + o0 * g.w.ld, g.w.ld, min((int64_t)BO, g.d_out - o0), g.d_in, lds0 + S::X_BYTES, wave, lane,
            [](int r) { return (int64_t)(r / 32 * 32 + r % 16 / 4 * 8 + r / 16 % 2 * 4 + r % 4); });
    ls.init(g, t0, o0, lds0 + 2 * S::STAGE, lds0 + 2 * S::STAGE + 2 * S::SCALES, wave, lane);
    // The step that is being requested, and the stage (as bytes) it goes to.
    int asked = 0;
    uint32_t soff = 0, last = 0, into = 0;
    bool live = true;
    auto begin = [&](int step, uint32_t stage) {
        live = step < steps, soff = (uint32_t)step * 128u, last = step == steps - 1 ? 0xFFFFFFFFu : 0u, into = stage;
        lx.rsrc[2] = live ? lx.range : 0u, lw.rsrc[2] = live ? lw.range : 0u;
    };
    auto load = [&](int i) {  // load i of that step: the scales first
        if (i == 0)
            ls.load(into != 0, live);
        else if (i <= S::JX)
            lx.load(i - 1, into, soff, last);
        else
            lw.load(i - 1 - S::JX, into, soff, last);
    };

    // A lane's place in a tile of 16 rows: row i16, chunks g4 and g4 + 4; `from`: the stage that is read (as bytes).
    const uint32_t at0 = (uint32_t)(i16 * 128 + ((g4 ^ ((i16 >> 1) & 7)) << 4)), at1 = at0 ^ 64u;
    uint32_t from = 0, x0 = at0 + wt * S::WT * 128, x1 = at1 + wt * S::WT * 128, w0 = at0 + S::X_BYTES + wo * S::WO * 128, w1 = at1 + S::X_BYTES + wo * S::WO * 128;
    auto turn_to = [&](uint32_t stage) {
        const uint32_t by = stage - from;
        from = stage, x0 += by, x1 += by, w0 += by, w1 += by;
    };
    auto fragment = [&](uint32_t a, uint32_t b, int tile) {
        union {
            i32x8_t v;
            uint4 q[2];
        } f;
        f.q[0] = *reinterpret_cast<const uint4 *>(lds + a + tile * 2048);
        f.q[1] = *reinterpret_cast<const uint4 *>(lds + b + tile * 2048);
        return f.v;
    };

    f32x4_t acc[TU][TJ];
#pragma unroll
    for (int u = 0; u < TU; ++u)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[u][j] = (f32x4_t){0, 0, 0, 0};
    i32x8_t xf[TJ], wf[4];
    // Scales of a step, as read and as used: powers of two as bytes for the matrix instruction, or the products of X's and W's.
    constexpr int XS = SCALE == SCALE_F32 ? TJ : TJ / 4;
    uint32_t xs_read[XS], ws_read, xs[IN_MFMA ? XS : 1], ws = 0;
    float fs[IN_MFMA ? 1 : TJ];
    uint32_t w_byte = (uint32_t)reinterpret_cast<uint64_t>(g.w.scales) + (uint32_t)((o0 + wo * S::WO) / kBlock8 * g.w.ld_scales);  // (of the step's scale)
    auto read_scales = [&] {
        const unsigned char *at = lds + 2 * S::STAGE + (from != 0 ? S::SCALES : 0);
        ws_read = *reinterpret_cast<const uint32_t *>(at + S::XS_BYTES + wo * S::WO / kBlock8 * 4);
#pragma unroll
        for (int q = 0; q < XS; ++q) xs_read[q] = *reinterpret_cast<const uint32_t *>(at + (wt * S::WT + i16 * TJ) * (SCALE == SCALE_F32 ? 4 : 1) + 4 * q);
    };
    auto take_scales = [&] {
        if constexpr (SCALE == SCALE_F32) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) fs[j] = __uint_as_float(xs_read[j]) * __uint_as_float(ws_read);
        } else {
            const uint32_t w = ws_read >> ((w_byte++ & 3) * 8);
            if constexpr (IN_MFMA) {
                ws = w;
#pragma unroll
                for (int q = 0; q < XS; ++q) xs[q] = xs_read[q];
            } else {
#pragma unroll
                for (int j = 0; j < TJ; ++j) fs[j] = e8m0_to_f32(xs_read[j / 4] >> (j % 4 * 8) & 255u) * e8m0_to_f32(w & 255u);
            }
        }
    };
    auto read_first = [&] {  // what a step finds in registers
#pragma unroll
        for (int j = 0; j < TJ; ++j) xf[j] = fragment(x0, x1, j);
#pragma unroll
        for (int u = 0; u < PD; ++u) wf[u] = fragment(w0, w1, u);
    };

    constexpr int TAIL = PD * TJ;  // MFMAs behind the barrier
    constexpr int LOADS = S::LOADS;
    begin(0, 0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(i);
    begin(1, S::STAGE);
    constexpr int EARLY = [] {
        int c = 0;
        for (int i = 0; i < LOADS; ++i) c += i * S::SPAN / LOADS < TAIL ? 1 : 0;
        return c;
    }();
#pragma unroll
    for (int i = 0; i < EARLY; ++i) load(i);
    wait_for_loads<EARLY>();
    __syncthreads();
    read_first();
    read_scales();
    take_scales();
    asked = 1;

    // Step by step: the first fragments and the scales are in registers.  A fragment of X gives its place to the next step's
    // behind its last use, so that one set is enough.
    for (int left = steps; left > 0; --left) {
        if (CUT && left == 1) {
            // The chunk of 16 that the contraction ends in: what lies behind the end becomes zeros, in LDS.
            const int c = (int)(g.d_in % kBlock8) / 16;
            for (int row = tid; row < BT + BO; row += S::THREADS) {
                uint4 *at = reinterpret_cast<uint4 *>(lds + from + row * 128 + ((c ^ ((row >> 1) & 7)) << 4));
                *at = first_bytes(*at, g.d_in % 16);
            }
            __syncthreads();
            read_first();
        }
        [[maybe_unused]] bf16x8_t xw[EXACT ? TJ : 1][4], ww[4];
        if constexpr (EXACT) {
#pragma unroll
            for (int j = 0; j < TJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) xw[j][q] = widened<F8>(xf[j], q);
        }
        [[maybe_unused]] f32x4_t part[3];
        for_each<S::MFMAS + (IN_MFMA ? 0 : 2)>([&](auto index) __attribute__((always_inline)) {
            constexpr int i = decltype(index)::value, u = i / TJ, j = i % TJ, q = i - (TU - PD) * TJ, slot = q >= 0 ? q : i + TAIL;
            if constexpr (q == 0) {  // every fragment of W of this stage is in registers, the next step's data are there
                wait_for_loads<0>();
                __syncthreads();
                begin(++asked, from);
                turn_to(S::STAGE - from);
            }
            if constexpr (i < S::MFMAS) {
                if constexpr (IN_MFMA) {
                    add_scaled_products<F8, j % 4, S::PER_SIMD != 1>(wf[u % 4], xf[j], acc[u][j], ws, xs[j / 4]);
                } else if constexpr (EXACT) {
                    if constexpr (j == 0)
#pragma unroll
                        for (int k = 0; k < 4; ++k) ww[k] = widened<F8_E4M3>(wf[u % 4], k);
                    part[i % 3] = block_products(ww, xw[j]);
                } else {
                    part[i % 3] = block_products<F8>(wf[u % 4], xf[j]);
                }
                if constexpr (!IN_MFMA) pin(part[i % 3]);
                // fragments of W ahead, the scales, and in the last row of tiles X's fragments of the next step
                if constexpr (j == 0) wf[(u + PD) % 4] = fragment(w0, w1, (u + PD) % TU);
                if constexpr (q == 1) read_scales();
                if constexpr (u == TU - 1) xf[j] = fragment(x0, x1, j);
                for_each<LOADS>([&](auto l) __attribute__((always_inline)) {
                    if constexpr (decltype(l)::value * S::SPAN / LOADS == slot) load(decltype(l)::value);
                });
            }
            if constexpr (!IN_MFMA && i >= 2) {
                constexpr int k = i - 2;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[k / TJ][k % TJ][r] = fmaf(part[k % 3][r], fs[k % TJ], acc[k / TJ][k % TJ][r]);
                pin(acc[k / TJ][k % TJ]);
            }
            if constexpr (i < S::MFMAS) __builtin_amdgcn_sched_barrier(0);
        });
        take_scales();
    }
    wait_for_loads<0>();
    if constexpr (IN_MFMA) settle_sums<S::PER_SIMD != 1>(acc);

    // Tiles 2 v and 2 v + 1 hold outputs 32 v + 8 g4 .. + 7 of the lane's tokens.
#pragma unroll
    for (int v = 0; v < TU / 2; ++v) {
        const int64_t o = o0 + wo * S::WO + 32 * v + 8 * g4, valid = g.d_out - o;
        float b[8];
        if (g.bias != nullptr) load8<T>((const T *)g.bias + (valid > 0 ? o : 0), valid, b);
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const int64_t token = t0 + wt * S::WT + i16 * TJ + j;
            float y[8];
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = acc[2 * v][j][r], y[4 + r] = acc[2 * v + 1][j][r];
            if (g.bias != nullptr)
#pragma unroll
                for (int r = 0; r < 8; ++r) y[r] += b[r];
            if (token < g.n) store8<T>((T *)g.Y + token * g.d_out + (valid > 0 ? o : 0), valid, y);
        }
    }
}

// Which product takes which tile.
typedef Tile8<256, 256, 2, 2, 3, 40, 1> Large8;   // 4 waves of 128 x 128, powers of two
typedef Tile8<256, 256, 4, 2, 3, 20, 2> Eight8;   // 8 waves of 64 x 128, fp32 scales
typedef Tile8<128, 128, 2, 2, 3, 12, 2> Mid8;     // 4 waves of 64 x 64

template <typename S, int F8, int SCALE, typename T>
void launch_tile(const Linear8Args &g, hipStream_t stream) {
    const unsigned tiles = (unsigned)((g.n + S::BT - 1) / S::BT * ((g.d_out + S::BO - 1) / S::BO));
    if (g.d_in % 16 != 0)
        linear8_tile_kernel<S, F8, SCALE, T, true><<<tiles, S::THREADS, 0, stream>>>(g);
    else
        linear8_tile_kernel<S, F8, SCALE, T, false><<<tiles, S::THREADS, 0, stream>>>(g);
}

}  // namespace

template <int F8, int SCALE, typename T>
void launch_linear8_tiles(const Linear8Args &g, bool large, hipStream_t stream) {
    if constexpr (sizeof(T) == 2) {
        if (large) return launch_tile<std::conditional_t<SCALE == SCALE_E8M0, Large8, Eight8>, F8, SCALE, T>(g, stream);
    }
    launch_tile<Mid8, F8, SCALE, T>(g, stream);
}

}  // namespace rmm
