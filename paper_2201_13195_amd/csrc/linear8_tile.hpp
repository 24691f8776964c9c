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

// BT x BO outputs on NT x NO waves.  PD fragments of W are read ahead, so that the one barrier of a step stands PD fragments before
// its end, and the loads of the step that is STAGES ahead, into the stage that is free then, have STAGES - 1 steps to arrive.  They are
// spread over the MFMAs behind the barrier.  KS groups of such waves share the contraction, every KS-th step a group's; each has stages of
// its own, and the barrier is one for all.  Measured beside what is below, bf16 results, the same operands again and again, in us:
//   - 128 x 128 tiles, four stages and one group: 1024 x 4096 -> 4096 with powers of two 23.8, with fp32 scales 25.9 (two groups of two
//     stages 24.8, 24.9); one group leaves a SIMD one wave, whose reads nothing hides
//   - 64 x 128 tiles, two groups of two stages: 512 x 4096 -> 4096 19.5 (three stages 16.9); one group of five 21.8
//   - a second barrier, behind which half of a 256 x 256 tile's loads have half a step more: 16384 x 4096 -> 4096 with powers of two
//     217 -> 212, with fp32 scales 228 -> 236
//   - every other tile backwards along the contraction: 16384 x 4096 -> 4096 with powers of two 207 -> 209
template <int BT_, int BO_, int NT_, int NO_, int KS_, int STAGES_>
struct Tile8 {
    static constexpr int BT = BT_, BO = BO_, NT = NT_, NO = NO_, KS = KS_, STAGES = STAGES_, PD = 3;
    static constexpr int WAVES = NT * NO, THREADS = 64 * WAVES * KS;  // waves of a group
    static constexpr int WT = BT / NT, WO = BO / NO, TJ = WT / 16, TU = WO / 16;  // of a wave: rows, 16-row tiles
    static constexpr int JX = BT / 8 / WAVES, JW = BO / 8 / WAVES, LOADS = JX + JW + 1;  // 1 KB loads of a wave and step, one of scales
    static constexpr int X_BYTES = BT * 128, W_BYTES = BO * 128, STAGE = X_BYTES + W_BYTES;
    static constexpr int XS_BYTES = BT * 4, SCALES = XS_BYTES + 256;  // of a stage: X's, W's
    static constexpr int GROUP = STAGES * (STAGE + SCALES), LDS_BYTES = KS * GROUP + 256;  // (the last 256: of waves without a share of the scales)
    static constexpr int MFMAS = TU * TJ;
    static_assert(BT % (8 * WAVES) == 0 && BO % (8 * WAVES) == 0 && WT % 64 == 0 && WO % 64 == 0 && 128 % WO == 0, "shares of a wave");
    static_assert(KS == 1 || (KS == 2 && TU % 4 == 0 && WAVES * TU * TJ * 1024 <= LDS_BYTES), "each of two groups sums half of the outputs");
    static_assert(PD == 3 && TU % 4 == 0 && LOADS <= 2 * PD * TJ && LDS_BYTES <= 160 * 1024, "ring of four fragments, loads behind the barrier");
    static_assert(KS == 1 ? STAGES == 2 : STAGES >= 2, "requests reach into one further tile; with two groups there is none");
};

// A wave-uniform value, which the compiler then keeps in a scalar register.
__device__ __forceinline__ uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ uint64_t scalar(uint64_t v) { return scalar((uint32_t)v) | (uint64_t)scalar((uint32_t)(v >> 32)) << 32; }

// Bytes that a descriptor spans: the rows of an operand that a tile has, dense up to their pitch.
struct Span {
    uint64_t base;
    uint32_t range;
    __device__ __forceinline__ u32x4_t descriptor() const { return (u32x4_t){(uint32_t)base, (uint32_t)(base >> 32), range, 0x00020000u}; }
};
__device__ __forceinline__ Span rows_of(const Mat8 &m, int64_t row0, int64_t rows, bool there) {
    return {scalar(reinterpret_cast<uint64_t>(m.data) + (uint64_t)(row0 * m.ld)), scalar(there ? (uint32_t)(rows * m.ld) : 0u)};
}

// One row-major operand on its way into LDS, J loads of a wave: 32-bit offsets from the tile's first row.  Rows that the tile does
// not have lie behind the descriptor's range: zeros.
template <int J>
struct Loads8 {
    Span at;
    uint32_t off[J], beyond[2], to;
    // `row_of`: which row (of the tile) LDS row r holds
    template <typename F>
    __device__ __forceinline__ void init(int64_t ld, int64_t d, uint32_t lds, int wave, int lane, F row_of) {
        to = scalar(lds + (uint32_t)(wave * J * 1024));
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = (wave * J + j) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            off[j] = (uint32_t)row_of(row) * (uint32_t)ld + (uint32_t)chunk * 16u;
            if (j < 2) beyond[j] = chunk * 16 < (int)((d - 1) % 128) + 1 ? 0u : 0x80000000u;  // in the last step
        }
    }
    // Load j of the step at byte `soff` of the rows into stage byte `stage`.
    __device__ __forceinline__ void load(int j, uint32_t stage, uint32_t soff, uint32_t last) const {
        load_to_lds(at.descriptor(), to + stage + (uint32_t)j * 1024u, off[j] | (last & beyond[j & 1]), soff);
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
    Span at, next;               // (the next tile's)
    uint64_t base_step;          // X: from step to step
    uint32_t off, next_off, off_step, to, stage_bytes;
    __device__ __forceinline__ void init(const Linear8Args &g, uint32_t lds, uint32_t idle, int wave) {
        base_step = scalar(wave < XL ? (uint64_t)g.x.ld_scales * (SIZE * S::KS) : (uint64_t)0), off_step = scalar(wave == XL ? (uint32_t)(SIZE * S::KS) : 0u);
        to = scalar(wave < XL ? lds + (uint32_t)wave * 256u : wave == XL ? lds + (uint32_t)S::XS_BYTES : idle), stage_bytes = scalar(wave <= XL ? (uint32_t)S::SCALES : 0u);
    }
    // Where the scales of a tile begin, from block `step` on.
    __device__ __forceinline__ void place(const Linear8Args &g, int64_t t0, int64_t o0, int step, bool there, int wave, int lane) {
        uint64_t base = reinterpret_cast<uint64_t>(g.x.scales) + (uint64_t)(step * g.x.ld_scales) * SIZE;
        uint32_t range = 0;
        next_off = 0x80000000u;
        if (wave < XL) {
            const int64_t first = t0 + wave * (256 / SIZE), left = g.n - first;
            base += (uint64_t)first * SIZE, range = left > 0 ? (uint32_t)((min((int64_t)(256 / SIZE), left) * SIZE + 3) & ~(int64_t)3) : 0u;
            next_off = lane * 4;
        } else if (wave == XL) {
            const int64_t blocks = (g.d_out + kBlock8 - 1) / kBlock8 - o0 / kBlock8;
            const uint64_t first = reinterpret_cast<uint64_t>(g.w.scales) + (uint64_t)(o0 / kBlock8 * g.w.ld_scales + step) * SIZE;
            base = first & ~(uint64_t)3, range = 0x7FFFFFFFu;
            if (lane < S::BO / kBlock8 && lane < blocks) next_off = (uint32_t)(first & 3) + (uint32_t)(lane * g.w.ld_scales) * SIZE;
        }
        next = {scalar(base), scalar(there ? range : 0u)};
    }
    __device__ __forceinline__ void turn(bool yes) {
        at.base = yes ? next.base : at.base, at.range = yes ? next.range : at.range, off = yes ? next_off : off;
    }
    __device__ __forceinline__ void load(uint32_t stage) {
        load_dwords_to_lds(at.descriptor(), to + stage * stage_bytes, off & ~3u);
        at.base += base_step, off += off_step;
    }
};

// CUT: the contraction is no multiple of 16.
template <typename S, int F8, int SCALE, typename T, bool CUT>
__global__ void __launch_bounds__(S::THREADS, 2) linear8_tile_kernel(Linear8Args g) {
    constexpr bool EXACT = sizeof(T) == 4, IN_MFMA = SCALE == SCALE_E8M0 && !EXACT;
    constexpr int TJ = S::TJ, TU = S::TU, PD = S::PD, BT = S::BT, BO = S::BO;
    // (its size given at the launch: knowing that one work-group fills a compute unit, the compiler has the matrix instructions write to
    // accumulation registers and copies the results from there, 64 x 128 tiles 22 us instead of 17)
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int tid = threadIdx.x % (64 * S::WAVES), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = S::KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * S::WAVES));
    const int wt = wave / S::NO, wo = wave % S::NO, i16 = lane & 15, g4 = lane >> 4;
    // Work-groups are dealt round-robin to the 8 XCDs, each with an L2 of its own: one XCD gets a run of consecutive positions, and
    // positions go through bands of eight tile rows (tokens), column by column, so that what runs on an XCD shares rows of both.
    // A work-group takes every so many-th position of its XCD's run, and requests the first steps of its next tile under the last ones
    // of this: no tile but the first waits for its operands, and the results are on their way to memory under the next tile's MFMAs.
    const uint32_t tiles_t = (uint32_t)((g.n + BT - 1) / BT), tiles_o = (uint32_t)((g.d_out + BO - 1) / BO), tiles = tiles_t * tiles_o;
    const uint32_t xcd = blockIdx.x % 8, turns = (gridDim.x - xcd + 7) / 8, first = xcd * (tiles / 8) + min(xcd, tiles % 8), count = tiles / 8 + (xcd < tiles % 8);
    auto tile_at = [&](uint32_t position, int64_t &t0, int64_t &o0) {
        const uint32_t tile = first + position, band = tile / (8 * tiles_o), in = tile - band * 8 * tiles_o;
        const uint32_t rows = min(8u, tiles_t - band * 8), col = in / rows;
        t0 = (int64_t)scalar(band * 8 + in - col * rows) * BT, o0 = (int64_t)scalar(col) * BO;
    };
    const int blocks = (int)((g.d_in + kBlock8 - 1) / kBlock8), steps = (blocks + S::KS - 1) / S::KS;  // step s of a group: block s KS + group

    typedef __attribute__((address_space(3))) unsigned char *lds_ptr_t;
    unsigned char *const mine = lds + group * S::GROUP;
    const uint32_t lds0 = scalar((uint32_t)(uintptr_t)(lds_ptr_t)mine);
    Loads8<S::JX> lx;
    Loads8<S::JW> lw;
    ScaleLoads8<S, SCALE> ls;
    lx.init(g.x.ld, g.d_in, lds0, wave, lane, [](int r) { return r / S::WT * S::WT + r % 16 * TJ + r % S::WT / 16; });
    lw.init(g.w.ld, g.d_in, lds0 + S::X_BYTES, wave, lane, [](int r) { return r / 32 * 32 + r % 16 / 4 * 8 + r / 16 % 2 * 4 + r % 4; });
    ls.init(g, lds0 + S::STAGES * S::STAGE, (uint32_t)(uintptr_t)(lds_ptr_t)lds + S::KS * S::GROUP, wave);
    // The tile whose operands are requested after the one that is being requested.
    Span next_x, next_w;
    int64_t next_t0 = 0, next_o0 = 0;
    auto place = [&](uint32_t position) {
        const bool there = position < count;
        tile_at(there ? position : 0u, next_t0, next_o0);
        next_x = rows_of(g.x, next_t0, min((int64_t)BT, g.n - next_t0), there);
        next_w = rows_of(g.w, next_o0, min((int64_t)BO, g.d_out - next_o0), there);
        ls.place(g, next_t0, next_o0, group, there, wave, lane);
        asm volatile("s_nop 4" : "+s"(next_x.base), "+s"(next_x.range), "+s"(next_w.base), "+s"(next_w.range), "+s"(ls.next.base), "+s"(ls.next.range));  // (as settle)
    };
    // The step that is being requested, and the stage it goes to.
    int asked = steps - 1;
    uint32_t soff = 0, last = 0, into = S::STAGES - 1;
    auto begin = [&] {
        const bool turn = asked == steps - 1;
        asked = turn ? 0 : asked + 1, into = into == S::STAGES - 1 ? 0 : into + 1;
        lx.at.base = turn ? next_x.base : lx.at.base, lx.at.range = turn ? next_x.range : lx.at.range;
        lw.at.base = turn ? next_w.base : lw.at.base, lw.at.range = turn ? next_w.range : lw.at.range;
        ls.turn(turn);
        const int block = asked * S::KS + group;
        if (S::KS > 1) {  // the last step of a group may be none: zeros
            const bool none = block >= blocks;
            lx.at.range = scalar(none ? 0u : lx.at.range), lw.at.range = scalar(none ? 0u : lw.at.range), ls.at.range = scalar(none ? 0u : ls.at.range);
        }
        // (a tile that is not there has no bytes, and no offset either: the check takes it from the range, unsigned)
        soff = lx.at.range == 0 ? 0u : (uint32_t)block * 128u, last = block == blocks - 1 ? 0xFFFFFFFFu : 0u;
    };
    auto load = [&](int i) {  // load i of that step: the scales first
        if (i == 0)
            ls.load(into);
        else if (i <= S::JX)
            lx.load(i - 1, into * S::STAGE, soff, last);
        else
            lw.load(i - 1 - S::JX, into * S::STAGE, soff, last);
    };

    // A lane's place in a tile of 16 rows: row i16, chunks g4 and g4 + 4; `from`: the stage that is read.
    const uint32_t at0 = (uint32_t)(i16 * 128 + ((g4 ^ ((i16 >> 1) & 7)) << 4)), at1 = at0 ^ 64u;
    uint32_t from = 0, x0 = at0 + wt * S::WT * 128, x1 = at1 + wt * S::WT * 128, w0 = at0 + S::X_BYTES + wo * S::WO * 128, w1 = at1 + S::X_BYTES + wo * S::WO * 128;
    auto turn_stage = [&] {
        const bool around = from == S::STAGES - 1;
        const uint32_t by = around ? 0u - (uint32_t)((S::STAGES - 1) * S::STAGE) : (uint32_t)S::STAGE;
        from = around ? 0 : from + 1, x0 += by, x1 += by, w0 += by, w1 += by;
    };
    auto fragment = [&](uint32_t a, uint32_t b, int tile) {
        union {
            i32x8_t v;
            uint4 q[2];
        } f;
        f.q[0] = *reinterpret_cast<const uint4 *>(mine + a + tile * 2048);
        f.q[1] = *reinterpret_cast<const uint4 *>(mine + b + tile * 2048);
        return f.v;
    };

    f32x4_t acc[TU][TJ];
    i32x8_t xf[TJ], wf[4];
    // Scales of a step, as read and as used: powers of two as bytes for the matrix instruction, or the products of X's and W's.
    constexpr int XS = SCALE == SCALE_F32 ? TJ : TJ / 4;
    uint32_t xs_read[XS], ws_read, xs[IN_MFMA ? XS : 1], ws = 0;
    float fs[IN_MFMA ? 1 : TJ];
    [[maybe_unused]] float rest[SCALE == SCALE_E8M0 && EXACT ? TJ : 1];  // (a lane's fragments of X are of the tokens whose sums it holds)
    uint32_t w_byte = 0;  // address of the step's scale of W
    auto w_byte_of = [&](int64_t o0) { return (uint32_t)reinterpret_cast<uint64_t>(g.w.scales) + (uint32_t)((o0 + wo * S::WO) / kBlock8 * g.w.ld_scales) + group; };
    auto read_scales = [&] {
        const unsigned char *at = mine + S::STAGES * S::STAGE + from * S::SCALES;
        ws_read = *reinterpret_cast<const uint32_t *>(at + S::XS_BYTES + wo * S::WO / kBlock8 * 4);
#pragma unroll
        for (int q = 0; q < XS; ++q) xs_read[q] = *reinterpret_cast<const uint32_t *>(at + (wt * S::WT + i16 * TJ) * (SCALE == SCALE_F32 ? 4 : 1) + 4 * q);
    };
    auto take_scales = [&] {
        if constexpr (SCALE == SCALE_F32) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) fs[j] = __uint_as_float(xs_read[j]) * __uint_as_float(ws_read);
        } else {
            const uint32_t w = ws_read >> ((w_byte & 3) * 8);
            w_byte += S::KS;
            if constexpr (IN_MFMA) {
                ws = w;
#pragma unroll
                for (int q = 0; q < XS; ++q) xs[q] = xs_read[q];
            } else {
#pragma unroll
                for (int j = 0; j < TJ; ++j) {
                    const PowerProduct p = power_product(xs_read[j / 4] >> (j % 4 * 8) & 255u, w & 255u);
                    fs[j] = p.s, rest[j] = __uint_as_float(p.rest << 23);
                }
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
    constexpr int LATE = 2;  // MFMAs between one and the use of its result
    constexpr int STORES = TJ * TU / 2;  // of a wave, at least, where the tile has all its rows and columns
    constexpr int AHEAD = (S::STAGES - 2) * LOADS;  // behind the loads of the next step
    static_assert((S::STAGES - 1) * LOADS <= 63 && AHEAD + STORES <= 63, "what a wait can count");
    uint32_t position = blockIdx.x / 8;
    place(position);
    int64_t t0 = next_t0, o0 = next_o0;
    begin();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(i);
    place(position + turns);
#pragma unroll
    for (int k = 1; k < S::STAGES; ++k) {
        begin();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(i);
    }
    wait_for_loads<(S::STAGES - 1) * LOADS>();
    __syncthreads();
    read_first();
    read_scales();
    w_byte = w_byte_of(o0);
    take_scales();

    for (bool stored = false;;) {
#pragma unroll
    for (int u = 0; u < TU; ++u)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[u][j] = (f32x4_t){0, 0, 0, 0};

    // Step by step: the first fragments and the scales are in registers.  A fragment of X gives its place to the next step's
    // behind its last use, so that one set is enough.
    for (int left = steps; left > 0; --left) {
        if (CUT && left == 1) {
            // The chunk of 16 that the contraction ends in: what lies behind the end becomes zeros, in LDS.
            const int c = (int)(g.d_in % kBlock8) / 16;
            const bool ends = (steps - 1) * S::KS + group == blocks - 1;  // (the other group's last step is whole, or none)
            for (int row = tid; ends && row < BT + BO; row += 64 * S::WAVES) {
                uint4 *at = reinterpret_cast<uint4 *>(mine + from * S::STAGE + row * 128 + ((c ^ ((row >> 1) & 7)) << 4));
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
                for (int q = 0; q < 4; ++q) xw[j][q] = widened<F8>(xf[j], q, SCALE == SCALE_F32 ? 1.0f : rest[SCALE == SCALE_F32 ? 0 : j]);
        }
        [[maybe_unused]] f32x4_t part[LATE + 1];
        for_each<S::MFMAS + (IN_MFMA ? 0 : LATE)>([&](auto index) __attribute__((always_inline)) {
            constexpr int i = decltype(index)::value, u = i / TJ, j = i % TJ, q = i - (TU - PD) * TJ;
            if constexpr (q == 0) {  // every fragment of W of this stage is in registers, the next step's data are there
                if (stored && left > steps - (S::STAGES - 1))
                    wait_for_loads<AHEAD + STORES>();  // (behind those loads the results of the tile before went out)
                else
                    wait_for_loads<AHEAD>();
                __syncthreads();
                begin();
                turn_stage();
            }
            if constexpr (i < S::MFMAS) {
                if constexpr (IN_MFMA) {
                    add_scaled_products<F8, j % 4>(wf[u % 4], xf[j], acc[u][j], ws, xs[j / 4]);
                } else if constexpr (EXACT) {
                    if constexpr (j == 0)
#pragma unroll
                        for (int k = 0; k < 4; ++k) ww[k] = widened<F8_E4M3>(wf[u % 4], k);
                    part[i % (LATE + 1)] = block_products(ww, xw[j]);
                } else {
                    part[i % (LATE + 1)] = block_products<F8>(wf[u % 4], xf[j]);
                }
                if constexpr (!IN_MFMA) pin(part[i % (LATE + 1)]);
                // fragments of W ahead, the scales, and in the last row of tiles X's fragments of the next step
                if constexpr (j == 0) wf[(u + PD) % 4] = fragment(w0, w1, (u + PD) % TU);
                if constexpr (q == 1) read_scales();
                if constexpr (u == TU - 1) xf[j] = fragment(x0, x1, j);
                for_each<LOADS>([&](auto l) __attribute__((always_inline)) {
                    if constexpr (decltype(l)::value * TAIL / LOADS == q) load(decltype(l)::value);
                });
            }
            if constexpr (!IN_MFMA && i >= LATE) {
                constexpr int k = i - LATE;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[k / TJ][k % TJ][r] = fmaf(part[k % (LATE + 1)][r], fs[k % TJ], acc[k / TJ][k % TJ][r]);
                pin(acc[k / TJ][k % TJ]);
            }
            if constexpr (i < S::MFMAS) __builtin_amdgcn_sched_barrier(0);
        });
        if (left == 1) w_byte = w_byte_of(next_o0);
        take_scales();
    }
    if constexpr (IN_MFMA) settle_sums(acc);
    if constexpr (S::KS == 2) {
        // Half of the outputs is the first group's, half the second's: each hands over what it has of the other's.
        wait_for_loads<0>();  // (into LDS, of the steps behind the last: zeros)
        __syncthreads();
        f32x4_t *const over = reinterpret_cast<f32x4_t *>(lds) + wave * (TU * TJ * 64) + lane;
        auto exchange = [&](auto mine_first) __attribute__((always_inline)) {
            constexpr int keep = decltype(mine_first)::value, give = TU / 2 - keep;
#pragma unroll
            for (int u = 0; u < TU / 2; ++u)
#pragma unroll
                for (int j = 0; j < TJ; ++j) over[((give + u) * TJ + j) * 64] = acc[give + u][j];
            __syncthreads();
#pragma unroll
            for (int u = 0; u < TU / 2; ++u)
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[keep + u][j] += over[((keep + u) * TJ + j) * 64];
        };
        if (group == 0)
            exchange(std::integral_constant<int, 0>());
        else
            exchange(std::integral_constant<int, TU / 2>());
    }

    // Tiles 2 v and 2 v + 1 hold outputs 32 v + 8 g4 .. + 7 of the lane's tokens.
    const bool whole = t0 + BT <= g.n && o0 + BO <= g.d_out;
    const int64_t token0 = t0 + wt * S::WT + i16 * TJ, out0 = o0 + wo * S::WO + 8 * g4;
    // (token by token, so that its lines fill up at once: 16384 x 1024 -> 4096, 8 waves, 82 us with the tokens inside, 77 like this)
    auto store = [&](int j, int v, bool checked) __attribute__((always_inline)) {
        const int64_t o = out0 + 32 * v, valid = g.d_out - o;
        float y[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = acc[2 * v][j][r], y[4 + r] = acc[2 * v + 1][j][r];
        if (checked && g.bias != nullptr) {  // (adding +0 would turn a -0 into +0: only where a bias exists)
            float b[8];
            load8<T>((const T *)g.bias + (valid > 0 ? o : 0), valid, b);
#pragma unroll
            for (int r = 0; r < 8; ++r) y[r] += b[r];
        }
        if (!checked)
            store8<T>((T *)g.Y + (token0 + j) * g.d_out + o, 8, y);
        else if (token0 + j < g.n)
            store8<T>((T *)g.Y + (token0 + j) * g.d_out + (valid > 0 ? o : 0), valid, y);
    };
    const bool checked = !whole || g.bias != nullptr;
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int v = 0; v < TU / 2; ++v) {
            if (S::KS == 2 && v / (TU / 4) != group) continue;
            if (checked)
                store(j, v, true);
            else
                store(j, v, false);
        }
    position += turns;
    if (position >= count) break;
    stored = whole;
    t0 = next_t0, o0 = next_o0;
    place(position + turns);
    }
    wait_for_loads<0>();  // (of no tile: zeros, but into LDS that is another work-group's from here on)
}

typedef Tile8<256, 256, 4, 2, 1, 2> Large8;   // 8 waves of 64 x 128
typedef Tile8<128, 128, 2, 2, 1, 2> Mid8;     // 4 waves of 64 x 64, two work-groups to a compute unit
typedef Tile8<128, 128, 2, 2, 2, 2> Split8;   // twice such waves, where there are no more tiles than compute units
typedef Tile8<64, 128, 1, 2, 2, 3> Half8;     // twice 2 waves of 64 x 64

template <typename S, int F8, int SCALE, typename T>
void launch_tile(const Linear8Args &g, hipStream_t stream) {
    const int64_t tiles = (g.n + S::BT - 1) / S::BT * ((g.d_out + S::BO - 1) / S::BO), places = 256 * (160 * 1024 / S::LDS_BYTES);
    const int64_t steps = (g.d_in + kBlock8 - 1) / kBlock8;
    const unsigned grid = (unsigned)(S::KS == 1 && steps >= 2 && tiles > places ? places : tiles);  // (requests reach into one further tile, no more)
    if (g.d_in % 16 != 0)
        linear8_tile_kernel<S, F8, SCALE, T, true><<<grid, S::THREADS, S::LDS_BYTES, stream>>>(g);
    else
        linear8_tile_kernel<S, F8, SCALE, T, false><<<grid, S::THREADS, S::LDS_BYTES, stream>>>(g);
}

}  // namespace

}  // namespace rmm
