// Root-mean-square norm of rows, with the addition of a residual in front and 8-bit rows behind, and its backward pass.
//
//   forward    h = x + r (rounded);  rstd = 1 / sqrt(mean h^2 + eps);  y = h rstd w
//   backward   g = dy w, hhat = h rstd:  dx = rstd (g - hhat mean(g hhat)) + dh;   dw = sum over rows of dy hhat
//
// Memory bounds both, so every row is read once and stays in registers until it is written: a lane holds CH runs of
// eight columns, WPR waves hold a row (8 CH 64 WPR columns), 16 lanes hold a block of 128 columns, whose largest magnitude
// is then four lane exchanges away.  Work-groups go through the rows in strides, so that the weights are read once a
// work-group and dw is summed in registers; its partial sums, one row of d numbers a work-group, are added by a second
// kernel in a fixed order.  Rows too long for the registers of 16 waves are read twice, and their dw has a kernel of its own.
#include "quant8.hpp"

namespace rmm {

namespace {

constexpr int kRun = 8;  // columns of a lane's run

// Sum over the WPR waves of a row, the same in all of them (red: two rows of WPR numbers, taken in turns so that one
// barrier a row is enough).
template <int WPR, typename F>
__device__ __forceinline__ F row_sum(F v, F *red, int turn) {
    v = sum_of_64(v);
    if constexpr (WPR > 1) {
        F *to = red + (turn & 1) * WPR;
        if ((threadIdx.x & 63) == 0) to[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < WPR; ++i) v += to[i];
    }
    return v;
}

// Which rows and columns a thread takes.
template <int WPR>
struct Place {
    static constexpr int ROWS = WPR == 1 ? 4 : 1, THREADS = WPR == 16 ? 1024 : 256;
    int lane, wave, part, row;  // wave of the row, row of the work-group's
    __device__ __forceinline__ Place()
        : lane(threadIdx.x & 63), wave(threadIdx.x >> 6), part(WPR == 1 ? 0 : wave), row(WPR == 1 ? wave : 0) {}
    __device__ __forceinline__ int64_t col(int c) const { return ((int64_t)(c * WPR + part) * 64 + lane) * kRun; }
};

struct NormArgs {
    const void *X, *residual, *weight;
    void *H, *Y;
    Mat8 y8;
    int f8, scale;
    float *rstd;
    int64_t n, d;
    float eps;
    double inv_d;
};

// 1 / sqrt(mean + eps), from fp32 by a step of Newton's: `high` is its fp32 number, `low` what is missing.
struct Rstd {
    float high, low;
};
__device__ __forceinline__ Rstd rstd_of(double sum, const NormArgs &g) {
    const double m = sum * g.inv_d + (double)g.eps;
    const double r = (double)(1.0f / sqrtf((float)m)), s = r * (1.5 - 0.5 * m * r * r);
    // (where m is zero, infinite, no number or too far out for fp32, its own root says what fp32 makes of it; `low` where it has one)
    if (!(m >= 0x1p-120 && m < 0x1p120)) {
        const double x = 1.0 / sqrt(m);
        return {(float)x, x >= 0x1p-124 && x < 0x1p127 ? (float)(x - (double)(float)x) : 0.0f};
    }
    const float high = (float)s;
    return {high, (float)(s - (double)high)};
}

// Eight columns of y = h rstd w to 8 bits.  An 8-bit number is decided by where y / s lies between two of the format's, and
// is as far off as they are apart where y is off by little and crosses over: y is made to twice the bits of fp32 here, as y + low, and
// so is the largest magnitude, whose quotient is then rounded once.  A power of two takes y alone, as its quotients are exact; which power
// it is hangs on `low` where the largest magnitude lies one step of fp32 above top 2^k (top = 1.75 2^j): rounded to fp32 once, its quotient
// is 2^k up to 0.875 of that step.
struct Twice {
    float y, low;
};
__device__ __forceinline__ Twice twice(float h, const Rstd &r, float w) {
#pragma clang fp contract(off)  // (what a rounding left out would be counted twice where a sum takes the product whole)
    const float p = h * r.high, p_low = fmaf(h, r.low, fmaf(h, r.high, -p));
    const float v = p * w, v_low = fmaf(p_low, w, fmaf(p, w, -v)), y = v + v_low;
    return {y, v_low - (y - v)};
}
template <typename T, int F8, int SCALE>
__device__ __forceinline__ void put8(const NormArgs &g, int64_t row, int64_t col, int lane, const float (&h)[8], const Rstd &r, const float (&w)[8]) {
    float y[8], low[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const Twice t = twice(h[i], r, w[i]);
        y[i] = t.y, low[i] = t.low;
    }
    const uint32_t most = max_of_16(amax8(y));
    const float amax = __uint_as_float(most);
    float q = amax / top_of<F8>();
    if (SCALE == SCALE_F32 || (most & 0x7FFFFFu) == 0x600001u) {  // (the same in the 16 lanes)
        float more = -INFINITY;  // of those as large in fp32, what is missing of the largest
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            Twice t = {y[i], low[i]};
            // Made again for fp32 rows, whose registers are full: with powers of two 2048 x 16384 94 us, kept until here 99.  With the registers that
            // this frees bf16 rows get a fifth wave a SIMD and are slower: 16384 x 4096 95, kept 92.
            if constexpr (SCALE == SCALE_E8M0 && sizeof(T) == 4) {
                float again = h[i];
                asm("" : "+v"(again));
                t = twice(again, r, w[i]);
            }
            more = magnitude(t.y) == most ? fmaxf(more, t.y < 0.0f ? -t.low : t.low) : more;
        }
        q = fmaf(fmaf(-q, top_of<F8>(), amax) + max_of_16(more), 1.0f / top_of<F8>(), q);
    }
    const BlockScale s = block_scale<F8, SCALE>(q);
    if (col < g.d) {
        store8_bytes(g.y8.data + row * g.y8.ld + col, g.d - col, to_f8<F8, SCALE>(y, low, s));
        if ((lane & 15) == 0) store_scale<SCALE>(g.y8.scales, col / kBlock8 * g.y8.ld_scales + row, s);
    }
}
template <typename T>
__device__ __forceinline__ void put8(const NormArgs &g, int64_t row, int64_t col, int lane, const float (&h)[8], const Rstd &r, const float (&w)[8]) {
    if (g.f8 == F8_E4M3) {
        if (g.scale == SCALE_F32)
            put8<T, F8_E4M3, SCALE_F32>(g, row, col, lane, h, r, w);
        else
            put8<T, F8_E4M3, SCALE_E8M0>(g, row, col, lane, h, r, w);
    } else {
        if (g.scale == SCALE_F32)
            put8<T, F8_E5M2, SCALE_F32>(g, row, col, lane, h, r, w);
        else
            put8<T, F8_E5M2, SCALE_E8M0>(g, row, col, lane, h, r, w);
    }
}

// h of eight columns, written to H if there is a residual.
template <typename T, int MODE>
__device__ __forceinline__ void make_h(const NormArgs &g, int64_t row, int64_t col, const Run8<T> &x, const Run8<T> &r, float (&h)[8]) {
    values<T, MODE>(x, col, g.d, h);
    if (g.residual != nullptr) {
        float f[8];
        values<T, MODE>(r, col, g.d, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = rounded<T>(h[i] + f[i]);
        if (g.H != nullptr) store_run<T, MODE>((T *)g.H + row * g.d, col, g.d, h);
    }
}

template <typename T, int CH, int WPR, int MODE>
__global__ void __launch_bounds__(Place<WPR>::THREADS) rms_norm_kernel(NormArgs g) {
    __shared__ double red[2 * WPR];
    const Place<WPR> p;
    Run8<T> w[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = load_run<T, MODE>((const T *)g.weight, p.col(c), g.d);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * p.ROWS + p.row; row < g.n; row += (int64_t)gridDim.x * p.ROWS, ++turn) {
        Run8<T> x[CH], r[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) x[c] = load_run<T, MODE>((const T *)g.X + row * g.d, p.col(c), g.d);
        if (g.residual != nullptr)
#pragma unroll
            for (int c = 0; c < CH; ++c) r[c] = load_run<T, MODE>((const T *)g.residual + row * g.d, p.col(c), g.d);
        float h[CH][8];
        double sum = 0.0;  // (memory bounds the kernel all the same; in fp32 y would not have the bits that put8 makes it to)
#pragma unroll
        for (int c = 0; c < CH; ++c) make_h<T, MODE>(g, row, p.col(c), x[c], r[c], h[c]);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma((double)h[c][i], (double)h[c][i], sum);
        const Rstd rstd = rstd_of(row_sum<WPR>(sum, red, turn), g);
        if (g.rstd != nullptr && p.part == 0 && p.lane == 0) g.rstd[row] = rstd.high;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = p.col(c);
            float f[8];
            values<T, MODE>(w[c], col, g.d, f);
            if (g.y8.data != nullptr) put8<T>(g, row, col, p.lane, h[c], rstd, f);
            if (g.Y != nullptr) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * rstd.high * f[i];
                store_run<T, MODE>((T *)g.Y + row * g.d, col, g.d, h[c]);
            }
        }
    }
}

// Rows of any length, read twice (the second time mostly from L2).
template <typename T>
__device__ __forceinline__ void take_h(const NormArgs &g, int64_t row, int64_t col, float (&h)[8]) {
    const Run8<T> x = load_run<T, ROWS_RAGGED>((const T *)g.X + row * g.d, col, g.d);
    Run8<T> r;
    if (g.residual != nullptr) r = load_run<T, ROWS_RAGGED>((const T *)g.residual + row * g.d, col, g.d);
    make_h<T, ROWS_RAGGED>(g, row, col, x, r, h);
}
template <typename T>
__global__ void __launch_bounds__(1024) rms_norm_long_kernel(NormArgs g) {
    __shared__ double red[2 * 16];
    const Place<16> p;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < g.n; row += gridDim.x, ++turn) {
        float h[8];
        double sum = 0.0;
        for (int c = 0; p.col(c) < g.d; ++c) {
            take_h<T>(g, row, p.col(c), h);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma((double)h[i], (double)h[i], sum);
        }
        const Rstd rstd = rstd_of(row_sum<16>(sum, red, turn), g);
        if (g.rstd != nullptr && threadIdx.x == 0) g.rstd[row] = rstd.high;
        NormArgs again = g;  // (what was written is read back, by the thread that wrote it; the buffer may be that of X)
        if (g.residual != nullptr && g.H != nullptr) again.X = g.H, again.residual = nullptr;
        again.H = nullptr;
        for (int c = 0; p.col(c) - p.lane * kRun < g.d; ++c) {  // (whole waves: 16 lanes share a block)
            const int64_t col = p.col(c);
            float w[8];
            take_h<T>(again, row, col, h);
            values<T, ROWS_RAGGED>(load_run<T, ROWS_RAGGED>((const T *)g.weight, col, g.d), col, g.d, w);
            if (g.y8.data != nullptr) put8<T>(g, row, col, p.lane, h, rstd, w);
            if (g.Y != nullptr) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] = h[i] * rstd.high * w[i];
                store_run<T, ROWS_RAGGED>((T *)g.Y + row * g.d, col, g.d, h);
            }
        }
    }
}

struct NormBackwardArgs {
    const void *dY, *dH, *H, *weight;
    const float *rstd;
    void *dX;
    float *part;  // a row of d numbers for each work-group; null: no dweight
    int64_t n, d;
};

// What is read of a row; that of the next row is requested before this one is reduced (not with two runs a lane in 16 waves, 128
// registers each: there are enough requests between them).  4096 x 8192 bf16, 512 work-groups: one run a lane 57 us, two, half of the lanes
// idle, 73.
template <typename T, int CH>
struct BackwardRow {
    Run8<T> dy[CH], h[CH], dh[CH];
    float rstd;
};
template <typename T, int CH, int WPR, int MODE>
__device__ __forceinline__ void load_row(BackwardRow<T, CH> &q, const NormBackwardArgs &g, const Place<WPR> &p, int64_t row) {
    q.rstd = g.rstd[row];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        q.dy[c] = load_run<T, MODE>((const T *)g.dY + row * g.d, p.col(c), g.d);
        q.h[c] = load_run<T, MODE>((const T *)g.H + row * g.d, p.col(c), g.d);
    }
    if (g.dH != nullptr)
#pragma unroll
        for (int c = 0; c < CH; ++c) q.dh[c] = load_run<T, MODE>((const T *)g.dH + row * g.d, p.col(c), g.d);
}

template <typename T, int CH, int WPR, int MODE>
__global__ void __launch_bounds__(Place<WPR>::THREADS) rms_norm_backward_kernel(NormBackwardArgs g) {
    constexpr int PARKED = WPR == 1 ? 3 * CH * 64 * kRun : 1;  // dw of the waves that hold rows of their own
    __shared__ float red[2 * WPR];
    __shared__ float parked[PARKED];
    const Place<WPR> p;
    const float inv_d = 1.0f / (float)g.d;
    Run8<T> weight[CH];
    float dw[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        weight[c] = load_run<T, MODE>((const T *)g.weight, p.col(c), g.d);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.0f;
    }
    const int64_t step = (int64_t)gridDim.x * p.ROWS;
    int64_t row = (int64_t)blockIdx.x * p.ROWS + p.row;
    constexpr bool AHEAD = WPR < 16 || CH == 1;
    BackwardRow<T, CH> now, next;
    if (AHEAD && row < g.n) load_row<T, CH, WPR, MODE>(now, g, p, row);
    for (int turn = 0; row < g.n; row += step, ++turn) {
        if constexpr (!AHEAD)
            load_row<T, CH, WPR, MODE>(now, g, p, row);
        else if (row + step < g.n)
            load_row<T, CH, WPR, MODE>(next, g, p, row + step);
        float dy[CH][8], h[CH][8], sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float w[8];
            values<T, MODE>(now.dy[c], p.col(c), g.d, dy[c]), values<T, MODE>(now.h[c], p.col(c), g.d, h[c]), values<T, MODE>(weight[c], p.col(c), g.d, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[c][i] *= now.rstd;
                dw[c][i] = fmaf(dy[c][i], h[c][i], dw[c][i]);
                dy[c][i] *= w[i];
                sum = fmaf(dy[c][i], h[c][i], sum);
            }
        }
        if (g.dX != nullptr) {  // (the same for all)
            const float mean = row_sum<WPR>(sum, red, turn) * inv_d;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t col = p.col(c);
                float more[8];
                if (g.dH != nullptr) values<T, MODE>(now.dh[c], col, g.d, more);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = now.rstd * fmaf(-h[c][i], mean, dy[c][i]);
                    dy[c][i] = g.dH != nullptr ? v + more[i] : v;
                }
                store_run<T, MODE>((T *)g.dX + row * g.d, col, g.d, dy[c]);
            }
        }
        if constexpr (AHEAD) now = next;
    }
    if (g.part == nullptr) return;
    if constexpr (WPR == 1) {  // the four waves' sums, in the order of the waves
        if (p.wave > 0)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) parked[(((p.wave - 1) * CH + c) * 8 + i) * 64 + p.lane] = dw[c][i];
        __syncthreads();
        if (p.wave > 0) return;
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) dw[c][i] += parked[((q * CH + c) * 8 + i) * 64 + p.lane];
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = p.col(c);
        store8<float>(g.part + (int64_t)blockIdx.x * g.d + (col < g.d ? col : 0), g.d - col, dw[c]);
    }
}

// dX of rows of any length.
template <typename T>
__global__ void __launch_bounds__(1024) rms_norm_backward_long_kernel(NormBackwardArgs g) {
    __shared__ float red[2 * 16];
    const Place<16> p;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < g.n; row += gridDim.x, ++turn) {
        const float rstd = g.rstd[row];
        float dy[8], h[8], w[8], sum = 0.0f;
        auto take = [&](const void *from, int64_t col, float (&v)[8]) { values<T, ROWS_RAGGED>(load_run<T, ROWS_RAGGED>((const T *)from, col, g.d), col, g.d, v); };
        auto take_both = [&](int64_t col) {
            take((const T *)g.dY + row * g.d, col, dy), take((const T *)g.H + row * g.d, col, h), take(g.weight, col, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] *= rstd, dy[i] *= w[i];
        };
        for (int c = 0; p.col(c) < g.d; ++c) {
            take_both(p.col(c));
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(dy[i], h[i], sum);
        }
        const float mean = row_sum<16>(sum, red, turn) / (float)g.d;
        for (int c = 0; p.col(c) < g.d; ++c) {
            const int64_t col = p.col(c);
            float more[8];
            take_both(col);
            if (g.dH != nullptr) take((const T *)g.dH + row * g.d, col, more);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = rstd * fmaf(-h[i], mean, dy[i]);
                dy[i] = g.dH != nullptr ? v + more[i] : v;
            }
            store_run<T, ROWS_RAGGED>((T *)g.dX + row * g.d, col, g.d, dy);
        }
    }
}

// Partial sums of dw where the rows are too long: work-group (x, y) takes 512 columns of every gridDim.y-th row.
// Runs before dX is written (it may be the buffer of dY).
template <typename T>
__global__ void __launch_bounds__(64) rms_norm_dweight_kernel(NormBackwardArgs g) {
    for (int64_t c0 = (int64_t)blockIdx.x * 512; c0 < g.d; c0 += (int64_t)gridDim.x * 512) {
        const int64_t col = c0 + threadIdx.x * kRun;
        float dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int64_t row = blockIdx.y; row < g.n; row += gridDim.y) {
            const float rstd = g.rstd[row];
            float dy[8], h[8];
            values<T, ROWS_RAGGED>(load_run<T, ROWS_RAGGED>((const T *)g.dY + row * g.d, col, g.d), col, g.d, dy);
            values<T, ROWS_RAGGED>(load_run<T, ROWS_RAGGED>((const T *)g.H + row * g.d, col, g.d), col, g.d, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[i] = fmaf(dy[i], h[i] * rstd, dw[i]);
        }
        store8<float>(g.part + (int64_t)blockIdx.y * g.d + (col < g.d ? col : 0), g.d - col, dw);
    }
}

// dweight[j] = sum of part[p][j], p = 0 .. parts - 1: 16 columns a work-group, 64 threads a column.
template <typename T>
__global__ void __launch_bounds__(1024) sum_parts_kernel(const float *__restrict__ part, int parts, int64_t d, T *__restrict__ out) {
    __shared__ float sums[64][17];
    const int c = threadIdx.x & 15, s = threadIdx.x >> 4;
    for (int64_t c0 = (int64_t)blockIdx.x * 16; c0 < d; c0 += (int64_t)gridDim.x * 16) {
        float v = 0.0f;
        if (c0 + c < d)
#pragma unroll 8
            for (int p = s; p < parts; p += 64) v += part[(int64_t)p * d + c0 + c];
        __syncthreads();
        sums[s][c] = v;
        __syncthreads();
        if (threadIdx.x < 64) {  // four threads a column, then their four sums
            const int cc = threadIdx.x & 15, q = threadIdx.x >> 4;
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) t += sums[q * 16 + i][cc];
            t += __shfl_xor(t, 16, 64);
            t += __shfl_xor(t, 32, 64);
            if (q == 0 && c0 + cc < d) store_f32<T>(out + c0 + cc, t);
        }
    }
}

// Columns that CH runs a lane in WPR waves hold.
constexpr int64_t columns(int ch, int wpr) { return (int64_t)ch * wpr * 64 * kRun; }
int64_t rows_a_group(int64_t d) { return d <= columns(2, 1) ? 4 : 1; }
constexpr int64_t kMostForward = 2048;  // work-groups: eight for each compute unit
// Two, or the one of 16 waves that its registers hold (each has a row of partial sums of dw: 4096 x 8192 bf16 45.8 us, with two 56.1; with one of
// four waves 16384 x 4096 113.8, with two 101.1, with three 107.6).
int64_t most_backward(int64_t d) { return d <= columns(2, 4) ? 512 : 256; }
// (four runs a lane in 16 waves are more than their registers hold: with 8-bit rows, 1000 x 32768 bf16 85 us, read twice 62; 2048 x 16384
// with four runs 134, with two 58)
bool long_rows(int64_t d) { return d > columns(2, 16); }
int64_t backward_groups(int64_t n, int64_t d) {
    if (long_rows(d)) return n < 64 ? n : 64;
    const int64_t groups = (n + rows_a_group(d) - 1) / rows_a_group(d);
    return groups < most_backward(d) ? groups : most_backward(d);
}

}  // namespace

// (rows of fewer than eight columns are a kind of their own, of the smallest kernel alone)
#define LAUNCH(KERNEL, CH, WPR, THREADS) \
    (d % 8 == 0 ? KERNEL<T, CH, WPR, ROWS_EVEN><<<grid, THREADS, 0, stream>>>(g) : KERNEL<T, CH, WPR, ROWS_RAGGED><<<grid, THREADS, 0, stream>>>(g))

size_t norm_backward_partials(int64_t n, int64_t d) { return (size_t)backward_groups(n, d) * (size_t)d; }

template <typename T>
hipError_t launch_rms_norm(const T *X, const T *residual, const T *weight, T *H, T *Y, const Mat8 *Y8, int f8, int scale, float *rstd,
                           int64_t n, int64_t d, float eps, hipStream_t stream) {
    const NormArgs g = {X, residual, weight, H, Y, Y8 != nullptr ? *Y8 : Mat8{nullptr, 0, nullptr, 0}, f8, scale, rstd, n, d, eps, 1.0 / (double)d};
    const int64_t groups = (n + rows_a_group(d) - 1) / rows_a_group(d);
    const unsigned grid = (unsigned)(groups < kMostForward ? groups : kMostForward);
    if (d < 8)
        rms_norm_kernel<T, 1, 1, ROWS_TINY><<<grid, 256, 0, stream>>>(g);
    else if (d <= columns(1, 1))
        LAUNCH(rms_norm_kernel, 1, 1, 256);
    else if (d <= columns(2, 1))
        LAUNCH(rms_norm_kernel, 2, 1, 256);
    else if (d <= columns(1, 4))
        LAUNCH(rms_norm_kernel, 1, 4, 256);
    else if (d <= columns(2, 4))
        LAUNCH(rms_norm_kernel, 2, 4, 256);
    else if (d <= columns(4, 4))
        LAUNCH(rms_norm_kernel, 4, 4, 256);
    else if (!long_rows(d))
        LAUNCH(rms_norm_kernel, 2, 16, 1024);
    else
        rms_norm_long_kernel<T><<<grid, 1024, 0, stream>>>(g);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_rms_norm_backward(const T *dY, const T *dH, const T *H, const T *weight, const float *rstd, T *dX, T *dweight,
                                    float *part, int64_t n, int64_t d, hipStream_t stream) {
    const NormBackwardArgs g = {dY, dH, H, weight, rstd, dX, dweight != nullptr ? part : nullptr, n, d};
    const unsigned grid = (unsigned)backward_groups(n, d);
    if (long_rows(d)) {
        const int64_t wide = (d + 511) / 512;
        if (dweight != nullptr)
            rms_norm_dweight_kernel<T><<<dim3((unsigned)(wide < (1 << 20) ? wide : (1 << 20)), grid), 64, 0, stream>>>(g);
        if (dX != nullptr) rms_norm_backward_long_kernel<T><<<(unsigned)(n < kMostForward ? n : kMostForward), 1024, 0, stream>>>(g);
    } else if (d < 8) {
        rms_norm_backward_kernel<T, 1, 1, ROWS_TINY><<<grid, 256, 0, stream>>>(g);
    } else if (d <= columns(1, 1)) {
        LAUNCH(rms_norm_backward_kernel, 1, 1, 256);
    } else if (d <= columns(2, 1)) {
        LAUNCH(rms_norm_backward_kernel, 2, 1, 256);
    } else if (d <= columns(1, 4)) {
        LAUNCH(rms_norm_backward_kernel, 1, 4, 256);
    } else if (d <= columns(2, 4)) {
        LAUNCH(rms_norm_backward_kernel, 2, 4, 256);
    } else if (d <= columns(1, 16)) {
        LAUNCH(rms_norm_backward_kernel, 1, 16, 1024);
    } else {
        LAUNCH(rms_norm_backward_kernel, 2, 16, 1024);
    }
    if (dweight != nullptr) {
        const int64_t wide = (d + 15) / 16;
        sum_parts_kernel<T><<<(unsigned)(wide < (1 << 20) ? wide : (1 << 20)), 1024, 0, stream>>>(part, (int)grid, d, dweight);
    }
    return hipGetLastError();
}

#undef LAUNCH

#define INSTANCES(T)                                                                                                                 \
    template hipError_t launch_rms_norm<T>(const T *, const T *, const T *, T *, T *, const Mat8 *, int, int, float *, int64_t, int64_t, \
                                           float, hipStream_t);                                                                      \
    template hipError_t launch_rms_norm_backward<T>(const T *, const T *, const T *, const T *, const float *, T *, T *, float *, int64_t, \
                                                    int64_t, hipStream_t);
INSTANCES(bf16_t)
INSTANCES(float)
#undef INSTANCES

}  // namespace rmm
