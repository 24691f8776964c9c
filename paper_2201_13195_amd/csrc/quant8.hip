// bf16 / fp32 matrices to 8-bit rows (a scale for each 128 columns of a row) and to 8-bit weights (a scale for each
// 128 x 128 block, and the transposed matrix from the same read).  Both read every element once and keep it in registers
// between the maximum and the conversion; memory bounds them.
#include "quant8.hpp"

namespace rmm {

namespace {

constexpr int kRowsPerGroup = 16;  // rows of a work-group: 16 lanes each
// Blocks of 128 columns, one after the other, all loaded first.  16384 x 4096 bf16, buffers in turn: one 43.4 us, two 41.1, four 41.8, eight 43.5;
// fp32 68.4, 67.7, 71.8, 83.0.
constexpr int kBlocksPerGroup = 2;

// Work-group (x, y): rows 16 x .., blocks kBlocksPerGroup y ..  The 16 lanes of a row read 256 (bf16) or 512 consecutive bytes.
template <typename T, int F8, int SCALE, int MODE>
__global__ void __launch_bounds__(256) quantize_rows8_kernel(const T *__restrict__ A, int64_t n, int64_t d, Mat8 out) {
    const int lane16 = threadIdx.x & 15;
    const int64_t row = (int64_t)blockIdx.x * kRowsPerGroup + (threadIdx.x >> 4);
    if (row >= n) return;  // (16 lanes leave together: those of a row share its maximum)
    const int64_t blocks = (d + kBlock8 - 1) / kBlock8;
    for (int64_t b0 = (int64_t)blockIdx.y * kBlocksPerGroup; b0 < blocks; b0 += (int64_t)gridDim.y * kBlocksPerGroup) {
        Run8<T> run[kBlocksPerGroup];
#pragma unroll
        for (int i = 0; i < kBlocksPerGroup; ++i) {
            const int64_t col = (b0 + i) * kBlock8 + lane16 * 8;
            run[i] = load_run<T, MODE>(A + row * d, col, d);
        }
#pragma unroll
        for (int i = 0; i < kBlocksPerGroup; ++i) {
            if (b0 + i >= blocks) break;
            const int64_t col = (b0 + i) * kBlock8 + lane16 * 8;
            float v[8];
            values<T, MODE>(run[i], col, d, v);
            const BlockScale s = block_scale<F8, SCALE>(max_of_16(amax8(v)));
            const uint2 q = to_f8<F8, SCALE>(v, s);
            if constexpr (MODE == ROWS_EVEN) {
                if (col < d) *reinterpret_cast<uint2 *>(out.data + row * out.ld + col) = q;
            } else {
                store8_bytes(out.data + row * out.ld + col, d - col, q);
            }
            if (lane16 == 0) store_scale<SCALE>(out.scales, (b0 + i) * out.ld_scales + row, s);
        }
    }
}

// 4 x 4 bytes: b[j] = byte j of a[0], a[1], a[2], a[3].
__device__ __forceinline__ void transpose_4x4(uint32_t (&a)[4]) {
    const uint32_t lo01 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
    const uint32_t lo23 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
    a[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u), a[1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
    a[2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u), a[3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
}

// A work-group for each 128 x 128 block: a thread holds 4 x 8 elements (rows 4 g .., columns 8 l ..).  The transposed bytes go through
// LDS, four rows of a column at a time, and leave it as whole lines.  (8 x 8 elements a thread, written from registers in pieces of 8
// bytes: 4096 x 1024 9.1 us, 768 x 768 7.9; like this 7.6 and 6.0.  A kernel of one row is 5 by the same clock.)
template <typename T, int F8, int SCALE, int MODE>
__global__ void __launch_bounds__(512) quantize_weight8_kernel(const T *__restrict__ W, int64_t rows, int64_t cols, Mat8 out, Mat8 out_t) {
    __shared__ uint32_t most[8];
    // Column c: 32 dwords, dword g of four rows at position (g + 4 (c / 8)) % 32, so that neither side meets in the banks.
    __shared__ __attribute__((aligned(16))) uint32_t turned[128][32];
    const int64_t blocks_c = (cols + kBlock8 - 1) / kBlock8, blocks = (rows + kBlock8 - 1) / kBlock8 * blocks_c;
    const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const int64_t br = block / blocks_c, bc = block - br * blocks_c;
        const int64_t row0 = br * kBlock8 + g * 4, col0 = bc * kBlock8 + l * 8;
        Run8<T> run[4];
        float v[8];
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            run[r] = load_run<T, MODE>(W + min(row0 + r, rows - 1) * cols, col0, cols);
        }
        auto take = [&](int r) { values<T, MODE>(run[r], row0 + r < rows ? col0 : cols + 8, cols, v); };  // (rows that do not exist: zeros)
#pragma unroll
        for (int r = 0; r < 4; ++r) take(r), m = max(m, amax8(v));
        m = max_of_16(m);
        const uint32_t m01 = max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16));
        const uint32_t m23 = max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48));
        __syncthreads();  // (of the block before: its scale and its transposed bytes have been read)
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = max(m01, m23);
        __syncthreads();
        m = most[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) m = max(m, most[i]);
        const BlockScale s = block_scale<F8, SCALE>(m);
        uint32_t q[2][4];  // [columns 0-3, 4-7][row]
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            take(r);
            const uint2 p = to_f8<F8, SCALE>(v, s);
            q[0][r] = p.x, q[1][r] = p.y;
            if (row0 + r < rows && col0 < cols) store8_bytes(out.data + (row0 + r) * out.ld + col0, cols - col0, p);
        }
        if (threadIdx.x == 0) store_scale<SCALE>(out.scales, br * out.ld_scales + bc, s);
        if (out_t.data == nullptr) continue;
        if (threadIdx.x == 0) store_scale<SCALE>(out_t.scales, bc * out_t.ld_scales + br, s);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            transpose_4x4(q[h]);
#pragma unroll
            for (int c = 0; c < 4; ++c) turned[8 * l + 4 * h + c][(g + 4 * l) & 31] = q[h][c];
        }
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
            const int c = (threadIdx.x >> 3) + 64 * pass, chunk = threadIdx.x & 7;  // 16 rows
            const uint4 bytes = *reinterpret_cast<const uint4 *>(&turned[c][(4 * chunk + 4 * (c >> 3)) & 31]);
            const int64_t col = bc * kBlock8 + c, row = br * kBlock8 + 16 * chunk;
            if (col >= cols) continue;
            uint8_t *to = out_t.data + col * out_t.ld + row;
            if (row + 16 <= rows) {
                *reinterpret_cast<uint4 *>(to) = bytes;
            } else {
                store8_bytes(to, rows - row, make_uint2(bytes.x, bytes.y));
                store8_bytes(to + 8, rows - row - 8, make_uint2(bytes.z, bytes.w));
            }
        }
    }
}

template <typename T, int F8, int SCALE>
void quantize_rows8(dim3 grid, const T *A, int64_t n, int64_t d, const Mat8 &out, hipStream_t stream) {
    switch (rows_mode(d)) {
        case ROWS_EVEN: quantize_rows8_kernel<T, F8, SCALE, ROWS_EVEN><<<grid, 256, 0, stream>>>(A, n, d, out); break;
        case ROWS_RAGGED: quantize_rows8_kernel<T, F8, SCALE, ROWS_RAGGED><<<grid, 256, 0, stream>>>(A, n, d, out); break;
        default: quantize_rows8_kernel<T, F8, SCALE, ROWS_TINY><<<grid, 256, 0, stream>>>(A, n, d, out);
    }
}
template <typename T, int F8, int SCALE>
void quantize_weight8(unsigned grid, const T *W, int64_t rows, int64_t cols, const Mat8 &out, const Mat8 &out_t, hipStream_t stream) {
    switch (rows_mode(cols)) {
        case ROWS_EVEN: quantize_weight8_kernel<T, F8, SCALE, ROWS_EVEN><<<grid, 512, 0, stream>>>(W, rows, cols, out, out_t); break;
        case ROWS_RAGGED: quantize_weight8_kernel<T, F8, SCALE, ROWS_RAGGED><<<grid, 512, 0, stream>>>(W, rows, cols, out, out_t); break;
        default: quantize_weight8_kernel<T, F8, SCALE, ROWS_TINY><<<grid, 512, 0, stream>>>(W, rows, cols, out, out_t);
    }
}

// The four instances of a function template by format and kind of scale.
#define RMM_BY_FORMAT(CALL)                                                                                             \
    (f8 == F8_E4M3 ? (scale == SCALE_F32 ? CALL(F8_E4M3, SCALE_F32) : CALL(F8_E4M3, SCALE_E8M0))                        \
                   : (scale == SCALE_F32 ? CALL(F8_E5M2, SCALE_F32) : CALL(F8_E5M2, SCALE_E8M0)))

}  // namespace

template <typename T>
hipError_t launch_quantize_rows8(const T *A, int64_t n, int64_t d, int f8, int scale, const Mat8 &out, hipStream_t stream) {
    const int64_t groups = (n + kRowsPerGroup - 1) / kRowsPerGroup, blocks = (d + kBlock8 - 1) / kBlock8;
    // (2^31 rows are 2^27 work-groups of 2^8 threads, beyond the 2^32 threads of a launch: those are launched in parts)
    constexpr int64_t kMost = 1 << 20;
    for (int64_t g = 0; g < groups; g += kMost) {
        const int64_t row0 = g * kRowsPerGroup, here = groups - g < kMost ? groups - g : kMost;
        const int64_t width = (blocks + kBlocksPerGroup - 1) / kBlocksPerGroup, cut = width < 1024 ? width : 1024;
        const Mat8 o = {out.data + row0 * out.ld, out.ld, (char *)out.scales + row0 * (scale == SCALE_F32 ? 4 : 1), out.ld_scales};
#define CALL(F, S) quantize_rows8<T, F, S>(dim3((unsigned)here, (unsigned)cut), A + row0 * d, n - row0, d, o, stream)
        RMM_BY_FORMAT(CALL);
#undef CALL
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_quantize_weight8(const T *W, int64_t rows, int64_t cols, int f8, int scale, const Mat8 &out, const Mat8 *out_t,
                                   hipStream_t stream) {
    const int64_t blocks = ((rows + kBlock8 - 1) / kBlock8) * ((cols + kBlock8 - 1) / kBlock8);
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
    const Mat8 t = out_t != nullptr ? *out_t : Mat8{nullptr, 0, nullptr, 0};
#define CALL(F, S) quantize_weight8<T, F, S>(grid, W, rows, cols, out, t, stream)
    RMM_BY_FORMAT(CALL);
#undef CALL
    return hipGetLastError();
}

template hipError_t launch_quantize_rows8<bf16_t>(const bf16_t *, int64_t, int64_t, int, int, const Mat8 &, hipStream_t);
template hipError_t launch_quantize_rows8<float>(const float *, int64_t, int64_t, int, int, const Mat8 &, hipStream_t);
template hipError_t launch_quantize_weight8<bf16_t>(const bf16_t *, int64_t, int64_t, int, int, const Mat8 &, const Mat8 *, hipStream_t);
template hipError_t launch_quantize_weight8<float>(const float *, int64_t, int64_t, int, int, const Mat8 &, const Mat8 *, hipStream_t);

}  // namespace rmm
