// C ABI of the 8-bit operands and of the norm in front of them: argument checks and dispatch (include/rmm.h).
#include "api_checks.hpp"
#include "quant8.hpp"

using namespace rmm;

namespace {

bool dtype_ok(int dtype) { return dtype == RMM_DTYPE_F32 || dtype == RMM_DTYPE_BF16; }

// A rows x cols matrix with the scales of rows, or those of weights.
bool mat8_ok(const rmm_mat8_t *m, int64_t rows, int64_t cols, bool weights) {
    if (m == nullptr || m->data == nullptr || m->scales == nullptr || !aligned16(m->data) || !aligned16(m->scales)) return false;
    if (m->f8 != RMM_F8_E4M3 && m->f8 != RMM_F8_E5M2) return false;
    if (m->scale != RMM_SCALE_F32 && m->scale != RMM_SCALE_E8M0) return false;
    if (m->ld < cols || m->ld % 16 != 0 || m->ld > kMaxDim || rows * m->ld >= 2 * kMaxElems) return false;
    const int64_t blocks = (cols + kBlock8 - 1) / kBlock8;
    if (weights) return m->ld_scales >= blocks && m->ld_scales <= ((int64_t)1 << 26);
    return m->ld_scales >= rows && m->ld_scales % 16 == 0 && m->ld_scales <= kMaxDim;
}
Mat8 as_mat8(const rmm_mat8_t *m) { return Mat8{(uint8_t *)m->data, m->ld, m->scales, m->ld_scales}; }

static_assert(RMM_F8_E4M3 == F8_E4M3 && RMM_F8_E5M2 == F8_E5M2 && RMM_SCALE_F32 == SCALE_F32 && RMM_SCALE_E8M0 == SCALE_E8M0, "enums");

template <typename T>
int quantize8(int64_t n, int64_t d, const void *A, const rmm_mat8_t *out, hipStream_t stream) {
    return from_hip(launch_quantize_rows8<T>((const T *)A, n, d, out->f8, out->scale, as_mat8(out), stream));
}
template <typename T>
int quantize8_weight(int64_t rows, int64_t cols, const void *W, const rmm_mat8_t *out, const rmm_mat8_t *out_t, hipStream_t stream) {
    const Mat8 t = out_t != nullptr ? as_mat8(out_t) : Mat8{nullptr, 0, nullptr, 0};
    return from_hip(launch_quantize_weight8<T>((const T *)W, rows, cols, out->f8, out->scale, as_mat8(out), out_t != nullptr ? &t : nullptr, stream));
}
template <typename T>
int linear8(int64_t n, int64_t d_in, int64_t d_out, const rmm_mat8_t *X, const rmm_mat8_t *W, const void *bias, void *Y, hipStream_t stream) {
    return from_hip(launch_linear8<T>(as_mat8(X), as_mat8(W), (const T *)bias, (T *)Y, n, d_in, d_out, X->f8, X->scale, stream));
}
template <typename T>
int norm(int64_t n, int64_t d, float eps, const void *X, const void *residual, const void *weight, void *H, void *Y, const rmm_mat8_t *Y8,
         float *rstd, hipStream_t stream) {
    const Mat8 y8 = Y8 != nullptr ? as_mat8(Y8) : Mat8{nullptr, 0, nullptr, 0};
    return from_hip(launch_rms_norm<T>((const T *)X, (const T *)residual, (const T *)weight, (T *)H, (T *)Y, Y8 != nullptr ? &y8 : nullptr,
                                       Y8 != nullptr ? Y8->f8 : 0, Y8 != nullptr ? Y8->scale : 0, rstd, n, d, eps, stream));
}
template <typename T>
int norm_backward(int64_t n, int64_t d, const void *dY, const void *dH, const void *H, const void *weight, const float *rstd, void *dX,
                  void *dweight, void *ws, hipStream_t stream) {
    return from_hip(launch_rms_norm_backward<T>((const T *)dY, (const T *)dH, (const T *)H, (const T *)weight, rstd, (T *)dX, (T *)dweight,
                                                (float *)ws, n, d, stream));
}

}  // namespace

extern "C" {

int rmm_quantize8(int64_t n, int64_t d, int dtype, const void *A, const rmm_mat8_t *out, void *stream) {
    if (!dims_ok(n, d) || !dtype_ok(dtype) || A == nullptr || !aligned16(A) || !mat8_ok(out, n, d, false)) return RMM_ERR_INVALID_ARG;
    return dtype == RMM_DTYPE_BF16 ? quantize8<bf16_t>(n, d, A, out, (hipStream_t)stream) : quantize8<float>(n, d, A, out, (hipStream_t)stream);
}

int rmm_quantize8_weight(int64_t rows, int64_t cols, int dtype, const void *W, const rmm_mat8_t *out, const rmm_mat8_t *out_t, void *stream) {
    if (!dims_ok(rows, cols) || !dtype_ok(dtype) || W == nullptr || !aligned16(W) || !mat8_ok(out, rows, cols, true)) return RMM_ERR_INVALID_ARG;
    if (out_t != nullptr && (!mat8_ok(out_t, cols, rows, true) || out_t->f8 != out->f8 || out_t->scale != out->scale)) return RMM_ERR_INVALID_ARG;
    return dtype == RMM_DTYPE_BF16 ? quantize8_weight<bf16_t>(rows, cols, W, out, out_t, (hipStream_t)stream)
                                   : quantize8_weight<float>(rows, cols, W, out, out_t, (hipStream_t)stream);
}

int rmm_linear8(int64_t n, int64_t d_in, int64_t d_out, int dtype, const rmm_mat8_t *X, const rmm_mat8_t *W, const void *bias, void *Y,
                void *stream) {
    if (!dims_ok(n, d_in) || !dims_ok(n, d_out) || !dims_ok(d_out, d_in) || !dtype_ok(dtype)) return RMM_ERR_INVALID_ARG;
    if (!mat8_ok(X, n, d_in, false) || !mat8_ok(W, d_out, d_in, true) || W->f8 != RMM_F8_E4M3 || W->scale != X->scale) return RMM_ERR_INVALID_ARG;
    if (Y == nullptr || !aligned16(Y) || !aligned16(bias)) return RMM_ERR_INVALID_ARG;
    return dtype == RMM_DTYPE_BF16 ? linear8<bf16_t>(n, d_in, d_out, X, W, bias, Y, (hipStream_t)stream)
                                   : linear8<float>(n, d_in, d_out, X, W, bias, Y, (hipStream_t)stream);
}

int rmm_rms_norm(int64_t n, int64_t d, int dtype, float eps, const void *X, const void *residual, const void *weight, void *H, void *Y,
                 const rmm_mat8_t *Y8, float *rstd, void *stream) {
    if (!dims_ok(n, d) || !dtype_ok(dtype) || X == nullptr || weight == nullptr || (Y == nullptr && Y8 == nullptr)) return RMM_ERR_INVALID_ARG;
    if (!(eps >= 0.0f && eps < INFINITY)) return RMM_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(residual) || !aligned16(weight) || !aligned16(H) || !aligned16(Y) || !aligned16(rstd)) return RMM_ERR_INVALID_ARG;
    if (Y8 != nullptr && !mat8_ok(Y8, n, d, false)) return RMM_ERR_INVALID_ARG;
    return dtype == RMM_DTYPE_BF16 ? norm<bf16_t>(n, d, eps, X, residual, weight, H, Y, Y8, rstd, (hipStream_t)stream)
                                   : norm<float>(n, d, eps, X, residual, weight, H, Y, Y8, rstd, (hipStream_t)stream);
}

size_t rmm_rms_norm_workspace_bytes(int64_t n, int64_t d, int dtype) {
    return dims_ok(n, d) && dtype_ok(dtype) ? round_up(norm_backward_partials(n, d) * sizeof(float), 256) : 0;
}

int rmm_rms_norm_backward(int64_t n, int64_t d, int dtype, const void *dY, const void *dH, const void *H, const void *weight,
                          const float *rstd, void *dX, void *dweight, void *ws, size_t ws_bytes, void *stream) {
    if (!dims_ok(n, d) || !dtype_ok(dtype) || dY == nullptr || H == nullptr || weight == nullptr || rstd == nullptr) return RMM_ERR_INVALID_ARG;
    if (dX == nullptr && dweight == nullptr) return RMM_ERR_INVALID_ARG;
    if (!aligned16(dY) || !aligned16(dH) || !aligned16(H) || !aligned16(weight) || !aligned16(rstd) || !aligned16(dX) || !aligned16(dweight) ||
        !aligned16(ws))
        return RMM_ERR_INVALID_ARG;
    if (dweight != nullptr && (ws == nullptr || ws_bytes < rmm_rms_norm_workspace_bytes(n, d, dtype))) return RMM_ERR_WORKSPACE;
    return dtype == RMM_DTYPE_BF16 ? norm_backward<bf16_t>(n, d, dY, dH, H, weight, rstd, dX, dweight, ws, (hipStream_t)stream)
                                   : norm_backward<float>(n, d, dY, dH, H, weight, rstd, dX, dweight, ws, (hipStream_t)stream);
}

}  // extern "C"
