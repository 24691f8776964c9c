// Y = X W^T (+ bias) with 8-bit operands: Y(i, o) = sum over blocks b of 128 contraction elements of
// sx(b, i) sw(o / 128, b) * (sum over the block of X W), in fp32.  Host side.
#include "linear8_frag.hpp"
#include "linear8_plan.hpp"

namespace rmm {

template <typename T>
hipError_t launch_linear8(const Mat8 &X, const Mat8 &W, const T *bias, T *Y, int64_t n, int64_t d_in, int64_t d_out, int f8, int scale,
                          hipStream_t stream) {
    const Linear8Args g = {X, W, bias, Y, n, d_in, d_out};
    const int kernel = linear8_plan(n, d_in, d_out, X.ld, W.ld, sizeof(T) == 4);
    if (f8 == F8_E4M3)
        scale == SCALE_F32 ? launch_linear8_by<F8_E4M3, SCALE_F32, T>(kernel, g, stream) : launch_linear8_by<F8_E4M3, SCALE_E8M0, T>(kernel, g, stream);
    else
        scale == SCALE_F32 ? launch_linear8_by<F8_E5M2, SCALE_F32, T>(kernel, g, stream) : launch_linear8_by<F8_E5M2, SCALE_E8M0, T>(kernel, g, stream);
    return hipGetLastError();
}

template hipError_t launch_linear8<bf16_t>(const Mat8 &, const Mat8 &, const bf16_t *, bf16_t *, int64_t, int64_t, int64_t, int, int, hipStream_t);
template hipError_t launch_linear8<float>(const Mat8 &, const Mat8 &, const float *, float *, int64_t, int64_t, int64_t, int, int, hipStream_t);

}  // namespace rmm
