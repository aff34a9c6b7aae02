// Declarations of the operators around the convolutions, between layers_api.hip and the kernels' files.
#pragma once

#include <type_traits>

#include "fused3_common.h"
#include "layers_common.h"

namespace fftconv {
namespace lay {

using f3::lds_barrier;

// row_norm.hip
constexpr int64_t MAX_ROW = 16384;
int rows_forward(const void *x, int64_t ldx, const void *r, int64_t ldr, const float *w, void *y, void *h, float *rstd, float *scale, int64_t T,
                 int64_t D, double eps, int norm, int i8, int dtype, hipStream_t s);
size_t rms_norm_backward_workspace(int64_t T, int64_t D, int dtype);
int rms_norm_backward(const void *dy, int64_t lddy, const void *h, const void *dh, const float *w, const float *rstd, void *dx, float *dw,
                      int64_t T, int64_t D, int dtype, void *workspace, hipStream_t s);

// checkpoint.hip
int act_pack(const void *x, int8_t *q, float *scale, int64_t B, int64_t C, int64_t N, bool tokens, int dtype, hipStream_t s);
int act_unpack(const int8_t *q, const float *scale, const int8_t *gq, const float *gscale, const void *gate, void *x, int64_t B, int64_t C,
               int64_t N, int dtype, hipStream_t s);

// linear_i8.hip
size_t linear_i8_workspace(int64_t T, int64_t K, int64_t O);
int linear_i8(const int8_t *xq, const float *xs, const int8_t *wq, const float *ws, const float *bias, void *y, int64_t B, int64_t N, int64_t K,
              int64_t O, int64_t parts, int dtype, void *workspace, hipStream_t s);

// weight_grad.hip
size_t weight_grad_workspace(int64_t B, int64_t N, int64_t O, int64_t C, int dtype_dy);
int weight_grad(const void *dy, const int8_t *q, const float *scale, void *dw, int64_t B, int64_t N, int64_t O, int64_t C, bool tokens,
                int dtype_dy, int dtype_dw, void *workspace, hipStream_t s);

}  // namespace lay
}  // namespace fftconv
