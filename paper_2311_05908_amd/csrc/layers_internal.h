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

// gated_scan.hip
size_t gated_scan_workspace(int64_t rows, int64_t N);
int gated_scan(const void *u, const void *w, const void *v, const float *state, const int32_t *lengths, void *y, float *last, float *kept, int64_t B,
               int64_t C, int64_t N, int gate, int dtype, void *workspace, hipStream_t s);
int gated_scan_backward(const void *dy, const void *u, const void *w, const void *v, const float *kept, const float *dlast, const int32_t *lengths,
                        void *du, void *dw, void *dv, float *dstate, int64_t B, int64_t C, int64_t N, int gate, int dtype, void *workspace,
                        hipStream_t s);
int gated_step(const void *u, const void *w, const void *v, const float *state, float *next, void *y, int64_t T, int gate, int dtype, hipStream_t s);

// block_scale.hip
int quantize_blocks(const void *x, int64_t ldx, uint8_t *q, float *scale, int64_t T, int64_t K, int dtype, hipStream_t s);
int quantize_blocks_channels(const void *x, uint8_t *q, float *scale, int64_t B, int64_t N, int64_t K, int64_t parts, int dtype, hipStream_t s);
int quantize_tiles(const void *x, int64_t ldx, uint8_t *q, float *scale, uint8_t *qt, float *scale_t, int64_t O, int64_t K, int dtype, hipStream_t s);

// linear_f8.hip
size_t linear_f8_workspace(int64_t T, int64_t K, int64_t O);
int linear_f8(const uint8_t *x, const float *xs, const uint8_t *w, const float *ws, const float *bias, void *y, int64_t B, int64_t N, int64_t K,
              int64_t O, int64_t parts, int dtype, void *workspace, hipStream_t s);

// grad_clip.hip
size_t clip_workspace(const int64_t *counts, int64_t tensors);
int clip_overlaps(const void *const *in, void *const *out, const int64_t *counts, const int *types, const int *types_out, int64_t tensors,
                  const float *norm_in, const float *norm, const void *workspace);
int clip_grads(const void *const *in, void *const *out, const int64_t *counts, const int *types, const int *types_out, int64_t tensors, double limit,
               double eps, const float *norm_in, float *norm, void *workspace, hipStream_t s);

}  // namespace lay
}  // namespace fftconv
