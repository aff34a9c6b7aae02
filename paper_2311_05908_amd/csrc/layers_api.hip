// C ABI of the operators around the convolutions: argument checks, then the kernels' files. See include/fftconv.h for the contracts.
#include "layers_internal.h"

using namespace fftconv;

namespace {

constexpr int64_t MOST = ((int64_t)1 << 31) - 1;
constexpr int64_t MOST_ROWS = MOST + 1 - 512;      // of a projection's operands: the end of the last tile, and a store's beyond it, fit 32 bits
constexpr int64_t MOST_OUT = (int64_t)1 << 42;     // values of a projection's result, so that its tiles are a number of 32 bits
constexpr int64_t MOST_DW = (int64_t)1 << 36;      // values of a weight's gradient
constexpr int64_t MOST_K = 131071;                 // sums of so many products of 8-bit numbers fit 32 bits

int bad(const char *who, const char *what)
{
    set_error("%s: %s", who, what);
    return FFTCONV_EINVAL;
}
bool known(int dtype) { return dtype == FFTCONV_F32 || dtype == FFTCONV_F16 || dtype == FFTCONV_BF16; }
int64_t size_of(int dtype) { return dtype == FFTCONV_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }
// a * b for non-negative numbers, or -1 where it is over `most`
int64_t times(int64_t a, int64_t b, int64_t most = MOST) { return a < 0 || b < 0 || (a > 0 && b > most / a) ? -1 : a * b; }

int check_rows(const char *who, const void *x, int64_t ldx, int64_t T, int64_t D, int dtype)
{
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (D < 1 || T < 0 || T > MOST) return bad(who, "T >= 0 and D >= 1 are wanted, T below 2^31");
    if (ldx < D) return bad(who, "rows overlap: their distance is below D");
    if (T > 0 && !x) return bad(who, "a tensor is NULL");
    if (!aligned(x, size_of(dtype))) return bad(who, "a tensor is not aligned to its elements");
    if (D > lay::MAX_ROW) {
        set_error("%s: rows of %lld values: up to %lld are supported", who, (long long)D, (long long)lay::MAX_ROW);
        return FFTCONV_EUNSUPPORTED;
    }
    return FFTCONV_OK;
}

int check_acts(const char *who, int64_t B, int64_t C, int64_t N, int dtype)
{
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (B < 0 || C < 1 || N < 1) return bad(who, "B >= 0, C >= 1 and N >= 1 are wanted");
    if (times(B, C, INT64_MAX / 64) < 0 || times(times(B, C, INT64_MAX / 64), N, INT64_MAX / 64) < 0) return bad(who, "too many values");
    if (times(times(B, C, INT64_MAX / 64), (N + 127) / 128, INT64_MAX / 64) > (int64_t)1 << 35) {
        set_error("%s: over 2^35 runs of 128 samples", who);
        return FFTCONV_EUNSUPPORTED;
    }
    return FFTCONV_OK;
}

int check_linear(const char *who, int64_t B, int64_t N, int64_t K, int64_t O, int64_t parts, int dtype)
{
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (B < 0 || N < 1 || K < 1 || O < 1 || times(B, N, MOST_ROWS) < 0 || O > MOST_ROWS)
        return bad(who, "B >= 0, N, K, O >= 1 are wanted, B N and O up to 2^31 - 512");
    if (parts < 0 || (parts > 0 && O % parts != 0)) return bad(who, "parts has to divide O");
    if (times(B * N, O, MOST_OUT) < 0) {
        set_error("%s: B N O=%lld x %lld values of y: up to 2^42 are supported", who, (long long)(B * N), (long long)O);
        return FFTCONV_EUNSUPPORTED;
    }
    if (K > MOST_K) {
        set_error("%s: sums of K=%lld products may leave 32 bits: up to %lld are supported", who, (long long)K, (long long)MOST_K);
        return FFTCONV_EUNSUPPORTED;
    }
    return FFTCONV_OK;
}

int check_weight(const char *who, int64_t B, int64_t N, int64_t O, int64_t C, int dtype)
{
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (B < 0 || N < 1 || O < 1 || C < 1 || O > MOST || C > MOST || N > MOST || times(B, (N + 127) / 128) < 0)
        return bad(who, "B >= 0, N, O, C >= 1 are wanted, N, O, C and B ceil(N / 128) below 2^31");
    if (N > ((int64_t)1 << 22) || O > ((int64_t)1 << 22) || C > ((int64_t)1 << 22)) {        // (distances inside a tile are 32-bit numbers)
        set_error("%s: sequences of %lld samples, %lld x %lld channels: up to 2^22 are supported", who, (long long)N, (long long)O, (long long)C);
        return FFTCONV_EUNSUPPORTED;
    }
    if (O * C > MOST_DW) {                             // (tiles of 512 threads: a launch has less than 2^32)
        set_error("%s: %lld x %lld values of dw: up to 2^36 are supported", who, (long long)O, (long long)C);
        return FFTCONV_EUNSUPPORTED;
    }
    return FFTCONV_OK;
}

}  // namespace

extern "C" {

int fftconv_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const float *weight, void *y, void *h, float *rstd,
                     float *scale, int64_t T, int64_t D, double eps, int dtype, void *stream)
{
    const char *const who = "fftconv_rms_norm";
    FC_TRY(check_rows(who, x, ldx, T, D, dtype));
    if (residual) FC_TRY(check_rows(who, residual, ldr, T, D, dtype));
    if (!(eps >= 0.0) || eps > 3e38) return bad(who, "eps has to be a number >= 0");
    if (T == 0) return FFTCONV_OK;
    if (!weight || !y) return bad(who, "a tensor is NULL");
    if (!aligned(weight, 4) || !aligned(rstd, 4) || !aligned(scale, 4) || !aligned(h, size_of(dtype)) || !aligned(y, scale ? 1 : size_of(dtype)))
        return bad(who, "a tensor is not aligned to its elements");
    return lay::rows_forward(x, ldx, residual, ldr, weight, y, h, rstd, scale, T, D, eps, 1, scale != nullptr, dtype, (hipStream_t)stream);
}

int fftconv_quantize_rows(const void *x, int64_t ldx, int8_t *q, float *scale, int64_t T, int64_t D, int dtype, void *stream)
{
    const char *const who = "fftconv_quantize_rows";
    FC_TRY(check_rows(who, x, ldx, T, D, dtype));
    if (T == 0) return FFTCONV_OK;
    if (!q || !scale) return bad(who, "a tensor is NULL");
    if (!aligned(scale, 4)) return bad(who, "a tensor is not aligned to its elements");
    return lay::rows_forward(x, ldx, nullptr, 0, nullptr, q, nullptr, nullptr, scale, T, D, 0.0, 0, 1, dtype, (hipStream_t)stream);
}

size_t fftconv_workspace_bytes_rms_norm_backward(int64_t T, int64_t D, int dtype)
{
    return T < 1 || D < 1 || D > lay::MAX_ROW || T > MOST || !known(dtype) ? 0 : lay::rms_norm_backward_workspace(T, D, dtype);
}

int fftconv_rms_norm_backward(const void *dy, int64_t lddy, const void *h, const void *dh, const float *weight, const float *rstd, void *dx,
                              float *dweight, int64_t T, int64_t D, int dtype, void *workspace, void *stream)
{
    const char *const who = "fftconv_rms_norm_backward";
    FC_TRY(check_rows(who, dy, lddy, T, D, dtype));
    FC_TRY(check_rows(who, h, D, T, D, dtype));
    if (!dweight || !weight || (T > 0 && (!rstd || !dx))) return bad(who, "a tensor is NULL");
    if (!aligned(weight, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(workspace, 4) || !aligned(dh, size_of(dtype)) ||
        !aligned(dx, size_of(dtype)))
        return bad(who, "a tensor is not aligned to its elements");
    if (!workspace && fftconv_workspace_bytes_rms_norm_backward(T, D, dtype) != 0) return bad(who, "the workspace is NULL");
    return lay::rms_norm_backward(dy, lddy, h, dh, weight, rstd, dx, dweight, T, D, dtype, workspace, (hipStream_t)stream);
}

size_t fftconv_workspace_bytes_linear_i8(int64_t B, int64_t N, int64_t K, int64_t O, int64_t parts, int dtype)
{
    if (B < 1 || check_linear("fftconv_workspace_bytes_linear_i8", B, N, K, O, parts, dtype) != FFTCONV_OK) return 0;
    return lay::linear_i8_workspace(B * N, K, O);
}

int fftconv_linear_i8(const int8_t *x, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, int64_t B,
                      int64_t N, int64_t K, int64_t O, int64_t parts, int dtype, void *workspace, void *stream)
{
    const char *const who = "fftconv_linear_i8";
    FC_TRY(check_linear(who, B, N, K, O, parts, dtype));
    if (B == 0) return FFTCONV_OK;
    if (!x || !x_scale || !w || !w_scale || !y) return bad(who, "a tensor is NULL");
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(workspace, 4) || !aligned(y, size_of(dtype)))
        return bad(who, "a tensor is not aligned to its elements");
    if (!workspace && fftconv_workspace_bytes_linear_i8(B, N, K, O, parts, dtype) != 0) return bad(who, "the workspace is NULL");
    return lay::linear_i8(x, x_scale, w, w_scale, bias, y, B, N, K, O, parts, dtype, workspace, (hipStream_t)stream);
}

int fftconv_act_pack(const void *x, int8_t *q, float *scale, int64_t B, int64_t C, int64_t N, int tokens, int dtype, void *stream)
{
    const char *const who = "fftconv_act_pack";
    FC_TRY(check_acts(who, B, C, N, dtype));
    if (B == 0) return FFTCONV_OK;
    if (!x || !q || !scale) return bad(who, "a tensor is NULL");
    if (!aligned(x, size_of(dtype)) || !aligned(scale, 4)) return bad(who, "a tensor is not aligned to its elements");
    return lay::act_pack(x, q, scale, B, C, N, tokens != 0, dtype, (hipStream_t)stream);
}

int fftconv_act_unpack(const int8_t *q, const float *scale, const int8_t *gate_q, const float *gate_scale, const void *gate, void *x, int64_t B,
                       int64_t C, int64_t N, int dtype, void *stream)
{
    const char *const who = "fftconv_act_unpack";
    FC_TRY(check_acts(who, B, C, N, dtype));
    if ((gate_q != nullptr) != (gate_scale != nullptr) || (gate_q && gate)) return bad(who, "gate_q goes with gate_scale and without gate");
    if (B == 0) return FFTCONV_OK;
    if (!q || !scale || !x) return bad(who, "a tensor is NULL");
    if (!aligned(x, size_of(dtype)) || !aligned(gate, size_of(dtype)) || !aligned(scale, 4) || !aligned(gate_scale, 4))
        return bad(who, "a tensor is not aligned to its elements");
    return lay::act_unpack(q, scale, gate_q, gate_scale, gate, x, B, C, N, dtype, (hipStream_t)stream);
}

size_t fftconv_workspace_bytes_linear_grad_weight(int64_t B, int64_t N, int64_t O, int64_t C, int tokens, int dtype)
{
    (void)tokens;
    if (check_weight("fftconv_workspace_bytes_linear_grad_weight", B, N, O, C, dtype) != FFTCONV_OK) return 0;
    return lay::weight_grad_workspace(B, N, O, C, dtype);
}

int fftconv_linear_grad_weight(const void *dy, const int8_t *q, const float *scale, void *dw, int64_t B, int64_t N, int64_t O, int64_t C,
                               int tokens, int dtype, int dtype_dw, void *workspace, void *stream)
{
    const char *const who = "fftconv_linear_grad_weight";
    FC_TRY(check_weight(who, B, N, O, C, dtype));
    if (dtype_dw != FFTCONV_F32 && dtype_dw != dtype) return bad(who, "dw is in fp32 or in the type of dy");
    if (!dw || !workspace || (B > 0 && (!dy || !q || !scale))) return bad(who, "a tensor is NULL");
    if (!aligned(dy, size_of(dtype)) || !aligned(scale, 4) || !aligned(dw, size_of(dtype_dw)) || !aligned(workspace, 4))
        return bad(who, "a tensor is not aligned to its elements");
    return lay::weight_grad(dy, q, scale, dw, B, N, O, C, tokens != 0, dtype, dtype_dw, workspace, (hipStream_t)stream);
}

}  // extern "C"
