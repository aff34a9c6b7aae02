// C ABI of the operators around the convolutions: argument checks, then the kernels' files. See include/fftconv.h for the contracts.
#include "layers_internal.h"

using namespace fftconv;

namespace {

constexpr int64_t MOST = ((int64_t)1 << 31) - 1;
constexpr int64_t MOST_ROWS = MOST + 1 - 512;      // of a projection's operands: the end of the last tile, and a store's beyond it, fit 32 bits
constexpr int64_t MOST_OUT = (int64_t)1 << 42;     // values of a projection's result, so that its tiles are a number of 32 bits
constexpr int64_t MOST_DW = (int64_t)1 << 36;      // values of a weight's gradient
constexpr int64_t MOST_K = 131071;                 // sums of so many products of 8-bit numbers fit 32 bits
constexpr int64_t MOST_K_F8 = (int64_t)1 << 20;    // (places within a tile's 256 rows are 32-bit numbers)
constexpr int64_t MOST_COUNT = (int64_t)1 << 40;   // values of a gradient

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

// What a call reads or writes; nothing where `at` is NULL, or of no bytes.
struct Place {
    const void *at;
    int64_t bytes;
};
bool meet(const Place &a, const Place &b)
{
    return a.at && b.at && a.bytes > 0 && b.bytes > 0 && (uintptr_t)a.at < (uintptr_t)b.at + (uintptr_t)b.bytes && (uintptr_t)b.at < (uintptr_t)a.at + (uintptr_t)a.bytes;
}
// Whether one of the first `written` places meets another one.
template <int N> bool overlap(const Place (&p)[N], int written)
{
    for (int i = 0; i < written; ++i)
        for (int j = i + 1; j < N; ++j)
            if (meet(p[i], p[j])) return true;
    return false;
}

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

int check_linear(const char *who, int64_t B, int64_t N, int64_t K, int64_t O, int64_t parts, int dtype, int64_t most_k, const char *why_k)
{
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (B < 0 || N < 1 || K < 1 || O < 1 || times(B, N, MOST_ROWS) < 0 || O > MOST_ROWS)
        return bad(who, "B >= 0, N, K, O >= 1 are wanted, B N and O up to 2^31 - 512");
    if (parts < 0 || (parts > 0 && O % parts != 0)) return bad(who, "parts has to divide O");
    if (times(B * N, O, MOST_OUT) < 0) {
        set_error("%s: B N O=%lld x %lld values of y: up to 2^42 are supported", who, (long long)(B * N), (long long)O);
        return FFTCONV_EUNSUPPORTED;
    }
    if (K > most_k) {
        set_error("%s: %s=%lld%s: up to %lld are supported", who, why_k, (long long)K, most_k == MOST_K ? " products may leave 32 bits" : "", (long long)most_k);
        return FFTCONV_EUNSUPPORTED;
    }
    return FFTCONV_OK;
}
int check_i8(const char *who, int64_t B, int64_t N, int64_t K, int64_t O, int64_t parts, int dtype)
{
    return check_linear(who, B, N, K, O, parts, dtype, MOST_K, "sums of K");
}
int check_f8(const char *who, int64_t B, int64_t N, int64_t K, int64_t O, int64_t parts, int dtype)
{
    return check_linear(who, B, N, K, O, parts, dtype, MOST_K_F8, "rows of K");
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

int check_scan(const char *who, int64_t B, int64_t C, int64_t N, int gate, int dtype)
{
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (gate != FFTCONV_GATE_SIGMOID && gate != FFTCONV_GATE_LOG) return bad(who, "unknown gate");
    if (B < 0 || C < 1 || N < 1 || N > MOST || times(B, C) < 0) return bad(who, "B >= 0, C >= 1 and N >= 1 are wanted, B C and N below 2^31");
    if (times(B * C, N, INT64_MAX / 64) < 0) return bad(who, "too many values");
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
    if (B < 1 || check_i8("fftconv_workspace_bytes_linear_i8", B, N, K, O, parts, dtype) != FFTCONV_OK) return 0;
    return lay::linear_i8_workspace(B * N, K, O);
}

int fftconv_linear_i8(const int8_t *x, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, int64_t B,
                      int64_t N, int64_t K, int64_t O, int64_t parts, int dtype, void *workspace, void *stream)
{
    const char *const who = "fftconv_linear_i8";
    FC_TRY(check_i8(who, B, N, K, O, parts, dtype));
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

size_t fftconv_workspace_bytes_gated_scan(int64_t B, int64_t C, int64_t N, int dtype)
{
    if (check_scan("fftconv_workspace_bytes_gated_scan", B, C, N, FFTCONV_GATE_LOG, dtype) != FFTCONV_OK) return 0;
    return lay::gated_scan_workspace(B * C, N);
}

int fftconv_gated_scan(const void *u, const void *w, const void *v, const float *state, const int32_t *lengths, void *y, float *last, float *kept,
                       int64_t B, int64_t C, int64_t N, int gate, int dtype, void *workspace, void *stream)
{
    const char *const who = "fftconv_gated_scan";
    FC_TRY(check_scan(who, B, C, N, gate, dtype));
    if (B == 0) return FFTCONV_OK;
    if (!u || !w || !y) return bad(who, "a tensor is NULL");
    const int64_t to = size_of(dtype);
    if (!aligned(u, to) || !aligned(w, to) || !aligned(v, to) || !aligned(y, to) || !aligned(state, 4) || !aligned(lengths, 4) || !aligned(last, 4) ||
        !aligned(kept, 4) || !aligned(workspace, 8))
        return bad(who, "a tensor is not aligned to its elements");
    const int64_t work = (int64_t)lay::gated_scan_workspace(B * C, N), rows = 4 * B * C, all = to * B * C * N;
    if (!workspace && work != 0) return bad(who, "the workspace is NULL");
    const Place places[] = {{y, all}, {last, rows}, {kept, rows * ((N + 511) / 512)}, {workspace, work}, {u, all}, {w, all}, {v, all}, {state, rows}, {lengths, 4 * B}};
    if (overlap(places, 4)) return bad(who, "a result or the workspace overlaps another tensor");
    return lay::gated_scan(u, w, v, state, lengths, y, last, kept, B, C, N, gate, dtype, workspace, (hipStream_t)stream);
}

int fftconv_gated_scan_backward(const void *dy, const void *u, const void *w, const void *v, const float *kept, const float *dlast,
                                const int32_t *lengths, void *du, void *dw, void *dv, float *dstate, int64_t B, int64_t C, int64_t N, int gate,
                                int dtype, void *workspace, void *stream)
{
    const char *const who = "fftconv_gated_scan_backward";
    FC_TRY(check_scan(who, B, C, N, gate, dtype));
    if ((v != nullptr) != (dv != nullptr)) return bad(who, "dv goes with v");
    if (B == 0) return FFTCONV_OK;
    if (!dy || !u || !w || !kept || !du || !dw) return bad(who, "a tensor is NULL");
    const int64_t to = size_of(dtype);
    if (!aligned(dy, to) || !aligned(u, to) || !aligned(w, to) || !aligned(v, to) || !aligned(du, to) || !aligned(dw, to) || !aligned(dv, to) ||
        !aligned(kept, 4) || !aligned(dlast, 4) || !aligned(lengths, 4) || !aligned(dstate, 4) || !aligned(workspace, 8))
        return bad(who, "a tensor is not aligned to its elements");
    const int64_t work = (int64_t)lay::gated_scan_workspace(B * C, N), rows = 4 * B * C, all = to * B * C * N;
    if (!workspace && work != 0) return bad(who, "the workspace is NULL");
    const Place places[] = {{du, all}, {dw, all}, {dv, all}, {dstate, rows}, {workspace, work}, {dy, all}, {u, all}, {w, all}, {v, all}, {kept, rows * ((N + 511) / 512)},
                            {dlast, rows}, {lengths, 4 * B}};
    if (overlap(places, 5)) return bad(who, "a result or the workspace overlaps another tensor");
    return lay::gated_scan_backward(dy, u, w, v, kept, dlast, lengths, du, dw, dv, dstate, B, C, N, gate, dtype, workspace, (hipStream_t)stream);
}

int fftconv_gated_step(const void *u, const void *w, const void *v, const float *state, float *next, void *y, int64_t T, int gate, int dtype,
                       void *stream)
{
    const char *const who = "fftconv_gated_step";
    FC_TRY(check_scan(who, T, 1, 1, gate, dtype));
    if (T == 0) return FFTCONV_OK;
    if (!u || !w || !state || !next || !y) return bad(who, "a tensor is NULL");
    const int64_t to = size_of(dtype);
    if (!aligned(u, to) || !aligned(w, to) || !aligned(v, to) || !aligned(y, to) || !aligned(state, 4) || !aligned(next, 4))
        return bad(who, "a tensor is not aligned to its elements");
    const Place places[] = {{next, 4 * T}, {y, to * T}, {u, to * T}, {w, to * T}, {v, to * T}, {next == state ? nullptr : state, 4 * T}};
    if (overlap(places, 2)) return bad(who, "a result overlaps another tensor (next may be state itself)");
    return lay::gated_step(u, w, v, state, next, y, T, gate, dtype, (hipStream_t)stream);
}

int fftconv_quantize_blocks(const void *x, int64_t ldx, uint8_t *q, float *scale, int64_t T, int64_t K, int dtype, void *stream)
{
    const char *const who = "fftconv_quantize_blocks";
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (T < 0 || T > MOST || K < 1) return bad(who, "T >= 0 and K >= 1 are wanted, T below 2^31");
    if (K > MOST_K_F8) {
        set_error("%s: rows of K=%lld: up to %lld are supported", who, (long long)K, (long long)MOST_K_F8);
        return FFTCONV_EUNSUPPORTED;
    }
    if (ldx < K || times(T, ldx, INT64_MAX / 64) < 0) return bad(who, "the distance of rows is below K, or too large");
    if (T == 0) return FFTCONV_OK;
    if (!x || !q || !scale) return bad(who, "a tensor is NULL");
    if (!aligned(x, size_of(dtype)) || !aligned(scale, 4)) return bad(who, "a tensor is not aligned to its elements");
    return lay::quantize_blocks(x, ldx, q, scale, T, K, dtype, (hipStream_t)stream);
}

int fftconv_quantize_blocks_channels(const void *x, uint8_t *q, float *scale, int64_t B, int64_t N, int64_t K, int64_t parts, int dtype, void *stream)
{
    const char *const who = "fftconv_quantize_blocks_channels";
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (B < 0 || N < 1 || K < 1 || times(B, N) < 0) return bad(who, "B >= 0, N >= 1 and K >= 1 are wanted, B N below 2^31");
    if (parts < 1 || K % parts != 0) return bad(who, "parts has to divide K");
    if (K > MOST_K_F8) {
        set_error("%s: rows of K=%lld: up to %lld are supported", who, (long long)K, (long long)MOST_K_F8);
        return FFTCONV_EUNSUPPORTED;
    }
    if (B == 0) return FFTCONV_OK;
    if (!x || !q || !scale) return bad(who, "a tensor is NULL");
    if (!aligned(x, size_of(dtype)) || !aligned(scale, 4)) return bad(who, "a tensor is not aligned to its elements");
    return lay::quantize_blocks_channels(x, q, scale, B, N, K, parts, dtype, (hipStream_t)stream);
}

int fftconv_quantize_tiles(const void *x, int64_t ldx, uint8_t *q, float *scale, uint8_t *qt, float *scale_t, int64_t O, int64_t K, int dtype, void *stream)
{
    const char *const who = "fftconv_quantize_tiles";
    if (!known(dtype)) return bad(who, "unknown dtype");
    if (O < 1 || K < 1 || O > MOST || K > MOST) return bad(who, "O, K >= 1 are wanted, below 2^31");
    if (ldx < K || times(O, ldx, INT64_MAX / 64) < 0) return bad(who, "the distance of rows is below K, or too large");
    if (!x || (!q && !qt)) return bad(who, "a tensor is NULL");
    if ((q != nullptr) != (scale != nullptr) || (qt != nullptr) != (scale_t != nullptr)) return bad(who, "8-bit values go with their scales");
    if (!aligned(x, size_of(dtype)) || !aligned(scale, 4) || !aligned(scale_t, 4)) return bad(who, "a tensor is not aligned to its elements");
    return lay::quantize_tiles(x, ldx, q, scale, qt, scale_t, O, K, dtype, (hipStream_t)stream);
}

size_t fftconv_workspace_bytes_linear_f8(int64_t B, int64_t N, int64_t K, int64_t O, int64_t parts, int dtype)
{
    if (B < 1 || check_f8("fftconv_workspace_bytes_linear_f8", B, N, K, O, parts, dtype) != FFTCONV_OK) return 0;
    return lay::linear_f8_workspace(B * N, K, O);
}

int fftconv_linear_f8(const uint8_t *x, const float *x_scale, const uint8_t *w, const float *w_scale, const float *bias, void *y, int64_t B, int64_t N,
                      int64_t K, int64_t O, int64_t parts, int dtype, void *workspace, void *stream)
{
    const char *const who = "fftconv_linear_f8";
    FC_TRY(check_f8(who, B, N, K, O, parts, dtype));
    if (B == 0) return FFTCONV_OK;
    if (!x || !x_scale || !w || !w_scale || !y) return bad(who, "a tensor is NULL");
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(workspace, 4) || !aligned(y, size_of(dtype)))
        return bad(who, "a tensor is not aligned to its elements");
    if (!workspace && fftconv_workspace_bytes_linear_f8(B, N, K, O, parts, dtype) != 0) return bad(who, "the workspace is NULL");
    return lay::linear_f8(x, x_scale, w, w_scale, bias, y, B, N, K, O, parts, dtype, workspace, (hipStream_t)stream);
}

size_t fftconv_workspace_bytes_clip_grads(const int64_t *counts, int64_t tensors)
{
    if (tensors < 0 || (tensors > 0 && !counts)) return 0;
    for (int64_t i = 0; i < tensors; ++i)
        if (counts[i] < 0 || counts[i] > MOST_COUNT) return 0;
    return lay::clip_workspace(counts, tensors);
}

int fftconv_clip_grads(const void *const *grads, void *const *out, const int64_t *counts, const int *dtypes, const int *dtypes_out, int64_t tensors,
                       double max_norm, double eps, const float *norm_in, float *norm, void *workspace, void *stream)
{
    const char *const who = "fftconv_clip_grads";
    if (tensors < 0 || (tensors > 0 && (!grads || !counts || !dtypes))) return bad(who, "an array is NULL, or the number of tensors below 0");
    if (!norm_in && !workspace) return bad(who, "the workspace is NULL");
    if (!out && norm_in) return bad(who, "nothing to do: a norm is given, and no tensors to write");
    if (!aligned(norm, 4) || !aligned(norm_in, 4) || !aligned(workspace, 8)) return bad(who, "a tensor is not aligned to its elements");
    if (out && (!(max_norm >= 0.0) || !(eps >= 0.0) || (max_norm == 0.0 && eps == 0.0))) return bad(who, "max_norm and eps have to be numbers >= 0, one of them above");
    const int *const types_out = dtypes_out ? dtypes_out : dtypes;
    for (int64_t i = 0; i < tensors; ++i) {
        if (!known(dtypes[i])) return bad(who, "unknown dtype");
        if (counts[i] < 0 || counts[i] > MOST_COUNT) return bad(who, "a tensor has 0 to 2^40 values");
        if (out && types_out[i] != dtypes[i] && types_out[i] != FFTCONV_F32) return bad(who, "results are in the type of the gradient or in fp32");
        if (counts[i] > 0 && (!grads[i] || (out && !out[i]))) return bad(who, "a tensor is NULL");
        if (!aligned(grads[i], size_of(dtypes[i])) || (out && !aligned(out[i], size_of(types_out[i])))) return bad(who, "a tensor is not aligned to its elements");
    }
    const int found = lay::clip_overlaps(grads, out, counts, dtypes, types_out, tensors, norm_in, norm, workspace);
    if (found < 0) {
        set_error("%s: no memory", who);
        return FFTCONV_ENOMEM;
    }
    if (found) return bad(who, "what is written (results, norm, workspace) overlaps something else");
    return lay::clip_grads(grads, out, counts, dtypes, types_out, tensors, max_norm, eps, norm_in, norm, workspace, (hipStream_t)stream);
}

}  // extern "C"
