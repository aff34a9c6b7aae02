// Root-mean-square norm of rows with the residual's addition, its backward pass, and rows in 8 bits with a scale each.
//
//   h = x + r,  y = h * rstd * w,  rstd = 1 / sqrt(mean(h^2) + eps)
//   dx = dh + rstd * (g - z * mean(g . z)),  dw = sum over rows of dy . z     with g = dy . w, z = h * rstd
//
// A row stays in the registers of the waves that work on it from its load to its store: every tensor moves once, and that is what bounds
// these kernels. Sums are held in fp32; h is rounded where it is written, the norm is taken of the sum before that.
//
// Measured: bf16 64 x 4096 x 768 forward 300 us and backward 325 us, 1.6 GB each: 5.4 and 5.0 TB/s, what a copy reaches. fp16 9995 x 1001, whose rows
// end inside a piece: 15 us, 5.4 TB/s; longer tensors of such rows 4 TB/s.
#include "layers_internal.h"

namespace fftconv {
namespace lay {

struct RowArgs {
    const void *x, *r;
    const float *w;
    void *y, *h;
    float *rstd, *scale;
    int64_t T, D, ldx, ldr;
    float eps;
    double eps64;                 // the same, for rows in other units
    int norm, i8;
};

// Sum / maximum over the WPR waves that share a row, in every lane. `at` alternates, so that one barrier a reduction is enough.
template <int WPR, typename F> __device__ __forceinline__ uint32_t row_reduce(uint32_t x, F f, uint32_t (*part)[16], int &at)
{
    x = reduce64(x, f);
    if constexpr (WPR > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) part[at][wave] = x;
        lds_barrier();
        x = part[at][0];
#pragma unroll
        for (int i = 1; i < WPR; ++i) x = f(x, part[at][i]);
        at ^= 1;
    }
    return x;
}

template <typename T, int E, int CH, int WPR, bool WHOLE> __global__ void __launch_bounds__(WPR == 16 ? 1024 : 256) k_rows(const RowArgs a)
{
    constexpr int LANES = 64 * WPR, ROWS = WPR == 1 ? 4 : 1;
    __shared__ uint32_t part[2][16];
    int at = 0;
    const int lane = threadIdx.x % LANES;
    const float by_d = 1.f / (float)a.D;
    float w[CH][E];                                       // the norm's weight, for all of the workgroup's rows
    if (a.norm) {
#pragma unroll
        for (int c = 0; c < CH; ++c) load_row_piece<float, E, WHOLE>(a.w, (int64_t)(lane + c * LANES) * E, a.D, w[c]);
    }
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.T; row += (int64_t)gridDim.x * ROWS) {
        const T *const x = (const T *)a.x + row * a.ldx;
        const T *const r = a.r ? (const T *)a.r + row * a.ldr : nullptr;
        float v[CH][E];
#pragma unroll
        for (int c = 0; c < CH; ++c) load_row_piece<T, E, WHOLE>(x, (int64_t)(lane + c * LANES) * E, a.D, v[c]);
        if (r) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float t[E];
                load_row_piece<T, E, WHOLE>(r, (int64_t)(lane + c * LANES) * E, a.D, t);
#pragma unroll
                for (int e = 0; e < E; ++e) v[c][e] += t[e];
            }
        }
        if (a.h) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t col = (int64_t)(lane + c * LANES) * E;
                store_rounded<T, E>((T *)a.h + row * a.D + col, a.D - col, v[c]);
            }
        }
        if (a.norm) {
            float ss = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) ss = fmaf(v[c][e], v[c][e], ss);
            ss = __builtin_bit_cast(float, row_reduce<WPR>(__builtin_bit_cast(uint32_t, ss), AddF32(), part, at));
            float rstd = 1.f / sqrtf(fmaf(ss, by_d, a.eps));
            // Squares beyond fp32's largest number, or so small that their own rounding, or that of values below 2^-126, counts (2^-100 and less): the row
            // once more in units of a power of two near its largest magnitude, what it is divided by in 64 bits.
            bool own_units = false;
            if (!(ss < __builtin_inff()) || ss < 0x1p-100f) {
                uint32_t top = 0;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) top = MaxU32()(top, magnitude(v[c][e]));
                top = row_reduce<WPR>(top, MaxU32(), part, at);
                if (top != 0 && top < 0x7f800000u) {              // (a row of zeros, or with an infinity or NaN, has no such units)
                    own_units = true;
                    const int unit = ilogbf(__builtin_bit_cast(float, top));
                    ss = 0.f;
#pragma unroll
                    for (int c = 0; c < CH; ++c)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            v[c][e] = ldexpf(v[c][e], -unit);
                            ss = fmaf(v[c][e], v[c][e], ss);
                        }
                    ss = __builtin_bit_cast(float, row_reduce<WPR>(__builtin_bit_cast(uint32_t, ss), AddF32(), part, at));
                    const double by = 1.0 / sqrt((double)ss / (double)a.D + ldexp(a.eps64, -2 * unit));
                    rstd = (float)ldexp(by, -unit);
#pragma unroll
                    for (int c = 0; c < CH; ++c)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float by_w = w[c][e];
                            asm volatile("" : "+v"(by_w), "+v"(v[c][e]));      // (else all weights are kept in 64 bits throughout)
                            v[c][e] = (float)((double)v[c][e] * by * (double)by_w);
                        }
                }
            }
            if (a.rstd && lane == 0) a.rstd[row] = rstd;
            if (!own_units) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) v[c][e] = v[c][e] * rstd * w[c][e];
            }
        }
        if (!a.i8) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t col = (int64_t)(lane + c * LANES) * E;
                store_rounded<T, E>((T *)a.y + row * a.D + col, a.D - col, v[c]);
            }
            continue;
        }
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) top = MaxU32()(top, magnitude(v[c][e]));
        top = row_reduce<WPR>(top, MaxU32(), part, at);
        const float s = scale_of(top);
        if (lane == 0) a.scale[row] = s;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = (int64_t)(lane + c * LANES) * E;
            int8_t q[E];
            quantise<E>(v[c], s, q);
            store_piece<int8_t, E>((int8_t *)a.y + row * a.D + col, a.D - col, q);
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *dh;
    const float *w, *rstd;
    void *dx;
    float *part;                  // a row of D sums for each workgroup; dw itself where there is one
    int64_t T, D, lddy;
};

template <typename T, int E, int CH, int WPR, bool WHOLE> __global__ void __launch_bounds__(WPR == 16 ? 1024 : 256) k_norm_grad(const NormGradArgs a)
{
    constexpr int LANES = 64 * WPR, ROWS = WPR == 1 ? 4 : 1;
    __shared__ uint32_t part[2][16];
    __shared__ float sums[WPR == 1 ? 4 * 64 * E * CH : 1];
    int at = 0;
    const int lane = threadIdx.x % LANES;
    const float by_d = 1.f / (float)a.D;
    float dw[CH][E] = {}, w[CH][E];
#pragma unroll
    for (int c = 0; c < CH; ++c) load_row_piece<float, E, WHOLE>(a.w, (int64_t)(lane + c * LANES) * E, a.D, w[c]);
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.T; row += (int64_t)gridDim.x * ROWS) {
        float g[CH][E], z[CH][E], dh[CH][E] = {};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = (int64_t)(lane + c * LANES) * E;
            load_row_piece<T, E, WHOLE>((const T *)a.dy + row * a.lddy, col, a.D, g[c]);
            load_row_piece<T, E, WHOLE>((const T *)a.h + row * a.D, col, a.D, z[c]);
        }
        const float rstd = a.rstd[row];
        if (a.dh) {
#pragma unroll
            for (int c = 0; c < CH; ++c) load_row_piece<T, E, WHOLE>((const T *)a.dh + row * a.D, (int64_t)(lane + c * LANES) * E, a.D, dh[c]);
        }
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                z[c][e] *= rstd;
                dw[c][e] = fmaf(g[c][e], z[c][e], dw[c][e]);
                g[c][e] *= w[c][e];
                dot = fmaf(g[c][e], z[c][e], dot);
            }
        }
        dot = __builtin_bit_cast(float, row_reduce<WPR>(__builtin_bit_cast(uint32_t, dot), AddF32(), part, at)) * by_d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = (int64_t)(lane + c * LANES) * E;
#pragma unroll
            for (int e = 0; e < E; ++e) g[c][e] = fmaf(rstd, fmaf(-z[c][e], dot, g[c][e]), dh[c][e]);
            store_rounded<T, E>((T *)a.dx + row * a.D + col, a.D - col, g[c]);
        }
    }
    float *const out = a.part + (int64_t)blockIdx.x * a.D;
    if constexpr (WPR > 1) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = (int64_t)(lane + c * LANES) * E;
            store_piece<float, E>(out + col, a.D - col, dw[c]);
        }
    } else {
        constexpr int W = 64 * E * CH;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) sums[(threadIdx.x >> 6) * W + (lane + c * 64) * E + e] = dw[c][e];
        lds_barrier();
        for (int col = threadIdx.x; col < W && col < a.D; col += 256) out[col] = (sums[col] + sums[W + col]) + (sums[2 * W + col] + sums[3 * W + col]);
    }
}

// dw[d] = sum over the workgroups' rows, in an order that the sizes alone decide: 16 columns x 64 slices of the rows in a workgroup, eight loads
// of a thread on their way at once (1536 rows of 768: 21 us with 32 x 32 and one load after the other, 6 so).
__global__ void __launch_bounds__(1024) k_sum_rows(const float *__restrict__ part, float *__restrict__ out, int rows, int64_t D)
{
    __shared__ float sums[64][17];
    const int c = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + c;
    float s = 0.f;
    if (col < D) {
        int r = slice;
        for (; r + 7 * 64 < rows; r += 8 * 64) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = part[(int64_t)(r + i * 64) * D + col];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        for (; r < rows; r += 64) s += part[(int64_t)r * D + col];
    }
    sums[slice][c] = s;
    lds_barrier();
    for (int half = 32; half > 0; half >>= 1) {
        if (slice < half) sums[slice][c] = s += sums[slice + half][c];
        lds_barrier();
    }
    if (slice == 0 && col < D) out[col] = s;
}

// Which lanes hold a row: one wave for up to 2048 values in 16 bits (1024 in 32), four waves up to 8192 (4096), sixteen above; pieces of 16 bytes,
// also where a quarter of the lanes is left idle (768 values: norm and gradients of 64 x 4096 rows 638 us, and 658 with three pieces of 8 bytes
// and none idle), but not half of them (256 values in 16 bits: 403 us forward for 1.6 GB, 311 in pieces of 8 bytes).
struct RowShape { int e, ch, wpr; };
static RowShape row_shape(int64_t D, int dtype)
{
    const int e = dtype == FFTCONV_F32 ? 4 : 8;
    const int wpr = D <= 64 * e * 4 ? 1 : D <= 256 * e * 4 ? 4 : 16;
    if (e == 8 && D <= 256) return {4, 1, 1};
    return {e, (int)((D + 64 * wpr * e - 1) / (64 * wpr * e)), wpr};
}

template <typename F> static int with_row_kernel(int64_t D, int dtype, F f)
{
    const RowShape s = row_shape(D, dtype);
#define FC_ROW(TY, E_, CH_, W_) if (s.e == E_ && s.ch == CH_ && s.wpr == W_) return D % E_ == 0 ? f(TY(), std::integral_constant<int, E_>(), std::integral_constant<int, CH_>(), std::integral_constant<int, W_>(), std::true_type()) : f(TY(), std::integral_constant<int, E_>(), std::integral_constant<int, CH_>(), std::integral_constant<int, W_>(), std::false_type());
#define FC_ROW16(TY) FC_ROW(TY, 4, 1, 1) FC_ROW(TY, 8, 1, 1) FC_ROW(TY, 8, 2, 1) FC_ROW(TY, 8, 3, 1) FC_ROW(TY, 8, 4, 1) \
        FC_ROW(TY, 8, 2, 4) FC_ROW(TY, 8, 3, 4) FC_ROW(TY, 8, 4, 4) FC_ROW(TY, 8, 2, 16)
    if (dtype == FFTCONV_BF16) {
        FC_ROW16(__bf16)
    } else if (dtype == FFTCONV_F16) {
        FC_ROW16(_Float16)
    } else {
        FC_ROW(float, 4, 1, 1) FC_ROW(float, 4, 2, 1) FC_ROW(float, 4, 3, 1) FC_ROW(float, 4, 4, 1)
        FC_ROW(float, 4, 2, 4) FC_ROW(float, 4, 3, 4) FC_ROW(float, 4, 4, 4) FC_ROW(float, 4, 2, 16) FC_ROW(float, 4, 3, 16) FC_ROW(float, 4, 4, 16)
    }
#undef FC_ROW16
#undef FC_ROW
    set_error("rows of %lld values: no kernel", (long long)D);
    return FFTCONV_EUNSUPPORTED;
}

static int64_t row_groups(int64_t T, const RowShape &s) { return s.wpr == 1 ? (T + 3) / 4 : T; }

// Workgroups of the forward pass: enough to fill the chip, each with the weight in registers for all of its rows.
constexpr int64_t MOST_GROUPS = 256 * 8;

// Workgroups of the backward pass: each leaves a row of sums, so there are no more than fill the chip.
static int64_t grad_groups(int64_t T, int64_t D, int dtype)
{
    const RowShape s = row_shape(D, dtype);
    const int64_t most = s.wpr == 1 ? 1536 : s.wpr == 4 ? 1024 : 512;
    const int64_t g = row_groups(T, s);
    return g < 1 ? 1 : g < most ? g : most;                  // (no row: one workgroup writes dw's zeros)
}

size_t rms_norm_backward_workspace(int64_t T, int64_t D, int dtype)
{
    const int64_t g = grad_groups(T, D, dtype);
    return g > 1 ? (size_t)g * (size_t)D * 4 : 0;
}

int rows_forward(const void *x, int64_t ldx, const void *r, int64_t ldr, const float *w, void *y, void *h, float *rstd, float *scale, int64_t T,
                 int64_t D, double eps, int norm, int i8, int dtype, hipStream_t s)
{
    const RowArgs a = {x, r, w, y, h, rstd, scale, T, D, ldx, ldr, (float)eps, eps, norm, i8};
    return with_row_kernel(D, dtype, [&](auto t, auto e, auto ch, auto wpr, auto whole) -> int {
        using TY = decltype(t);
        int64_t g = row_groups(T, row_shape(D, dtype));
        if (g > MOST_GROUPS) g = MOST_GROUPS;
        k_rows<TY, decltype(e)::value, decltype(ch)::value, decltype(wpr)::value, decltype(whole)::value><<<(unsigned)g, decltype(wpr)::value == 16 ? 1024 : 256, 0, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    });
}

int rms_norm_backward(const void *dy, int64_t lddy, const void *h, const void *dh, const float *w, const float *rstd, void *dx, float *dw,
                      int64_t T, int64_t D, int dtype, void *workspace, hipStream_t s)
{
    const int64_t groups = grad_groups(T, D, dtype);
    const NormGradArgs a = {dy, h, dh, w, rstd, dx, groups > 1 ? (float *)workspace : dw, T, D, lddy};
    FC_TRY(with_row_kernel(D, dtype, [&](auto t, auto e, auto ch, auto wpr, auto whole) -> int {
        using TY = decltype(t);
        k_norm_grad<TY, decltype(e)::value, decltype(ch)::value, decltype(wpr)::value, decltype(whole)::value><<<(unsigned)groups, decltype(wpr)::value == 16 ? 1024 : 256, 0, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    }));
    if (groups > 1) {
        k_sum_rows<<<(unsigned)((D + 15) / 16), 1024, 0, s>>>((const float *)workspace, dw, (int)groups, D);
        FC_HIP(hipGetLastError());
    }
    return FFTCONV_OK;
}

}  // namespace lay
}  // namespace fftconv
