// Activations kept for the backward pass in 8 bits: (B, C, N) with a scale for every 128 samples of a channel, and back.
//
//   s[b, c, j] = max |x[b, c, n]| / 127 over the run n = 128 j ... 128 j + 127,  q = round(x / s)
//   x^ = q s, or the product of two such with one rounding at the end (u . w, as the gradient of a gated convolution's filter takes it)
//
// Runs lie along the samples because that is the direction every gradient here sums over (a filter's, a projection's): within a run
// the scale comes out of the sum. Bound by the bytes moved.
#include "layers_internal.h"

namespace fftconv {
namespace lay {

// A run is 16 lanes of 8 values: one piece a lane, the largest magnitude from exchanges inside a row of 16 lanes.
template <typename T> __global__ void __launch_bounds__(256) k_pack(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale,
                                                                     int64_t total, int64_t runs, int64_t N)
{
    const int l = threadIdx.x & 15;
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < total; i += (int64_t)gridDim.x * 16) {
        const int64_t row = i / runs, n = (i - row * runs) * RUN + l * 8, left = N - n;
        float v[8];
        load_piece<T, 8>(x + row * N + n, left, v);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = MaxU32()(top, magnitude(v[e]));
        const float s = scale_of(reduce16(top, MaxU32()));
        int8_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = quantised(v[e], s);
        store_piece<int8_t, 8>(q + row * N + n, left, o);
        if (l == 0) scale[i] = s;
    }
}

// The same from (B, N, C): a workgroup takes one run of 64 channels and turns it over in LDS. Thread t reads 8 channels (t % 8) of the
// samples t / 8, t / 8 + 32, ...; the largest magnitude of a channel is taken over its four samples, then over the 32 threads of that piece.
template <typename T> __global__ void __launch_bounds__(256) k_pack_tokens(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale,
                                                                            int64_t C, int64_t N, int64_t runs, int64_t cgroups, int64_t total)
{
    __shared__ uint32_t tops[64];
    __shared__ uint32_t tile[64][RUN / 4 + 1];                 // [channel][samples, four to a word]
    for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
        const int64_t cg = w % cgroups, j = w / cgroups % runs, b = w / (cgroups * runs);
        const int64_t c0 = cg * 64 + (threadIdx.x & 7) * 8, n0 = j * RUN + (threadIdx.x >> 3) * 4;
        float v[4][8];
        if (threadIdx.x < 64) tops[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) load_piece<T, 8>(x + (b * N + n0 + i) * C + c0, n0 + i < N ? C - c0 : 0, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = MaxU32()(top, magnitude(v[i][e]));
            atomicMax(&tops[(threadIdx.x & 7) * 8 + e], top);  // (a maximum: no order of the threads changes it)
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = (threadIdx.x & 7) * 8 + e;
            const float s = scale_of(tops[c]);
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) word |= (uint32_t)(uint8_t)quantised(v[i][e], s) << (8 * i);
            tile[c][threadIdx.x >> 3] = word;
        }
        __syncthreads();
        if (threadIdx.x < 64 && cg * 64 + threadIdx.x < C) scale[(b * C + cg * 64 + threadIdx.x) * runs + j] = scale_of(tops[threadIdx.x]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = (threadIdx.x >> 3) + 32 * i, piece = threadIdx.x & 7;
            const int64_t left = N - j * RUN - piece * 16;
            if (cg * 64 + c < C && left > 0) {
                uint32_t words[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) words[k] = tile[c][piece * 4 + k];
                int8_t o[16];
                __builtin_memcpy(o, words, 16);
                store_piece<int8_t, 16>(q + (b * C + cg * 64 + c) * N + j * RUN + piece * 16, left, o);
            }
        }
        __syncthreads();
    }
}

template <typename T> __global__ void __launch_bounds__(256) k_unpack(const int8_t *__restrict__ q, const float *__restrict__ scale,
                                                                       const int8_t *__restrict__ gq, const float *__restrict__ gscale,
                                                                       const T *__restrict__ gate, T *__restrict__ x, int64_t total, int64_t runs,
                                                                       int64_t N)
{
    const int l = threadIdx.x & 15;
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < total; i += (int64_t)gridDim.x * 16) {
        const int64_t row = i / runs, n = (i - row * runs) * RUN + l * 8, left = N - n, at = row * N + n;
        float v[8], g[8];
        load_piece<int8_t, 8>(q + at, left, v);
        const float s = scale[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= s;
        if (gq) {
            load_piece<int8_t, 8>(gq + at, left, g);
            const float gs = gscale[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= g[e] * gs;
        } else if (gate) {
            load_piece<T, 8>(gate + at, left, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= g[e];
        }
        store_rounded<T, 8>(x + at, left, v);
    }
}

template <typename F> static int with_type(int dtype, F f)
{
    if (dtype == FFTCONV_BF16) return f(__bf16());
    if (dtype == FFTCONV_F16) return f(_Float16());
    return f(float());
}

static unsigned groups_of(int64_t n) { return (unsigned)(n < ((int64_t)1 << 30) ? n : (int64_t)1 << 30); }

int act_pack(const void *x, int8_t *q, float *scale, int64_t B, int64_t C, int64_t N, bool tokens, int dtype, hipStream_t s)
{
    const int64_t runs = (N + RUN - 1) / RUN;
    return with_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        if (tokens) {
            const int64_t cg = (C + 63) / 64, total = B * runs * cg;
            k_pack_tokens<T><<<groups_of(total), 256, 0, s>>>((const T *)x, q, scale, C, N, runs, cg, total);
        } else {
            const int64_t total = B * C * runs;
            k_pack<T><<<groups_of((total + 15) / 16), 256, 0, s>>>((const T *)x, q, scale, total, runs, N);
        }
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    });
}

int act_unpack(const int8_t *q, const float *scale, const int8_t *gq, const float *gscale, const void *gate, void *x, int64_t B, int64_t C,
               int64_t N, int dtype, hipStream_t s)
{
    const int64_t runs = (N + RUN - 1) / RUN, total = B * C * runs;
    return with_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        k_unpack<T><<<groups_of((total + 15) / 16), 256, 0, s>>>(q, scale, gq, gscale, (const T *)gate, (T *)x, total, runs, N);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    });
}

}  // namespace lay
}  // namespace fftconv
