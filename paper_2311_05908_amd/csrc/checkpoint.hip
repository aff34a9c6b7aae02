// Activations kept for the backward pass in 8 bits: (B, C, N) with a scale for every 128 samples of a channel, and back.
//
//   s[b, c, j] = max |x[b, c, n]| / 127 over the run n = 128 j ... 128 j + 127,  q = round(x / s)
//   x^ = q s, or the product of two such, in fp32, rounded to its type at the end (u . w, as the gradient of a gated convolution's filter takes it)
//
// Runs lie along the samples because that is the direction every gradient here sums over (a filter's, a projection's): within a run
// the scale comes out of the sum. Bound by the bytes moved: bf16 64 x 768 x 4096 packed in 129 us (4.7 TB/s), read back as a product in 129 us (6.2).
#include "layers_index.h"
#include "layers_internal.h"

namespace fftconv {
namespace lay {

// A run is 16 lanes of 8 values: one piece a lane, the largest magnitude from exchanges inside a row of 16 lanes. A workgroup takes 16 R runs, each
// lane R pieces at once. WHOLE: samples in runs, so that a tensor is one long row and nothing has to be divided.
template <typename T, bool WHOLE> __device__ __forceinline__ bool run_at(int64_t i, int64_t total, int64_t runs, int64_t N, int64_t &at, int64_t &left)
{
    const int l = threadIdx.x & 15;
    if (WHOLE) {
        at = i * RUN + l * 8, left = RUN;
    } else {
        const int64_t row = i / runs, n = (i - row * runs) * RUN + l * 8;
        at = row * N + n, left = N - n;
    }
    return i < total;
}

template <typename T, bool WHOLE> __global__ void __launch_bounds__(256) k_pack(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale,
                                                                                int64_t first, int64_t total, int64_t runs, int64_t N)
{
    constexpr int R = 2;
    const int64_t i0 = (first + blockIdx.x) * (16 * R) + (threadIdx.x >> 4);
    float v[R][8];
    int64_t at[R], left[R];
    bool there[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        there[r] = run_at<T, WHOLE>(i0 + r * 16, total, runs, N, at[r], left[r]);
        load_piece<T, 8>(x + at[r], there[r] ? left[r] : 0, v[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = MaxU32()(top, magnitude(v[r][e]));
        const float s = scale_of(reduce16(top, MaxU32()));
        int8_t o[8];
        quantise<8>(v[r], s, o);
        store_piece<int8_t, 8>(q + at[r], there[r] ? left[r] : 0, o);
        if (there[r] && (threadIdx.x & 15) == 0) scale[i0 + r * 16] = s;
    }
}

// The same from (B, N, C): a workgroup takes one run of 64 channels and turns it over in LDS. Thread t reads 8 channels (t % 8) of the four samples
// 4 (t / 8) ...; the largest magnitude of a channel is taken over its four samples, over the eight threads of the wave with the same channels by
// exchanges, and over the four waves by way of LDS. bf16 64 x 4096 x 768, three tensors in turn: 167 us, 3.6 TB/s, where
// k_pack takes 131: the steps of a workgroup follow each other.
template <typename T> __global__ void __launch_bounds__(256) k_pack_tokens(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale,
                                                                            int64_t C, int64_t N, uint32_t runs, uint32_t cgroups, uint32_t first)
{
    __shared__ __align__(16) uint32_t tops[4][64];
    __shared__ uint32_t tile[64][RUN / 4 + 1];                 // [channel][samples, four to a word]
    const int piece8 = threadIdx.x & 7, lane = threadIdx.x & 63;
    const uint32_t i = first + blockIdx.x, at = i / cgroups;      // (numbers of 32 bits: a division of 64 takes a tenth of a workgroup's time)
    const int64_t cg = i - at * cgroups, j = at % runs, b = at / runs;
    const int64_t c0 = cg * 64 + piece8 * 8, n0 = j * RUN + (threadIdx.x >> 3) * 4;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) load_piece<T, 8>(x + (b * N + n0 + i) * C + c0, n0 + i < N ? C - c0 : 0, v[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const MaxU32 most;
        uint32_t top = most(most(magnitude(v[0][e]), magnitude(v[1][e])), most(magnitude(v[2][e]), magnitude(v[3][e])));
        top = most(top, dpp<0x128>(top));                  // lanes ^ 8
        const auto r = __builtin_amdgcn_permlane16_swap(top, top, false, false);
        top = most(r[0], r[1]);
        const auto h = __builtin_amdgcn_permlane32_swap(top, top, false, false);
        if (lane < 8) tops[threadIdx.x >> 6][piece8 * 8 + e] = most(h[0], h[1]);
    }
    lds_barrier();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = piece8 * 8 + e;
        const MaxU32 most;
        const float s = scale_of(most(most(tops[0][c], tops[1][c]), most(tops[2][c], tops[3][c])));
        const float x4[4] = {v[0][e], v[1][e], v[2][e], v[3][e]};
        int8_t q4[4];
        quantise<4>(x4, s, q4);
        uint32_t word;
        __builtin_memcpy(&word, q4, 4);
        tile[c][threadIdx.x >> 3] = word;
        if (threadIdx.x < 8 && cg * 64 + c < C) scale[(b * C + cg * 64 + c) * runs + j] = s;
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (threadIdx.x >> 3) + 32 * i;
        const int64_t left = N - j * RUN - piece8 * 16;
        if (cg * 64 + c < C && left > 0) {
            uint32_t words[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) words[k] = tile[c][piece8 * 4 + k];
            int8_t o[16];
            __builtin_memcpy(o, words, 16);
            store_piece<int8_t, 16>(q + (b * C + cg * 64 + c) * N + j * RUN + piece8 * 16, left, o);
        }
    }
}

template <typename T, bool WHOLE> __global__ void __launch_bounds__(256) k_unpack(const int8_t *__restrict__ q, const float *__restrict__ scale,
                                                                                  const int8_t *__restrict__ gq, const float *__restrict__ gscale,
                                                                                  const T *__restrict__ gate, T *__restrict__ x, int64_t first,
                                                                                  int64_t total, int64_t runs, int64_t N)
{
    constexpr int R = 2;
    const int64_t i0 = (first + blockIdx.x) * (16 * R) + (threadIdx.x >> 4);
    float v[R][8], g[R][8], s[R], gs[R];
    int64_t at[R], left[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t i = i0 + r * 16;
        const bool there = run_at<T, WHOLE>(i, total, runs, N, at[r], left[r]);
        left[r] = there ? left[r] : 0;
        load_piece<int8_t, 8>(q + at[r], left[r], v[r]);
        s[r] = there ? scale[i] : 0.f;
        gs[r] = there && gq ? gscale[i] : 1.f;
        if (gq) load_piece<int8_t, 8>(gq + at[r], left[r], g[r]);
        else if (gate) load_piece<T, 8>(gate + at[r], left[r], g[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[r][e] *= s[r];
        if (gq || gate) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[r][e] *= g[r][e] * gs[r];
        }
        store_rounded<T, 8>(x + at[r], left[r], v[r]);
    }
}

template <typename F> static int with_type(int dtype, F f)
{
    if (dtype == FFTCONV_BF16) return f(__bf16());
    if (dtype == FFTCONV_F16) return f(_Float16());
    return f(float());
}

int act_pack(const void *x, int8_t *q, float *scale, int64_t B, int64_t C, int64_t N, bool tokens, int dtype, hipStream_t s)
{
    const int64_t runs = (N + RUN - 1) / RUN;
    return with_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        if (tokens) {
            const int64_t cg = (C + 63) / 64, total = B * runs * cg;
            if (total > INT32_MAX) {
                set_error("fftconv_act_pack: %lld tiles of 64 channels x 128 samples: up to 2^31 - 1 are supported", (long long)total);
                return FFTCONV_EUNSUPPORTED;
            }
            return in_pieces(total, 256, [&](int64_t first, unsigned g) -> int {
                k_pack_tokens<T><<<g, 256, 0, s>>>((const T *)x, q, scale, C, N, (uint32_t)runs, (uint32_t)cg, (uint32_t)first);
                FC_HIP(hipGetLastError());
                return FFTCONV_OK;
            });
        }
        const int64_t total = B * C * runs;
        return in_pieces((total + 31) / 32, 256, [&](int64_t first, unsigned g) -> int {
            if (N % RUN == 0) k_pack<T, true><<<g, 256, 0, s>>>((const T *)x, q, scale, first, total, runs, N);
            else k_pack<T, false><<<g, 256, 0, s>>>((const T *)x, q, scale, first, total, runs, N);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    });
}

int act_unpack(const int8_t *q, const float *scale, const int8_t *gq, const float *gscale, const void *gate, void *x, int64_t B, int64_t C,
               int64_t N, int dtype, hipStream_t s)
{
    const int64_t runs = (N + RUN - 1) / RUN, total = B * C * runs;
    return with_type(dtype, [&](auto t) -> int {
        using T = decltype(t);
        return in_pieces((total + 31) / 32, 256, [&](int64_t first, unsigned g) -> int {
            if (N % RUN == 0) k_unpack<T, true><<<g, 256, 0, s>>>(q, scale, gq, gscale, (const T *)gate, (T *)x, first, total, runs, N);
            else k_unpack<T, false><<<g, 256, 0, s>>>(q, scale, gq, gscale, (const T *)gate, (T *)x, first, total, runs, N);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    });
}

}  // namespace lay
}  // namespace fftconv
