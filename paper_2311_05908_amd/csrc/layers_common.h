// What the kernels around the convolutions share (row_norm.hip, linear_i8.hip, checkpoint.hip, weight_grad.hip): I/O types, loads and
// stores of any alignment, reductions over a wave.
#pragma once

#include "fftconv_internal.h"

namespace fftconv {
namespace lay {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

// Rows and runs whose largest magnitude is below 2^-100 are zeros with a scale of zero: their scale would come near the subnormal
// numbers, where its own rounding is no longer small.
constexpr float LEAST = 0x1p-100f;
constexpr int RUN = 128;                                      // samples of a channel that share a scale in a checkpoint

template <typename T> __device__ __forceinline__ float to_f32(T x) { return (float)x; }
template <typename T> __device__ __forceinline__ T from_f32(float x) { return (T)x; }      // round to nearest even

// N bytes at any alignment, as one access where N is 16, 8 or 4. (A copy of as many bytes from an array of 16-bit values comes out as one of twelve
// and one of four: rows of 2048 in bf16 3.9 TB/s instead of 5.)
typedef uint32_t any16 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t any8 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t any4 __attribute__((aligned(1)));
template <int N> struct Bytes { typedef any4 type; };
template <> struct Bytes<16> { typedef any16 type; };
template <> struct Bytes<8> { typedef any8 type; };
template <int N> __device__ __forceinline__ void load_bytes(const void *p, void *to)
{
    if constexpr (N > 16) {
        load_bytes<16>(p, to);
        load_bytes<N - 16>((const char *)p + 16, (char *)to + 16);
    } else {
        static_assert(N == 16 || N == 8 || N == 4, "piece");
        const typename Bytes<N>::type v = *(const typename Bytes<N>::type *)p;
        __builtin_memcpy(to, &v, N);
    }
}
template <int N> __device__ __forceinline__ void store_bytes(void *p, const void *from)
{
    if constexpr (N > 16) {
        store_bytes<16>(p, from);
        store_bytes<N - 16>((char *)p + 16, (const char *)from + 16);
    } else {
        static_assert(N == 16 || N == 8 || N == 4, "piece");
        typename Bytes<N>::type v;
        __builtin_memcpy(&v, from, N);
        *(typename Bytes<N>::type *)p = v;
    }
}

// E values from p, of which the first `left` are there (the others read as zero). A whole piece is one load of E * sizeof(T) bytes at any
// alignment of T.
template <typename T, int E> __device__ __forceinline__ void load_piece(const T *p, int64_t left, float (&v)[E])
{
    if (left >= E) {
        T raw[E];
        load_bytes<E * (int)sizeof(T)>(p, raw);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = to_f32(raw[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = e < left ? to_f32(p[e]) : 0.f;
    }
}

template <typename T, int E> __device__ __forceinline__ void store_piece(T *p, int64_t left, const T (&raw)[E])
{
    if (left >= E) {
        store_bytes<E * (int)sizeof(T)>(p, raw);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < left) p[e] = raw[e];
    }
}

template <typename T, int E> __device__ __forceinline__ void store_rounded(T *p, int64_t left, const float (&v)[E])
{
    T raw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) raw[e] = from_f32<T>(v[e]);
    store_piece<T, E>(p, left, raw);
}

// The same for rows whose length is a multiple of E: a piece is there or not (`left` is then 0 or below). One that is not is read at `row`'s beginning
// and set to zero: no branch parts the loads, so all of a row's are on their way together.
template <typename T, int E, bool WHOLE> __device__ __forceinline__ void load_row_piece(const T *row, int64_t col, int64_t D, float (&v)[E])
{
    if constexpr (WHOLE) {
        const bool there = col < D;
        T raw[E];
        load_bytes<E * (int)sizeof(T)>(row + (there ? col : 0), raw);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = there ? to_f32(raw[e]) : 0.f;
    } else {
        load_piece<T, E>(row + col, D - col, v);
    }
}

// A magnitude as an integer: of two, the larger number is the larger integer, infinities are above every finite number and NaN above
// infinities, so the largest of a row says whether anything in it is not finite.
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Reduction over groups of 16 lanes, or over the wave, every lane ending with the result: exchanges inside the vector unit (lane pairs, quads,
// half rows and rows of 16, then rows and halves of the wave swapped), no trip through LDS. The order of the additions is fixed.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <typename F> __device__ __forceinline__ uint32_t reduce16(uint32_t x, F f)
{
    x = f(x, dpp<0xB1>(x));       // lanes ^ 1
    x = f(x, dpp<0x4E>(x));       // lanes ^ 2
    x = f(x, dpp<0x141>(x));      // the other quad of the half row
    x = f(x, dpp<0x140>(x));      // the other half of the row
    return x;
}
template <typename F> __device__ __forceinline__ uint32_t reduce64(uint32_t x, F f)
{
    x = reduce16(x, f);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(r[0], r[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return f(h[0], h[1]);
}
struct AddF32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const
    {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
    }
};
struct MaxU32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
__device__ __forceinline__ float wave_sum(float x) { return __builtin_bit_cast(float, reduce64(__builtin_bit_cast(uint32_t, x), AddF32())); }
__device__ __forceinline__ uint32_t wave_max(uint32_t x) { return reduce64(x, MaxU32()); }

// Scale of values whose largest magnitude has these bits: max / 127; zero for values below LEAST; NaN where a value is not finite, so that
// nothing read back from 8 bits passes for a number that was there.
__device__ __forceinline__ float scale_of(uint32_t top)
{
    const float m = __builtin_bit_cast(float, top);
    return top >= 0x7f800000u ? __builtin_nanf("") : m < LEAST ? 0.f : m / 127.f;
}
// q = x / s rounded to the nearest integer, ties to even; the quotient is rounded as IEEE 754 has it, so that q is a function of x and s alone.
// Zero where the scale is zero or NaN.
__device__ __forceinline__ int8_t quantised(float x, float s) { return s > 0.f ? (int8_t)(int)rintf(x / s) : (int8_t)0; }

// The same for E values (4 or 8) of one scale. |x / s| is at most 127 and a bit, so x (1 / s), not rounded before 1.5 2^23 is added, is within
// 127 2^-24 of the quotient: its nearest integer, which that sum holds in its lowest bits, is the quotient's unless it lies within 2^-14 of a tie.
// Only there the quotient itself is taken (a wave in sixteen or so for eight values a lane): five instructions a value instead of fifteen.
template <int E> __device__ __forceinline__ void quantise(const float (&x)[E], float s, int8_t (&q)[E])
{
    constexpr float SHIFT = 12582912.f;
    const float by = s > 0.f ? 1.f / s : 0.f;
    float u[E], off = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        u[e] = fmaf(x[e], by, SHIFT);
        off = fmaxf(off, fabsf(fmaf(x[e], by, SHIFT - u[e])));
    }
    if (__builtin_amdgcn_ballot_w64(!(off < 0.5f - 0x1p-14f && s > 0.f)) != 0) {        // (or where there is no scale)
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = quantised(x[e], s);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = (int8_t)(uint8_t)__builtin_bit_cast(uint32_t, u[e]);
    }
}

}  // namespace lay
}  // namespace fftconv
