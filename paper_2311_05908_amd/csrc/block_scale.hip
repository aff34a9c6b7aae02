// Rows and weights in 8-bit floating point (e4m3) with a scale for each block: 1 x 128 of a row, 128 x 128 of a weight.
//
//   s = max |x| / 448 over the block,  q = x / s rounded to e4m3, to nearest even
//
// A block stays in registers from its load to its store, so the bytes bound these kernels; what is turned over on the way (rows from tensors that
// lie channel by channel, a weight's transpose) goes through LDS as bytes. Measured: fp32 16384 x 4096 with its transpose 82 us, 4.9 TB/s; bf16 3 x 64 x 768
// x 4096 to rows of 2304 340 us, 5.4 TB/s; f16 8192 x 4096 25 us, 4 TB/s; one row 3.4 us, of which the launch is most.
#include "layers_index.h"
#include "layers_internal.h"

namespace fftconv {
namespace lay {

constexpr int KB = 128;                     // values that share a scale

// A block's scale, and what its quotients are made with. The quotient is the one that IEEE 754 rounds, so that q is a function of the values alone:
// from the correctly rounded reciprocal, the product and its remainder give it in three operations, where nothing on the way leaves fp32's
// normal numbers; below 2^-64 the division itself is taken.
struct Scale {
    float s, by;
};
__device__ __forceinline__ Scale block_scale(uint32_t top)
{
    const float m = __builtin_bit_cast(float, top);
    Scale c;
    c.s = top >= 0x7f800000u ? __builtin_nanf("") : m < LEAST ? 0.f : m / 448.f;
    c.by = c.s > 0.f ? 1.f / c.s : 0.f;      // 0: no scale, or none that is a number: q is 0
    return c;
}
__device__ __forceinline__ float quotient_of(float x, Scale c)
{
    if (!(c.by > 0.f)) return 0.f;
    if (c.s < 0x1p-64f) return x / c.s;
    const float v = x * c.by;
    return fmaf(fmaf(-v, c.s, x), c.by, v);
}
// four values as bytes of a word
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

struct BlockArgs {
    const void *x;
    uint8_t *q;
    float *scale;                 // (blocks, T): block j of row i at j T + i
    int64_t T, K, ldx, first;
    int blocks, row_bits;         // rows of a workgroup: 2^row_bits
    int64_t wgs_k;                // workgroups along a row
    // from channels
    int64_t B, N;
    int per_part, tiles_n;
};

// Rows as they are: sixteen lanes to a block, eight values each; a workgroup takes 16 rows, four blocks of each one after the other, so that the 16
// scales of a block's are one piece of memory. (Few rows: sixteen blocks side by side.)
template <typename T> __global__ void __launch_bounds__(256) k_blocks(const BlockArgs a)
{
    const int64_t wg = a.first + blockIdx.x, wr = wg / a.wgs_k;
    const int group = threadIdx.x >> 4, l = threadIdx.x & 15;
    const int64_t row = (wr << a.row_bits) + (group & ((1 << a.row_bits) - 1));
    const int across = 16 >> a.row_bits, j0 = (int)(wg - wr * a.wgs_k) * 4 * across + (group >> a.row_bits);
    if (row >= a.T) return;
    const T *const x = (const T *)a.x + row * a.ldx;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t k = (int64_t)(j0 + i * across) * KB + l * 8;
        load_piece<T, 8>(x + k, a.K - k, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + i * across;
        if (j >= a.blocks) return;                               // (a block's sixteen lanes together)
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = MaxU32()(top, magnitude(v[i][e]));
        const Scale c = block_scale(reduce16(top, MaxU32()));
        if (l == 0) a.scale[(int64_t)j * a.T + row] = c.s;
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = quotient_of(v[i][e], c);
        const uint32_t w[2] = {to_e4m3(o[0], o[1], o[2], o[3]), to_e4m3(o[4], o[5], o[6], o[7])};
        uint8_t bytes[8];
        __builtin_memcpy(bytes, w, 8);
        const int64_t k = (int64_t)j * KB + l * 8;
        store_piece<uint8_t, 8>(a.q + row * a.K + k, a.K - k, bytes);
    }
}

// Rows from x (parts, B, K / parts, N): row (b, n) holds the sample n of every channel, part after part. A workgroup turns 128 channels of 64 samples
// over; a thread holds four channels of eight samples.
template <typename T> __global__ void __launch_bounds__(256) k_blocks_channels(const BlockArgs a)
{
    constexpr int STRIDE = 33;                                   // words of a sample's 128 bytes in LDS, moved on by a bank
    __shared__ uint32_t tops[4][64];
    __shared__ __align__(16) float scales[4][2][64];
    __shared__ uint32_t bytes[64 * STRIDE];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n8 = threadIdx.x & 7, c4 = threadIdx.x >> 3;
    int64_t wg = a.first + blockIdx.x;
    const int64_t per_b = (int64_t)a.blocks * a.tiles_n, b = wg / per_b;
    wg -= b * per_b;
    const int j = (int)(wg / a.tiles_n);
    const int64_t n0 = (wg - (int64_t)j * a.tiles_n) * 64;
    float v[4][8];
    int64_t part = ((int64_t)j * KB + 4 * c4) / a.per_part, within = (int64_t)j * KB + 4 * c4 - part * a.per_part;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool there = (int64_t)j * KB + 4 * c4 + i < a.K;
        const T *const x = (const T *)a.x + (there ? ((part * a.B + b) * a.per_part + within) * a.N : 0);
        load_piece<T, 8>(x + n0 + 8 * n8, there ? a.N - n0 - 8 * n8 : 0, v[i]);
        if (++within == a.per_part) within = 0, ++part;
    }
    uint32_t top[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        top[e] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top[e] = MaxU32()(top[e], magnitude(v[i][e]));
        top[e] = MaxU32()(top[e], dpp<0x128>(top[e]));           // lanes eight apart: the same samples
        const auto r = __builtin_amdgcn_permlane16_swap(top[e], top[e], false, false);
        top[e] = MaxU32()(r[0], r[1]);
        const auto h = __builtin_amdgcn_permlane32_swap(top[e], top[e], false, false);
        top[e] = MaxU32()(h[0], h[1]);
        if (lane < 8) tops[wave][8 * n8 + e] = top[e];
    }
    __syncthreads();
    {
        // a lane for a sample: the scale, and the reciprocal, in every wave
        uint32_t t = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) t = MaxU32()(t, tops[w][lane]);
        const Scale c = block_scale(t);
        scales[wave][0][lane] = c.s, scales[wave][1][lane] = c.by;
        if (wave == 0 && n0 + lane < a.N) a.scale[(int64_t)j * a.T + b * a.N + n0 + lane] = c.s;
    }
    __syncthreads();
    float s[8], by[8];
    __builtin_memcpy(s, &scales[wave][0][8 * n8], 32);
    __builtin_memcpy(by, &scales[wave][1][8 * n8], 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const Scale c = {s[e], by[e]};
        bytes[(8 * n8 + e) * STRIDE + c4] = to_e4m3(quotient_of(v[0][e], c), quotient_of(v[1][e], c), quotient_of(v[2][e], c), quotient_of(v[3][e], c));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int n = (threadIdx.x >> 3) + 32 * i, piece = threadIdx.x & 7;
        if (n0 + n >= a.N) continue;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = bytes[n * STRIDE + piece * 4 + e];
        uint8_t o[16];
        __builtin_memcpy(o, w, 16);
        const int64_t k = (int64_t)j * KB + piece * 16;
        store_piece<uint8_t, 16>(a.q + (b * a.N + n0 + n) * a.K + k, a.K - k, o);
    }
}

struct TileArgs {
    const void *x;
    uint8_t *q, *qt;
    float *scale, *scale_t;       // (tiles of O, tiles of K), (tiles of K, tiles of O)
    int64_t O, K, ldx, first;
    int tiles_o, tiles_k;
};

// A weight: a workgroup to a tile of 128 x 128, eight rows of eight values to a thread.
template <typename T> __global__ void __launch_bounds__(256) k_tiles(const TileArgs a)
{
    constexpr int STRIDE = 33;
    __shared__ uint32_t tops[4];
    __shared__ uint32_t bytes[KB * STRIDE];
    const int64_t wg = a.first + blockIdx.x;
    const int to = (int)(wg / a.tiles_k), tk = (int)(wg - (int64_t)to * a.tiles_k);
    const int i8 = threadIdx.x >> 4, j8 = threadIdx.x & 15;
    const int64_t o0 = (int64_t)to * KB + 8 * i8, k0 = (int64_t)tk * KB + 8 * j8;
    float v[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const bool there = o0 + r < a.O;
        load_piece<T, 8>((const T *)a.x + (there ? (o0 + r) * a.ldx + k0 : 0), there ? a.K - k0 : 0, v[r]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = MaxU32()(top, magnitude(v[r][e]));
    }
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) top = MaxU32()(top, tops[w]);
    const Scale c = block_scale(top);
    if (threadIdx.x == 0) {
        if (a.q) a.scale[(int64_t)to * a.tiles_k + tk] = c.s;
        if (a.qt) a.scale_t[(int64_t)tk * a.tiles_o + to] = c.s;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[r][e] = quotient_of(v[r][e], c);
    if (a.q) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint32_t w[2] = {to_e4m3(v[r][0], v[r][1], v[r][2], v[r][3]), to_e4m3(v[r][4], v[r][5], v[r][6], v[r][7])};
            uint8_t o[8];
            __builtin_memcpy(o, w, 8);
            if (o0 + r < a.O) store_piece<uint8_t, 8>(a.q + (o0 + r) * a.K + k0, a.K - k0, o);
        }
    }
    if (!a.qt) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        bytes[(8 * j8 + e) * STRIDE + 2 * i8] = to_e4m3(v[0][e], v[1][e], v[2][e], v[3][e]);
        bytes[(8 * j8 + e) * STRIDE + 2 * i8 + 1] = to_e4m3(v[4][e], v[5][e], v[6][e], v[7][e]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = (threadIdx.x >> 3) + 32 * i, piece = threadIdx.x & 7;
        const int64_t k = (int64_t)tk * KB + col, o = (int64_t)to * KB + piece * 16;
        if (k >= a.K) continue;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = bytes[col * STRIDE + piece * 4 + e];
        uint8_t out[16];
        __builtin_memcpy(out, w, 16);
        store_piece<uint8_t, 16>(a.qt + k * a.O + o, a.O - o, out);
    }
}

template <typename A, typename K> static int launch(A &a, int64_t groups, K kernel, hipStream_t s)
{
    return in_pieces(groups, 256, [&](int64_t first, unsigned n) -> int {
        a.first = first;
        kernel<<<n, 256, 0, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    });
}

int quantize_blocks(const void *x, int64_t ldx, uint8_t *q, float *scale, int64_t T, int64_t K, int dtype, hipStream_t s)
{
    BlockArgs a = {};
    a.x = x, a.q = q, a.scale = scale, a.T = T, a.K = K, a.ldx = ldx, a.blocks = (int)((K + KB - 1) / KB);
    a.row_bits = T >= 16 ? 4 : 0;
    const int across = 4 * (16 >> a.row_bits);
    a.wgs_k = (a.blocks + across - 1) / across;
    const int64_t groups = ((T + (1 << a.row_bits) - 1) >> a.row_bits) * a.wgs_k;
    return dtype == FFTCONV_BF16 ? launch(a, groups, k_blocks<__bf16>, s) : dtype == FFTCONV_F16 ? launch(a, groups, k_blocks<_Float16>, s) : launch(a, groups, k_blocks<float>, s);
}

int quantize_blocks_channels(const void *x, uint8_t *q, float *scale, int64_t B, int64_t N, int64_t K, int64_t parts, int dtype, hipStream_t s)
{
    BlockArgs a = {};
    a.x = x, a.q = q, a.scale = scale, a.T = B * N, a.K = K, a.B = B, a.N = N, a.blocks = (int)((K + KB - 1) / KB);
    a.per_part = (int)(K / parts), a.tiles_n = (int)((N + 63) / 64);
    const int64_t groups = B * a.blocks * a.tiles_n;
    return dtype == FFTCONV_BF16 ? launch(a, groups, k_blocks_channels<__bf16>, s)
         : dtype == FFTCONV_F16  ? launch(a, groups, k_blocks_channels<_Float16>, s)
                                 : launch(a, groups, k_blocks_channels<float>, s);
}

int quantize_tiles(const void *x, int64_t ldx, uint8_t *q, float *scale, uint8_t *qt, float *scale_t, int64_t O, int64_t K, int dtype, hipStream_t s)
{
    TileArgs a = {x, q, qt, scale, scale_t, O, K, ldx, 0, (int)((O + KB - 1) / KB), (int)((K + KB - 1) / KB)};
    const int64_t groups = (int64_t)a.tiles_o * a.tiles_k;
    return dtype == FFTCONV_BF16 ? launch(a, groups, k_tiles<__bf16>, s) : dtype == FFTCONV_F16 ? launch(a, groups, k_tiles<_Float16>, s) : launch(a, groups, k_tiles<float>, s);
}

}  // namespace lay
}  // namespace fftconv
