// Product of rows in e4m3 with a weight in e4m3, a scale for each 128 of a row and for each 128 x 128 of the weight:
//
//   y[t, o] = sum over blocks j of k (xs[j, t] ws[o / 128, j]) (sum over k in j of x[t, k] w[o, k]) + bias[o]
//
// The inner sums are the matrix cores' (fp32); each is added to the fp32 total with one multiply-add, its scale the product of the two, rounded.
// The weight's rows are the matrix cores' rows (R), the tokens their columns (S): a lane of an accumulator holds one token, so a block's scale is one
// number a lane, and the weight's scale is the same in the whole wave. Token by token a lane's four consecutive rows are neighbours in y; channel by
// channel the lanes are.
//
// Which kernel: up to 64 tokens k_f8_few, bound by the weight's bytes, but for very long rows and very many outputs. Above, with k in pieces of 16 bytes (both operands aligned to them), k_f8_large on
// tiles of 256 x 256 where these fill the compute units, else k_f8_small on 128 x 128 where there are 128 of those, or with k in ranges where there
// are fewer and k is 1024 or more. Rows of other lengths are laid out again for these where that pays (f8_padded); everything else is k_f8's, which
// takes any k at any alignment: among it fewer than 128 tiles with a k below 1024 (768 -> 768: 65 tokens 6.9 us, 1024 7.2, 2688 8.4, and 9.1 for 2689, from where on
// it is k_f8_small's; 768 -> 2304: 300 7.3, 896 8.6; a call takes 8 on the host; other kernels have not been tried there).
#include "layers_index.h"
#include "linear_common.h"

namespace fftconv {
namespace lay {

typedef __attribute__((ext_vector_type(8))) int i32x8;

struct F8Args {
    const uint8_t *x, *w;         // (T, K), (O, K)
    const float *xs, *ws, *bias;  // (blocks, T), (ceil(O / 128), blocks), O
    void *y;
    int64_t K, B;
    int T, O, blocks, row_tiles;  // blocks of k; tiles of O that have a scale
    int channels, N, per_part;
    uint32_t by_n, by_part;       // 2^32 over these, rounded up
    int beyond_cache;             // y is larger than the memory-side cache (256 MB) by far
    int tiles_r, tiles_s;
    int first;                    // tile of a launch's first workgroup (k_f8)
    int ranges, per;              // of k, whose sums of a tile are added up by a second kernel (1: all of k); blocks of one
    float *part;                  // (ranges, T, O)
};

// y[token_of(t) + output_of(o)] is the place of output o of token t.
__device__ __forceinline__ int64_t token_of(const F8Args &a, int t)
{
    if (!a.channels) return (int64_t)t * a.O;
    const int b = quotient(t, a.N, a.by_n);
    return t + (int64_t)b * (a.per_part - 1) * a.N;
}
__device__ __forceinline__ int64_t output_of(const F8Args &a, int o)
{
    if (!a.channels) return o;
    return (o + quotient(o, a.per_part, a.by_part) * (a.B - 1) * a.per_part) * a.N;
}

// Products of 32 x 32 x 128: operands of 2 x 32 bytes a lane, whichever of k they are, the same in both.
struct Half {
    uint4 a, b;
};
__device__ __forceinline__ i32x8 operand(const Half &h)
{
    const i32x8 v = {(int)h.a.x, (int)h.a.y, (int)h.a.z, (int)h.a.w, (int)h.b.x, (int)h.b.y, (int)h.b.z, (int)h.b.w};
    return v;
}
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
// eight values of e4m3 as bf16, which holds each of them
__device__ __forceinline__ bf16x8 widened(uint32_t lo, uint32_t hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    const bf16x8 v = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    return v;
}
// What the products of e4m3 keep: of eight neighbours along k, each down to 2^-13 of the largest one's power of two (by the operands' exponents), the rest dropped,
// then sums in fp32 (so does the instruction for any of the 8-bit formats; measured with one product of 2^16 and one of 2^16 down to 2^-9 beside it; sums
// computed so round to the kernels' results). That is 1.3e-5 of the result on normally distributed values, 3.3e-5 with one channel in a hundred twenty times
// as large: for results in 16 bits, whose own rounding is 2e-4 and more, of no account (one bf16 result in fifty is rounded the other way, one of fp16 in eight).
// fp32 results take the values to bf16, which holds them, and bf16's products, which are exact, at half the rate: 8192 x 4096 -> 16384 1142 us instead of 567.
template <bool CLOSE> __device__ __forceinline__ void product_of(const Half &r, const Half &s, f32x16 &c)
{
    if constexpr (!CLOSE) {
        c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(r), operand(s), c, 0, 0, 0, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(r.a.x, r.a.y), widened(s.a.x, s.a.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(r.a.z, r.a.w), widened(s.a.z, s.a.w), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(r.b.x, r.b.y), widened(s.b.x, s.b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(r.b.z, r.b.w), widened(s.b.z, s.b.w), c, 0, 0, 0);
    }
}
template <bool CLOSE> __device__ __forceinline__ void products(const Half (&r)[2], const Half (&s)[2], f32x16 &c)
{
    product_of<CLOSE>(r[0], s[0], c);
    product_of<CLOSE>(r[1], s[1], c);
}
template <bool CLOSE> __device__ __forceinline__ f32x4 products16(const Half &r, const Half &s)
{
    f32x4 c = {};
    if constexpr (!CLOSE) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(r), operand(s), c, 0, 0, 0, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(r.a.x, r.a.y), widened(s.a.x, s.a.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(r.a.z, r.a.w), widened(s.a.z, s.a.w), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(r.b.x, r.b.y), widened(s.b.x, s.b.y), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(r.b.z, r.b.w), widened(s.b.z, s.b.w), c, 0, 0, 0);
}

// The place in LDS of 16-byte piece c (0 .. 7) of a 128-byte row: two rows lie in the 256 bytes that a clock delivers, so the piece is moved by the
// row's number above that, and the same piece of sixteen rows in a run comes from banks of their own.
__device__ __forceinline__ int piece128(int row, int c) { return row * 128 + ((c ^ ((row >> 1) & 7)) << 4); }

// One accumulator of 32 x 32 to y: lane l holds token t (of column l % 32), register i output o0 + 8 (i / 4) + 4 (l / 32) + i % 4. Places of any kind.
template <typename T> __device__ __forceinline__ void store_f8(const F8Args &a, const f32x16 &acc, int o0, int t, int64_t token)
{
    const int half = (threadIdx.x >> 5) & 1;
    if (t >= a.T) return;
    T *const y = (T *)a.y + token;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int o = o0 + 8 * q + 4 * half;
        T v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(acc[4 * q + i] + (a.bias ? a.bias[min(o + i, a.O - 1)] : 0.f));
        if (!a.channels) {
            if (o < a.O) store_piece<T, 4>(y + o, a.O - o, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (o + i < a.O) y[output_of(a, o + i)] = v[i];
        }
    }
}

// Tiles of 64 FR outputs by 64 FS tokens, 2 x 2 waves; any k at any alignment, through registers.
template <typename T, int FR, int FS> __global__ void __launch_bounds__(256, 2) k_f8(const F8Args a)
{
    constexpr int BR = 64 * FR, BS = 64 * FS, STAGE = (BR + BS) * 128, PIECES = (BR + BS) * 8 / 256;
    extern __shared__ __align__(16) char lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int wr = wave >> 1, wsv = wave & 1;
    const int tile = a.first + (int)blockIdx.x, tr = tile / a.tiles_s, ts = tile % a.tiles_s;
    const int r0 = tr * BR, s0 = ts * BS;
    uint4 stage[PIECES];
    auto fetch = [&](int block) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = threadIdx.x + i * 256, row = p >> 3;
            const bool is_r = row < BR;
            const int g = is_r ? min(r0 + row, a.O - 1) : min(s0 + row - BR, a.T - 1);      // rows beyond the end: the last one, not stored
            stage[i] = load16((is_r ? a.w : a.x) + (int64_t)g * a.K, (int64_t)block * 128 + (threadIdx.x & 7) * 16, a.K);
        }
    };
    auto keep = [&](int buf) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = threadIdx.x + i * 256;
            *(uint4 *)(lds + buf * STAGE + piece128(p >> 3, p & 7)) = stage[i];
        }
    };
    int tokens[FS];
#pragma unroll
    for (int j = 0; j < FS; ++j) tokens[j] = s0 + (wsv * FS + j) * 32 + l32;
    const float *const ws = a.ws + (int64_t)min((r0 + wr * FR * 32) / 128, a.row_tiles - 1) * a.blocks;      // (a wave's outputs lie in one tile of the weight)
    f32x16 acc[FR][FS] = {};
    fetch(0);
    keep(0);
    lds_barrier();
    for (int k = 0; k < a.blocks; ++k) {
        if (k + 1 < a.blocks) fetch(k + 1);
        float s[FS];
#pragma unroll
        for (int j = 0; j < FS; ++j) s[j] = a.xs[(int64_t)k * a.T + min(tokens[j], a.T - 1)] * ws[k];
        const char *const base = lds + (k & 1) * STAGE;
        Half fs[FS][2];
#pragma unroll
        for (int j = 0; j < FS; ++j)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const int row = BR + (wsv * FS + j) * 32 + l32;
                fs[j][kk] = {*(const uint4 *)(base + piece128(row, kk * 4 + half)), *(const uint4 *)(base + piece128(row, kk * 4 + 2 + half))};
            }
#pragma unroll
        for (int i = 0; i < FR; ++i) {
            Half fr[2];
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const int row = (wr * FR + i) * 32 + l32;
                fr[kk] = {*(const uint4 *)(base + piece128(row, kk * 4 + half)), *(const uint4 *)(base + piece128(row, kk * 4 + 2 + half))};
            }
#pragma unroll
            for (int j = 0; j < FS; ++j) {
                f32x16 p = {};
                products<sizeof(T) == 4>(fr, fs[j], p);
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = fmaf(p[e], s[j], acc[i][j][e]);
            }
        }
        if (k + 1 < a.blocks) {
            keep((k + 1) & 1);
            lds_barrier();
        }
    }
#pragma unroll
    for (int j = 0; j < FS; ++j) {
        const int64_t token = token_of(a, min(tokens[j], a.T - 1));
#pragma unroll
        for (int i = 0; i < FR; ++i) store_f8<T>(a, acc[i][j], r0 + (wr * FR + i) * 32, tokens[j], token);
    }
}

// Results of a tile inside y whose rows' runs of 16 bytes do not end within: by way of 4 KB of LDS of the wave's own, so that a store writes 128 bytes in
// a row of eight rows, whole lines, instead of scattered words. An accumulator's values go there with the bias, rounded, in rows of y; 16-byte pieces
// (in rows of 64 bytes: rows) are moved so that the lanes that write at once meet no bank twice.
//
// Token by token: rows of ROW bytes to a token. 128: 64 outputs, of which this is part `part`; the halves of a piece change places in tokens 16 up. 64: 32 outputs.
template <typename T, int ROW> __device__ __forceinline__ void tokens_to_lds(char *own, const f32x16 &acc, int part, const float *bias)
{
    const int half = (threadIdx.x >> 5) & 1, l32 = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x4 b = *(const f32x4 *)(bias + 8 * q + 4 * half);
        const T t[4] = {from_f32<T>(acc[4 * q] + b[0]), from_f32<T>(acc[4 * q + 1] + b[1]), from_f32<T>(acc[4 * q + 2] + b[2]), from_f32<T>(acc[4 * q + 3] + b[3])};
        uint2 w;
        __builtin_memcpy(&w, t, 8);
        const int at = ROW == 128 ? (((4 * part + q) ^ ((l32 >> 1) & 7)) << 4) + ((half ^ (l32 >> 4)) << 3) : ((q ^ ((l32 >> 2) & 3)) << 4) + (half << 3);
        *(uint2 *)(own + l32 * ROW + at) = w;
    }
}
// Pieces t of a lane: of row lane / 8 + 8 t piece lane % 8 (128-byte rows), of row lane / 4 + 16 t piece lane % 4 (64-byte ones).
template <int ROW> __device__ __forceinline__ uint4 token_piece(const char *own, int t)
{
    const int lane = threadIdx.x & 63;
    if constexpr (ROW == 64) {
        const int c = (lane >> 2) + 16 * t;
        return *(const uint4 *)(own + c * 64 + (((lane & 3) ^ ((c >> 2) & 3)) << 4));
    } else {
        const int c = (lane >> 3) + 8 * t;
        const uint4 v = *(const uint4 *)(own + c * 128 + (((lane & 7) ^ ((c >> 1) & 7)) << 4));
        return t >= 2 ? make_uint4(v.z, v.w, v.x, v.y) : v;
    }
}
// Channel by channel: rows of WIDE tokens to an output: 64, of which this is 32-token part `part`, or 32. Values of two neighbouring lanes change places so
// that each lane writes a word: the even one of the first of two outputs, the odd one of the second.
template <typename T, int WIDE> __device__ __forceinline__ void channels_to_lds(char *own, const f32x16 &acc, int part, const float *bias)
{
    const int half = (threadIdx.x >> 5) & 1, l32 = threadIdx.x & 31, odd = l32 & 1;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x4 b = *(const f32x4 *)(bias + 8 * q + 4 * half);
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const T t[2] = {from_f32<T>(acc[4 * q + i] + b[i]), from_f32<T>(acc[4 * q + i + 1] + b[i + 1])};
            uint32_t w;
            __builtin_memcpy(&w, t, 4);
            const uint32_t n = dpp<0xB1>(w);                     // the neighbour's
            const uint32_t o = __builtin_amdgcn_perm(n, w, odd ? 0x03020706u : 0x05040100u);
            const int row = 8 * q + 4 * half + i + odd, moved = (row >> 2) & 1;
            if constexpr (WIDE == 64) *(uint32_t *)(own + row * 128 + (((part * 4 + (l32 >> 3)) ^ (moved << 2)) << 4) + ((l32 >> 1) & 3) * 4) = o;
            else *(uint32_t *)(own + (row ^ (moved << 1)) * 64 + (l32 >> 1) * 4) = o;
        }
    }
}
template <int WIDE> __device__ __forceinline__ uint4 output_piece(const char *own, int t)
{
    const int lane = threadIdx.x & 63, row = WIDE == 32 ? (lane >> 2) + 16 * t : (lane >> 3) + 8 * t, moved = (row >> 2) & 1;
    if constexpr (WIDE == 32) return *(const uint4 *)(own + (row ^ (moved << 1)) * 64 + ((lane & 3) << 4));
    else return *(const uint4 *)(own + row * 128 + (((lane & 7) ^ (moved << 2)) << 4));
}

// The same for operands in pieces of 16 bytes (K a multiple of 16): 2 x 4 waves, pieces straight to LDS, a block of 128 while the one before it is
// multiplied, in one stream over a workgroup's tiles. A wave holds the tokens' operands of a block and brings the weight's 32 rows at a time, one group
// ahead; sums of a block are two accumulators in turn, added to the totals while the next products run.
//
// Measured: f16 8192 x 4096 -> 16384 583 us, 1.9 PFLOP/s; bf16 64 x 4096 x 2304 -> 768 547 us, 1.7. The socket is at its cap back to back (1395 and 1399 of
// 1400 W), so joules count: the products with their reads of LDS alone take 327 us, the scales' multiply-adds 110 on top, what is brought 100, what is
// stored 80. (The library's product with one scale for each operand: 479 us on these values at the same cap.) Hence the large tile, whole lines to a
// store, and one multiply-add for a value and block. Bringing blocks a block and a half ahead, in two parts, 617 us; storing a tile's results among the next
// one's first products 722, for registers then go to memory; other orders of the tiles 569 to 620.
template <typename T, bool CHANNELS> __global__ void __launch_bounds__(512, 2) k_f8_large(const F8Args a, const Walk walk)
{
    constexpr int FR = 4, FS = 2, BR = 64 * FR, BS = 128 * FS, STAGE = (BR + BS) * 128, LI = (BR + BS) / 64;
    static_assert(BR == BS && LI % 4 == 0 && sizeof(T) == 2, "waves 0-3 bring the weight, 4-7 bring the tokens");
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int wr = wave >> 2, wsv = wave & 3;
    // tiles first, first + stride, ... below last
    const int wgs = gridDim.x, die = blockIdx.x % 8, dies = min(8, wgs), on_die = (wgs - die + 7) / 8;
    // (the dies that have a workgroup more have a tile more: 162 tiles, 1100 x 768 -> 2304, 11 us instead of 16)
    const int begin = die * (walk.tiles / dies) + min(die, walk.tiles % dies), last = begin + walk.tiles / dies + (die < walk.tiles % dies ? 1 : 0);
    const int first = begin + blockIdx.x / 8;
    const bool tail = a.K % 128 != 0;

    // This wave brings rows LI * 8 * (wave % 4) ... of the weight (waves 0-3) or the tokens (4-7), eight with an instruction, a piece of 16 bytes for each
    // lane, moved as piece128 has it; and, for itself, the scales of its 32 FS tokens and of its outputs.
    const bool is_r = wave < 4;
    const int rows = is_r ? a.O : a.T, block = is_r ? BR : BS;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_offset(lds)) + wave * LI * 1024;
    constexpr int OWN = 512, PRIVATE = 2 * OWN + FR * 128;       // a stage's scales of a wave; both stages' and the bias of its outputs
    char *const own = lds + 2 * STAGE + wave * PRIVATE;
    int f_tile = first, f_step = 0;                              // what is asked for next
    const char *base = nullptr, *xs = nullptr, *ws = nullptr;
    uint32_t off[LI], xs_off = 0;
    auto aim = [&] {                                             // at tile f_tile, or, after the last, once more at it
        int tr, ts;
        walk.place(min(f_tile, last - 1), tr, ts, a.tiles_r);
        const int row0 = (is_r ? tr : ts) * block;
        base = (const char *)(is_r ? a.w : a.x) + (int64_t)row0 * a.K - 3 * 1024;
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            const int row = (wave & 3) * 8 * LI + i * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
            off[i] = (uint32_t)(min(row0 + row, rows - 1) - row0) * (uint32_t)a.K + piece * 16 + 3 * 1024 - (i % 4) * 1024;
        }
        const int s0 = ts * BS;
        xs = (const char *)(a.xs + s0);
        xs_off = (uint32_t)(min(s0 + wsv * FS * 32 + (FS == 2 ? lane : l32), a.T - 1) - s0) * 4u;
        ws = (const char *)(a.ws + (int64_t)min((tr * BR + wr * FR * 32) / 128, a.row_tiles - 1) * a.blocks);
    };
    auto fetch = [&](int stage) {
        if (tail && f_step == a.blocks - 1) {          // what lies beyond K reads as zeros
#pragma unroll
            for (int i = 0; i < LI; ++i) {
                const int row = (wave & 3) * 8 * LI + i * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
                const char *const from = base + off[i] + (i % 4) * 1024;
                to_lds16((int64_t)f_step * 128 + piece * 16 < a.K ? from : (const char *)&zero_piece, lds + stage * STAGE + (wave * LI + i) * 1024);
            }
        } else {
#pragma unroll
            for (int i = 0; i < LI; i += 4) {
                const uint32_t four[4] = {off[i], off[i + 1], off[i + 2], off[i + 3]};
                to_lds16_rows<4>(uniform(base), four, __builtin_amdgcn_readfirstlane(to + stage * STAGE + i * 1024));
            }
        }
        to_lds4(uniform(xs), xs_off, own + stage * OWN);
        to_lds4(uniform(ws), 0, own + stage * OWN + 256);
        base += 128, xs += (int64_t)a.T * 4, ws += 4;
        if (++f_step == a.blocks) {
            f_step = 0, f_tile += on_die;
            aim();
        }
    };

    if (first >= last) return;
    aim();
    fetch(0);
    // where this lane's pieces are, from a stage's start: piece c of its row at ^ (c << 4)
    const int ro = piece128(wr * FR * 32 + l32, half), so = BR * 128 + piece128(wsv * FS * 32 + l32, half);
    Half fr[2][2], fs[FS][2];
    auto read = [&](Half (&to)[2], const char *at, int where) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) to[kk] = {*(const uint4 *)(at + (where ^ (kk << 6))), *(const uint4 *)(at + (where ^ (kk << 6) ^ 32))};
    };
    FC_ARRIVED(0);
    fetch(1);
    int stage = 0;
    read(fr[0], lds, ro);
#pragma unroll
    for (int j = 0; j < FS; ++j) read(fs[j], lds + j * 4096, so);
    for (int tile = first; tile < last; tile += on_die) {
        int tr, ts;
        walk.place(tile, tr, ts, a.tiles_r);
        const int steps = a.blocks;
        const char *const bias = uniform(a.bias ? (const char *)(a.bias + tr * BR) : (const char *)&zero_piece);
#pragma unroll
        for (int i = 0; i < FR; i += 2)
            to_lds4(bias, a.bias ? (uint32_t)(min(tr * BR + (wr * FR + i) * 32 + lane, a.O - 1) - tr * BR) * 4u : 0u, own + 2 * OWN + i * 128);
        f32x16 acc[FR][FS] = {};
        for (int k = 0; k < steps; ++k) {
            const char *const here = lds + stage * STAGE, *const scales = own + stage * OWN;
            float s[FS];
            const float w = *(const float *)(scales + 256);
#pragma unroll
            for (int j = 0; j < FS; ++j) s[j] = *(const float *)(scales + (j * 32 + l32) * 4) * w;
            const int next = stage ^ 1;
#pragma unroll
            for (int i = 0; i < FR; ++i) {
                f32x16 p[FS];
                if (i + 1 < FR) {
                    read(fr[(i + 1) & 1], here + (i + 1) * 4096, ro);
                } else {
                    FC_ARRIVED(0);                               // the next block is there, and every wave has read this one
                    if (k + 1 < steps) fetch(stage);             // (after a tile's last one its results go by way of that stage first)
                    read(fr[(i + 1) & 1], lds + next * STAGE, ro);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < FS; ++j) {
                    p[j] = f32x16{};
                    products<false>(fr[i & 1], fs[j], p[j]);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (i + 1 == FR) {
#pragma unroll
                    for (int j = 0; j < FS; ++j) read(fs[j], lds + next * STAGE + j * 4096, so);
                }
#pragma unroll
                for (int j = 0; j < FS; ++j) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = fmaf(p[j][e], s[j], acc[i][j][e]);
                    asm volatile("" : "+v"(acc[i][j]));          // (else the compiler adds all of a block's sums at its end, and keeps them until then)
                }
            }
            stage = next;
        }
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                           // (else the compiler keeps the places below in registers throughout the sums)
        const int l32 = lane & 31, r0 = tr * BR, s0 = ts * BS;
        const int r1 = r0 + wr * FR * 32, s1 = s0 + wsv * FS * 32;
        // All of it inside y, in one sequence and one part of y: places are linear in rows and columns.
        bool whole = r0 + BR <= a.O && s0 + BS <= a.T && (CHANNELS ? a.N : a.O) < 1 << 26;        // (32-bit distances of seven rows)
        if (CHANNELS)
            whole = whole && quotient(s0, a.N, a.by_n) == quotient(s0 + BS - 1, a.N, a.by_n) &&
                    quotient(r0, a.per_part, a.by_part) == quotient(r0 + BR - 1, a.per_part, a.by_part);
        if (whole) {
            // The stage of the last block: every wave has read it, and what comes there next is, in a wave's own 4 KB or more, that wave's own transfers.
            static_assert(LI >= 4, "a wave's results fit where its transfers go");
            char *const mine = lds + (stage ^ 1) * STAGE + wave * LI * 1024;
            const float *const bias = (const float *)(own + 2 * OWN);
            constexpr int W = 8;
            const uint32_t stride = CHANNELS ? (uint32_t)a.N : (uint32_t)a.O;
            const char *const y = uniform((const char *)((T *)a.y + token_of(a, s1) + output_of(a, r1)));
            const uint32_t at = ((uint32_t)(lane >> 3) * stride + (lane & 7) * W) * 2u;
            auto all = [&](auto beyond) {
                // four pieces a lane, from row i (of 32 outputs) and column j (of 32 tokens) on
                auto out = [&](int i, int j) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint4 v = CHANNELS ? output_piece<64>(mine, t) : token_piece<128>(mine, t);
                        const int row = 8 * t;
                        const int64_t place = CHANNELS ? (int64_t)(i * 32 + row) * stride + j * 32 : (int64_t)(j * 32 + row) * stride + i * 32;
                        put16<decltype(beyond)::value>((char *)y + place * 2 + at, v);
                    }
                };
                constexpr int PI = CHANNELS ? 1 : 2, PJ = CHANNELS ? 2 : 1;
#pragma unroll
                for (int i = 0; i < FR; i += PI)
#pragma unroll
                    for (int j = 0; j < FS; j += PJ) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int p = 0; p < PI; ++p)
#pragma unroll
                            for (int q = 0; q < PJ; ++q) {
                                if constexpr (CHANNELS) channels_to_lds<T, 64>(mine, acc[i + p][j + q], q, bias + (i + p) * 32);
                                else tokens_to_lds<T, 128>(mine, acc[i + p][j + q], p, bias + (i + p) * 32);
                            }
                        out(i, j);
                    }
            };
            if (a.beyond_cache) all(std::true_type());
            else all(std::false_type());
        } else {
#pragma unroll
            for (int j = 0; j < FS; ++j) {
                const int t = s1 + j * 32 + l32;
                const int64_t token = token_of(a, min(t, a.T - 1));
#pragma unroll
                for (int i = 0; i < FR; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    store_f8<T>(a, acc[i][j], r1 + i * 32, t, token);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        fetch(stage ^ 1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // nothing is on its way to LDS when the workgroup ends
}

// Tiles of 128 x 128, where there are too few of 256 x 256: 2 x 4 waves of 64 outputs by 32 tokens, four steps of 64 of k in LDS, asked for three steps ahead,
// for here it is how long a transfer takes that counts (4096 x 768 -> 2304: six blocks to a tile). Sums of a block stay in their accumulators over its two
// steps. Two workgroups share a compute unit, and one reads its operands while the other multiplies; ALONE, where there is a unit for every tile, a
// wave's own operands are read a step ahead, and its pieces asked for four ahead.
template <typename T, bool CHANNELS, bool SPLIT, bool ALONE> __global__ void __launch_bounds__(512, ALONE ? 2 : 4) k_f8_small(const F8Args a, const Walk walk)
{
    constexpr int FR = 2, BR = 128, BS = 128, BK = 64, STAGE = (BR + BS) * BK, STAGES = 4;
    constexpr bool CLOSE = sizeof(T) == 4;
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int wr = wave >> 2, wsv = wave & 3;
    // tiles first, first + stride, ... below last
    const int wgs = gridDim.x, die = blockIdx.x % 8, dies = min(8, wgs), on_die = (wgs - die + 7) / 8;
    // (the dies that have a workgroup more have a tile more: 162 tiles, 1100 x 768 -> 2304, 11 us instead of 16)
    const int begin = die * (walk.tiles / dies) + min(die, walk.tiles % dies), last = begin + walk.tiles / dies + (die < walk.tiles % dies ? 1 : 0);
    const int first = begin + blockIdx.x / 8;
    const int all_steps = (int)((a.K + BK - 1) / BK);
    const bool tail = a.K % BK != 0;
    // item i of the walk: tile i / ranges, range i % ranges of k
    auto item = [&](int i, int &tr, int &ts, int &range) {
        range = SPLIT ? i % a.ranges : 0;
        walk.place(SPLIT ? i / a.ranges : i, tr, ts, a.tiles_r);
    };
    auto steps_of = [&](int range) { return SPLIT ? min(2 * a.per, all_steps - 2 * range * a.per) : all_steps; };

    // This wave brings 32 rows of the weight (waves 0-3) or the tokens (4-7), sixteen with an instruction, a piece of 16 bytes for each lane, moved as
    // piece_at has it; and, for itself, with a block's first step, the scales of its 32 tokens (lanes 0-31) and of its outputs (one, in lanes 32-63).
    const bool is_r = wave < 4;
    const int rows = is_r ? a.O : a.T;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_offset(lds)) + wave * 2048;
    char *const own = lds + STAGES * STAGE + wave * (STAGES * 256 + 256);
    int f_tile = first, f_step = 0, f_steps = 0, f_first = 0;    // what is asked for next; steps of its range, and of those before it
    const char *base = nullptr, *scale = nullptr;
    uint32_t off[2];
    auto aim = [&] {                                             // at tile f_tile, or, after the last, once more at it
        int tr, ts, range;
        item(min(f_tile, last - 1), tr, ts, range);
        f_steps = steps_of(range), f_first = SPLIT ? 2 * range * a.per : 0;
        const int row0 = (is_r ? tr : ts) * 128;
        base = (const char *)(is_r ? a.w : a.x) + (int64_t)row0 * a.K + (int64_t)f_first * BK - 1024;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = (wave & 3) * 32 + i * 16 + (lane >> 2), piece = (lane & 3) ^ ((row >> 2) & 3);
            off[i] = (uint32_t)(min(row0 + row, rows - 1) - row0) * (uint32_t)a.K + piece * 16 + 1024 - i * 1024;
        }
        scale = half == 0 ? (const char *)(a.xs + (int64_t)(f_first / 2) * a.T + min(ts * BS + wsv * 32 + l32, a.T - 1))
                          : (const char *)(a.ws + (int64_t)min(tr, a.row_tiles - 1) * a.blocks + f_first / 2);
    };
    const int64_t scale_step = half == 0 ? (int64_t)a.T * 4 : 4;
    auto fetch = [&](int stage) {
        if (tail && f_first + f_step == all_steps - 1) {         // what lies beyond K reads as zeros
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int piece = (lane & 3) ^ ((lane >> 4) & 3);
                const char *const from = base + off[i] + i * 1024;
                to_lds16((int64_t)(f_first + f_step) * BK + piece * 16 < a.K ? from : (const char *)&zero_piece, lds + stage * STAGE + wave * 2048 + i * 1024);
            }
        } else {
            to_lds16_rows<2>(uniform(base), off, __builtin_amdgcn_readfirstlane(to + stage * STAGE));
        }
        if (f_step % 2 == 0) {
            to_lds4(scale, own + stage * 256);
            scale += scale_step;
        }
        base += BK;
        if (++f_step == f_steps) {
            f_step = 0, f_tile += on_die;
            aim();
        }
    };

    if (first >= last) return;
    aim();
#pragma unroll
    for (int i = 0; i < (ALONE ? STAGES : STAGES - 1); ++i) fetch(i);
    // where this lane's pieces are, from a stage's start: half of a row's, and the other two at ^ 32
    const int ro = piece_at(wr * FR * 32 + l32, half), so = BR * BK + piece_at(wsv * 32 + l32, half);
    Half fr[2][FR], fs[2];
    auto read = [&](int buf, const char *here) {
#pragma unroll
        for (int i = 0; i < FR; ++i) fr[buf][i] = {*(const uint4 *)(here + ro + i * 2048), *(const uint4 *)(here + (ro ^ 32) + i * 2048)};
        fs[buf] = {*(const uint4 *)(here + so), *(const uint4 *)(here + (so ^ 32))};
    };
    if constexpr (ALONE) {                                       // (or a step's are read when it comes)
        FC_ARRIVED(2 + 3 + 2);                                   // three transfers with a block's first step, two with its second
        read(0, lds);
    }
    int stage = 0;
    for (int tile = first; tile < last; tile += on_die) {
        int tr, ts, range;
        item(tile, tr, ts, range);
        const int steps = steps_of(range), r0 = tr * BR, s0 = ts * BS;
        if (!SPLIT)
            to_lds4(uniform(a.bias ? (const char *)(a.bias + r0) : (const char *)&zero_piece), a.bias ? (uint32_t)(min(r0 + wr * FR * 32 + lane, a.O - 1) - r0) * 4u : 0u,
                    own + STAGES * 256);
        f32x16 acc[FR] = {}, p[FR];
        float s = 0.f;
        auto step = [&](auto which, int k) {
            constexpr int KK = decltype(which)::value;
            const char *const here = lds + stage * STAGE, *const scales = own + stage * 256;
            const int next = stage + 1 < STAGES ? stage + 1 : 0;
            if (ALONE && KK == 0) s = *(const float *)(scales + l32 * 4) * *(const float *)(scales + 128);
            // This step's pieces (ALONE: the next one's) are there, those of the two after it on their way; every wave has read the last one's (this one's).
            FC_ARRIVED(2 + 3);
            // (the tile's last one is asked for after its results, which go by way of that stage)
            if (k + 1 < steps) fetch(ALONE ? stage : stage == 0 ? STAGES - 1 : stage - 1);
            if (!ALONE && KK == 0) s = *(const float *)(scales + l32 * 4) * *(const float *)(scales + 128);
            if constexpr (ALONE) {
                read(KK ^ 1, lds + next * STAGE);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < FR; ++i) {
                    if (KK == 0) p[i] = f32x16{};
                    product_of<CLOSE>(fr[KK][i], fs[KK], p[i]);
                }
            } else {
                const Half tokens = {*(const uint4 *)(here + so), *(const uint4 *)(here + (so ^ 32))};
#pragma unroll
                for (int i = 0; i < FR; ++i) {
                    const Half outputs = {*(const uint4 *)(here + ro + i * 2048), *(const uint4 *)(here + (ro ^ 32) + i * 2048)};
                    if (KK == 0) p[i] = f32x16{};
                    product_of<CLOSE>(outputs, tokens, p[i]);
                }
            }
            stage = next;
        };
        auto add = [&] {
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][e] = fmaf(p[i][e], s, acc[i][e]);
        };
        int k = 0;
        for (; k + 2 <= steps; k += 2) {
            step(std::integral_constant<int, 0>(), k);
            step(std::integral_constant<int, 1>(), k + 1);
            add();
        }
        if (k < steps) {                                         // (a last block of one step)
            step(std::integral_constant<int, 0>(), k);
            add();
            if (ALONE) fr[0][0] = fr[1][0], fr[0][1] = fr[1][1], fs[0] = fs[1];
        }
        const int free_stage = (stage + (ALONE ? 3 : 2)) & 3;    // the last step's, or the one's before it: every wave has read it
        const int r1 = r0 + wr * FR * 32, s1 = s0 + wsv * 32;
        if constexpr (SPLIT) {
            float *const part = a.part + (int64_t)range * a.T * a.O;
            const int t = s1 + l32;
#pragma unroll
            for (int i = 0; i < FR; ++i) {
                const int o = r1 + i * 32 + 4 * half;
                if (t >= a.T) continue;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float v[4] = {acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
                    if (o + 8 * q < a.O) store_piece<float, 4>(part + (int64_t)t * a.O + o + 8 * q, a.O - o - 8 * q, v);
                }
            }
            fetch(free_stage);
            continue;
        }
        // All of it inside y, in one sequence and one part of y: places are linear in rows and columns.
        bool whole = sizeof(T) == 2 && r0 + BR <= a.O && s0 + BS <= a.T && (CHANNELS ? a.N : a.O) < 1 << 26;       // (32-bit distances of fifteen rows)
        if (CHANNELS)
            whole = whole && quotient(s0, a.N, a.by_n) == quotient(s0 + BS - 1, a.N, a.by_n) &&
                    quotient(r0, a.per_part, a.by_part) == quotient(r0 + BR - 1, a.per_part, a.by_part);
        bool done = false;
        if constexpr (sizeof(T) == 2) {
            if (whole) {
                done = true;
                // What comes to the free stage next is, in a wave's own 2 KB, that wave's own transfers. The bias is there three steps after it was asked for; with
                // fewer steps it is waited for.
                if (steps < 4) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                char *const mine = lds + free_stage * STAGE + wave * 2048;
                const float *const bias = (const float *)(own + STAGES * 256);
                const uint32_t stride = CHANNELS ? (uint32_t)a.N : (uint32_t)a.O;
                const char *const y = uniform((const char *)((T *)a.y + token_of(a, s1) + output_of(a, r1)));
                const uint32_t at = ((uint32_t)(lane >> 2) * stride + (lane & 3) * 8) * 2u;
#pragma unroll
                for (int i = 0; i < FR; ++i) {
                    if constexpr (CHANNELS) channels_to_lds<T, 32>(mine, acc[i], 0, bias + i * 32);
                    else tokens_to_lds<T, 64>(mine, acc[i], 0, bias + i * 32);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const uint4 v = CHANNELS ? output_piece<32>(mine, t) : token_piece<64>(mine, t);
                        const int64_t place = CHANNELS ? (int64_t)(i * 32 + 16 * t) * stride : (int64_t)(16 * t) * stride + i * 32;
                        put16<false>((char *)y + place * 2 + at, v);
                    }
                }
            }
        }
        if (!done) {
            const int t = s1 + l32;
            const int64_t token = token_of(a, min(t, a.T - 1));
#pragma unroll
            for (int i = 0; i < FR; ++i) store_f8<T>(a, acc[i], r1 + i * 32, t, token);
        }
        __builtin_amdgcn_sched_barrier(0);
        fetch(free_stage);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // nothing is on its way to LDS when the workgroup ends
}

// y from the ranges' sums, in the ranges' order.
template <typename T> __global__ void __launch_bounds__(256) k_f8_sums(const F8Args a)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, size = (int64_t)a.T * a.O;
    if (i >= size) return;
    float sum[4] = {};
#pragma unroll 4
    for (int k = 0; k < a.ranges; ++k) {
        float v[4];
        load_piece<float, 4>(a.part + k * size + i, size - i, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (i + e >= size) return;
        const int t = (int)((i + e) / a.O), o = (int)(i + e - (int64_t)t * a.O);
        ((T *)a.y)[token_of(a, t) + output_of(a, o)] = from_f32<T>(sum[e] + (a.bias ? a.bias[o] : 0.f));
    }
}

// Rows whose length is no multiple of 16 are laid out again at a distance that is one, with zeros behind them, tokens and weight one after the other, where
// that is worth the bytes and another launch: rows of 2000 and T O K of 2^29 and more, or 2^22 results. In us, as they are and so: 4095 -> 4096 64 tokens 44 and
// 23, 300 67 and 33, 8192 386 and 161; 8191 -> 1000 100 tokens 60 and 24, 64 tokens 78 either way; 2047 -> 4096 100 tokens 29 and 23; 1001 -> 3001 2048
// tokens 34 and 26, but 300 14 and 20, 512 16 and 24; 63 -> 10176 5950 tokens 83 and 35.
static bool f8_padded(int64_t T, int64_t K, int64_t O)
{
    return T > 16 && K % 16 != 0 && (T >= (((int64_t)1 << 22) + O - 1) / O || (K >= 2000 && (double)T * (double)O * (double)K >= (double)((int64_t)1 << 29)));
}
struct PadArgs {
    const uint8_t *x, *w;
    uint8_t *to;
    int64_t T, K, first, pitch;   // first: row of a launch's first piece
    int pieces, count;            // of 16 bytes: of a row, of the launch
    uint32_t by_pieces;
};
__global__ void __launch_bounds__(256) k_f8_pad(const PadArgs a)
{
    const int i = (int)(blockIdx.x * 256 + threadIdx.x);
    if (i >= a.count) return;
    const int r = quotient(i, a.pieces, a.by_pieces), p = i - r * a.pieces;
    const int64_t row = a.first + r;
    const uint4 v = load16(row < a.T ? a.x + row * a.K : a.w + (row - a.T) * a.K, (int64_t)p * 16, a.K);
    *(uint4 *)(a.to + row * a.pitch + p * 16) = v;
}

// Into how many ranges k goes: where few tiles are left for the compute units, as many as give each one, of four blocks at least. Up to 64 tokens where that is
// faster than k_f8_few, which takes the longer the more blocks and sixteens of tokens there are, however few the outputs. In us, k_f8_few and ranges: 33 tokens,
// 8192 -> 4096 17.7 and 15.6, 4096 -> 4096 9.6 and 13.5; 17 tokens, 16384 -> 4096 25.3 and 20.9, 8192 -> 4096 12.5 and 15.3; one, 32768 -> 1024 25.8 and 20.3,
// 12288 -> 1024 10.4 and 15.2; 64 of 65536 -> 1024 148 and 29.
static int f8_ranges(int64_t T, int64_t K, int64_t O)
{
    const int64_t tiles = ((T + 127) / 128) * ((O + 127) / 128), blocks = (K + 127) / 128;
    if (T <= 64 && blocks * (T <= 16 ? 1 : T <= 32 ? 2 : 4) < 256) return 1;
    if ((K % 16 != 0 && !f8_padded(T, K, O)) || tiles >= 128) return 1;
    const int64_t most = 256 / tiles < blocks / 4 ? 256 / tiles : blocks / 4;
    if (most < 2) return 1;
    const int64_t per = (blocks + most - 1) / most;
    return (int)((blocks + per - 1) / per);
}

// Few tokens (up to 16 NT): what counts is how fast the weight streams in, so its rows go from memory straight into the operand registers, 16 NO to a wave. WK
// waves divide the blocks of k among themselves and add their sums up in LDS; the eight of a workgroup take 8 / WK such runs of outputs. More outputs to a
// wave (a token's row is then read less often) and fewer waves to a row (short rows) where enough workgroups are left. Measured: 1 x 4096 -> 4096 5.2 us, 3.2 TB/s
// of the weight's 16.8 MB, of which a launch is about half; 1 x 8192 -> 16384 27 us, 4.9 TB/s. Against one run of 16 outputs to a workgroup of eight waves:
// 2048 -> 65536 of 1 token 35 -> 25 us; 4096 -> 16384 of 33 38 -> 19; 8192 -> 16384 of 64 81 -> 37.
template <typename T, int NT, int NO, int WK> __global__ void __launch_bounds__(512) k_f8_few(const F8Args a)
{
    __shared__ f32x4 sums[8][NO * NT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    constexpr int RUNS = 8 / WK;
    static_assert(RUNS * NO <= 8, "a workgroup's outputs lie in one tile of the weight");
    const int64_t wg0 = ((int64_t)a.first + blockIdx.x) * (16 * NO * RUNS), o0 = wg0 + wave / WK * (16 * NO);
    const float *const ws = a.ws + wg0 / 128 * a.blocks;
    const uint8_t *x[NT], *w[NO];
    int t[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) t[j] = min(j * 16 + l16, a.T - 1), x[j] = a.x + (int64_t)t[j] * a.K;
#pragma unroll
    for (int i = 0; i < NO; ++i) w[i] = a.w + min(o0 + 16 * i + l16, (int64_t)a.O - 1) * a.K;
    f32x4 acc[NO][NT] = {};
    constexpr int U = NT == 1 ? 4 : NT * NO >= 8 ? 1 : 2;
    for (int k0 = wave % WK; k0 < a.blocks; k0 += WK * U) {
        Half fw[U][NO], fx[U][NT];
        float s[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = (int64_t)(k0 + WK * u) * 128 + quarter * 16;
            const int block = min(k0 + WK * u, a.blocks - 1);
#pragma unroll
            for (int i = 0; i < NO; ++i) fw[u][i] = {load16(w[i], k, a.K), load16(w[i], k + 64, a.K)};
            const float sw = ws[block];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                fx[u][j] = {load16(x[j], k, a.K), load16(x[j], k + 64, a.K)};
                // (a block beyond the last is one of zeros)
                s[u][j] = k0 + WK * u < a.blocks ? a.xs[(int64_t)block * a.T + t[j]] * sw : 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < NO; ++i) {
                    const f32x4 p = products16<sizeof(T) == 4>(fw[u][i], fx[u][j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], s[u][j], acc[i][j][e]);
                }
    }
#pragma unroll
    for (int i = 0; i < NO; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    lds_barrier();
    // lane l holds token l % 16 of the sixteen, outputs 4 (l / 16) ... + 3
    for (int i = threadIdx.x; i < RUNS * NO * NT * 256; i += 512) {
        const int e = i & 3, l = (i >> 2) & 63, tile = (i >> 8) % (NO * NT), r = (i >> 8) / (NO * NT);
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < WK; ++v) sum += sums[r * WK + v][tile][l][e];
        const int token = tile % NT * 16 + (l & 15);
        const int64_t o = wg0 + (r * NO + tile / NT) * 16 + 4 * (l >> 4) + e;
        if (token >= a.T || o >= a.O) continue;
        ((T *)a.y)[token_of(a, token) + output_of(a, (int)o)] = from_f32<T>(sum + (a.bias ? a.bias[o] : 0.f));
    }
}

template <typename T> static int run(F8Args &a, void *workspace, hipStream_t s)
{
    bool pieces = a.K % 16 == 0 && ((uintptr_t)a.x | (uintptr_t)a.w) % 16 == 0;
    a.ranges = f8_ranges(a.T, a.K, a.O);
    if (f8_padded(a.T, a.K, a.O)) {
        const int64_t rows = (int64_t)a.T + a.O;
        PadArgs p = {a.x, a.w, (uint8_t *)(((uintptr_t)workspace + 15) & ~(uintptr_t)15), a.T, a.K, 0, (a.K + 15) / 16 * 16, (int)((a.K + 15) / 16), 0, 0};
        p.by_pieces = reciprocal(p.pieces);
        const int64_t most = ((int64_t)1 << 30) / p.pieces;      // rows to a launch, whose pieces are a number of 32 bits
        for (; p.first < rows; p.first += most) {
            p.count = (int)((rows - p.first < most ? rows - p.first : most) * p.pieces);
            k_f8_pad<<<(unsigned)((p.count + 255) / 256), 256, 0, s>>>(p);
            FC_HIP(hipGetLastError());
        }
        a.x = p.to, a.w = p.to + a.T * p.pitch, a.K = p.pitch, pieces = true;
        workspace = p.to + rows * p.pitch;
    }
    auto tiles = [&](int64_t b) { return ((a.O + b - 1) / b) * ((a.T + b - 1) / b); };
    // Up to 64 tokens: in ranges where these are the faster, or on tiles where those fill the compute units, once or twice. In us, k_f8_few and tiles: 64 tokens,
    // 2048 -> 33000 33 and 24, 4096 -> 16384 21 and 27; 32 tokens, 2048 -> 65536 36 and 26, 8192 -> 40000 91 and 94; one, 1024 -> 65536 14 and 16; fp32,
    // 32 tokens, 2048 -> 65536 48 and 39.
    if (a.T <= 64 && !(pieces && (a.ranges > 1 || (a.T > 16 && tiles(128) >= (a.T > 32 ? 256 : 512))))) {
        auto few = [&](auto kernel, int64_t outputs) -> int {
            return in_pieces((a.O + outputs - 1) / outputs, 512, [&](int64_t first, unsigned g) -> int {
                a.first = (int)first;
                kernel<<<g, 512, 0, s>>>(a);
                FC_HIP(hipGetLastError());
                return FFTCONV_OK;
            });
        };
        const int64_t runs = ((int64_t)a.O + 15) / 16;           // of 16 outputs; 256 workgroups at least are wanted
        if (a.T <= 16) {
            if (a.blocks <= 8 && runs >= 4 * 256) return few(k_f8_few<T, 1, 1, 2>, 64);
            if (a.blocks <= 16 && runs >= 2 * 256) return few(k_f8_few<T, 1, 1, 4>, 32);
            return few(k_f8_few<T, 1, 1, 8>, 16);
        }
        if (a.T <= 32) return runs >= 2 * 256 ? few(k_f8_few<T, 2, 2, 8>, 32) : few(k_f8_few<T, 2, 1, 8>, 16);
        return runs >= 4 * 256 ? few(k_f8_few<T, 4, 4, 8>, 64) : runs >= 2 * 256 ? few(k_f8_few<T, 4, 2, 8>, 32) : few(k_f8_few<T, 4, 1, 8>, 16);
    }
    auto launch = [&](auto f) -> int {
        constexpr int F = decltype(f)::value, lds = 2 * 2 * 64 * F * 128;
        a.tiles_r = (a.O + 64 * F - 1) / (64 * F), a.tiles_s = (a.T + 64 * F - 1) / (64 * F);
        FC_TRY(raise_dynamic_lds((const void *)k_f8<T, F, F>, lds));
        return in_pieces((int64_t)a.tiles_r * a.tiles_s, 256, [&](int64_t first, unsigned g) -> int {
            a.first = (int)first;
            k_f8<T, F, F><<<g, 256, lds, s>>>(a);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    };
    auto launch_async = [&](auto kernel, int block, int lds, int most) -> int {
        a.tiles_r = (a.O + block - 1) / block, a.tiles_s = (a.T + block - 1) / block;
        const Walk w = {a.tiles_s, a.tiles_s <= 12 ? a.tiles_s : 8, a.tiles_r * a.tiles_s * a.ranges};
        FC_TRY(raise_dynamic_lds((const void *)kernel, lds));
        kernel<<<(unsigned)(w.tiles < most ? w.tiles : most), 512, lds, s>>>(a, w);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    };
    constexpr int LARGE_LDS = 2 * 512 * 128 + 8 * (2 * 512 + 512), SMALL_LDS = 4 * 256 * 64 + 8 * (4 * 256 + 256);
    using std::integral_constant;
    if (pieces && a.ranges > 1) {
        a.per = (a.blocks + a.ranges - 1) / a.ranges, a.part = (float *)workspace;
        FC_TRY(launch_async(k_f8_small<T, false, true, true>, 128, SMALL_LDS, 256));
        k_f8_sums<T><<<(unsigned)(((int64_t)a.T * a.O + 1023) / 1024), 256, 0, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    }
    a.ranges = 1;
    // The large tile where there is one for every compute unit, k has four blocks or more, and its last round of tiles leaves few units without one: a round of
    // 256 takes as long as 1.55 to 2 rounds of 512 small ones, two of which share a unit. In us, large and small: 64 x 4096 x 768 -> 2304 (36 rounds) 686 and
    // 855, 16384 x 768 -> 2304 (576 tiles) 62 and 53, 8192 x 768 -> 2304 (288) 42 and 31, 6400 x 1024 -> 7168 (700) 79 and 72, 65536 x 4096 -> 1024 (1024) 302 and
    // 393; 65536 -> 4096 with k of 512 268 and 280, of 256 224 and 190.
    if constexpr (sizeof(T) == 2) {
        if (pieces && a.blocks >= 4 && tiles(256) >= 256 && (double)tiles(128) / 512 > 1.85 * (double)((tiles(256) + 255) / 256))
            return a.channels ? launch_async(k_f8_large<T, true>, 256, LARGE_LDS, 256) : launch_async(k_f8_large<T, false>, 256, LARGE_LDS, 256);
    }
    if (pieces && tiles(128) >= 128 && tiles(128) <= 256)            // (one to a compute unit)
        return a.channels ? launch_async(k_f8_small<T, true, false, true>, 128, SMALL_LDS, 256) : launch_async(k_f8_small<T, false, false, true>, 128, SMALL_LDS, 256);
    if (pieces && tiles(128) > 256)
        return a.channels ? launch_async(k_f8_small<T, true, false, false>, 128, SMALL_LDS, 512) : launch_async(k_f8_small<T, false, false, false>, 128, SMALL_LDS, 512);
    if (tiles(128) >= 256) return launch(integral_constant<int, 2>());
    return launch(integral_constant<int, 1>());
}

size_t linear_f8_workspace(int64_t T, int64_t K, int64_t O)
{
    const int ranges = f8_ranges(T, K, O);
    return (ranges > 1 ? (size_t)ranges * (size_t)T * (size_t)O * 4 : 0) + (f8_padded(T, K, O) ? (size_t)(T + O) * (size_t)((K + 15) / 16 * 16) + 16 : 0);
}

int linear_f8(const uint8_t *x, const float *xs, const uint8_t *w, const float *ws, const float *bias, void *y, int64_t B, int64_t N, int64_t K,
              int64_t O, int64_t parts, int dtype, void *workspace, hipStream_t s)
{
    F8Args a = {};
    a.x = x, a.w = w, a.xs = xs, a.ws = ws, a.bias = bias, a.y = y, a.K = K, a.B = B, a.T = (int)(B * N), a.O = (int)O;
    a.blocks = (int)((K + 127) / 128), a.row_tiles = (int)((O + 127) / 128);
    a.channels = parts > 0, a.N = (int)N, a.per_part = (int)(parts ? O / parts : O);
    a.by_n = reciprocal(a.N), a.by_part = reciprocal(a.per_part);
    a.beyond_cache = B * N * O * (dtype == FFTCONV_F32 ? 4 : 2) > (int64_t)512 << 20;
    if (dtype == FFTCONV_BF16) return run<__bf16>(a, workspace, s);
    if (dtype == FFTCONV_F16) return run<_Float16>(a, workspace, s);
    return run<float>(a, workspace, s);
}

}  // namespace lay
}  // namespace fftconv
