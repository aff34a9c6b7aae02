// Gradient of a projection's weight from its input in 8 bits:
//
//   dw[o, c] = sum over b, n of dy[b, n, o] q[b, c, n] s[b, c, n / 128]
//
// Eight bits fit a 16-bit operand of the matrix cores, so the products are exact; dy in fp32 is split into three bf16 parts that
// add up to it, with three products for one. The scale belongs to a channel and a run of 128 samples, and the sums of a channel lie in one
// lane's registers, so it never touches an operand: the sums are kept in units of the current run's scale and multiplied by the quotient of
// the old scale and the new one from run to run, in fp32.
//
// A workgroup takes a tile of dw and a range of runs; the ranges' sums are added up in their order by a second kernel.
//
// Which kernel: k_weight_async for 16-bit dy in pieces of 16 bytes, k_weight for everything else (fp32, odd lengths, any alignment): it stages
// dy and q through registers, where it turns dy over, widens q and splits fp32, four waves before the products of a half run and four after
// them. bf16 8 x 4095, 1024 x 4096: 335 us, where 8 x 4096 takes 318 on the other one.
#include "async_lds.h"
#include "layers_index.h"

namespace fftconv {
namespace lay {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

template <typename T> struct Operand { using type = T; static constexpr int PARTS = 1; };
template <> struct Operand<float> { using type = __bf16; static constexpr int PARTS = 3; };

struct WeightArgs {
    const void *dy;
    const int8_t *q;
    const float *scale;
    float *part;                  // (splits, O, C), for the sums of more than one range and for those put aside
    void *dw;
    int sequences, N, O, C, runs, tiles_c, tiles;
    int blocks, per;              // runs of all sequences; of one workgroup
    int splits;
};

__device__ __forceinline__ f32x16 mfma16(uint4 a, uint4 b, f32x16 c, __bf16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma16(uint4 a, uint4 b, f32x16 c, _Float16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Place in LDS of piece c (8 samples, 16 bytes) of a row of 64: moved by bits 0-2 and 3-4 of the row, so that neither the eight rows that an
// operand's read takes at once nor the transposed pieces that sixteen lanes write at once meet in a bank.
__device__ __forceinline__ int place(int row, int c) { return row * 128 + ((c ^ ((row ^ ((row >> 3) & 3)) & 7)) << 4); }

// One 16-bit part after the other of values in T. Of fp32 the upper 8 bits of the fraction each time, cut off rather than rounded: three times 8 are all
// 24, and no finite number becomes an infinity. An infinity is the first part alone.
template <typename T, typename P> __device__ __forceinline__ void split(const T &v, P (&o)[Operand<T>::PARTS])
{
    if constexpr (sizeof(T) == 2) {
        o[0] = v;
    } else {
        float left = v;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const uint32_t upper = __builtin_bit_cast(uint32_t, left) & 0xffff0000u;
            o[p] = __builtin_bit_cast(P, (uint16_t)(upper >> 16));
            left -= __builtin_bit_cast(float, upper);
            if (p == 0) left = magnitude(v) == 0x7f800000u ? 0.f : left;
        }
    }
}

// 16 whole numbers of eight bits as 16-bit ones, exactly, or as zeros: a Gate of a run's scale tells which, for where the scale is zero the values stand
// for zeros, whatever they are. It costs no instruction of the widening. bf16: the upper halves of the fp32 numbers, two put together by a permutation
// whose selector takes zeros instead. f16: q + 128 in the lowest bits of 1024 is 1024 + 128 + q, of which one multiply-add leaves q, or nothing.
template <typename T> struct Gate;
template <> struct Gate<__bf16> {
    uint32_t pick;
    __device__ __forceinline__ explicit Gate(float scale = 1.f) : pick(scale == 0.f ? 0x0c0c0c0cu : 0x07060302u) {}
    __device__ __forceinline__ void widen(uint4 v, uint4 (&o)[2]) const
    {
        int8_t q[16];
        __builtin_memcpy(q, &v, 16);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, (float)q[2 * i + 1]), __builtin_bit_cast(uint32_t, (float)q[2 * i]), pick);
        o[0] = make_uint4(w[0], w[1], w[2], w[3]);
        o[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
};
template <> struct Gate<_Float16> {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
    f16x2 by, less;
    __device__ __forceinline__ explicit Gate(float scale = 1.f)
    {
        by = scale == 0.f ? f16x2{0, 0} : f16x2{1, 1};
        less = scale == 0.f ? f16x2{0, 0} : f16x2{-1152, -1152};
    }
    __device__ __forceinline__ void widen(uint4 v, uint4 (&o)[2]) const
    {
        const uint32_t q[4] = {v.x ^ 0x80808080u, v.y ^ 0x80808080u, v.z ^ 0x80808080u, v.w ^ 0x80808080u};
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t t = __builtin_amdgcn_perm(0x64646464u, q[i / 2], i % 2 ? 0x04030402u : 0x04010400u);
            w[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, t), by, less));
        }
        o[0] = make_uint4(w[0], w[1], w[2], w[3]);
        o[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
};

// 16 bytes from p, of which the first `left` are wanted and the others read as zero, without reading beyond `end` (the tensor's, which has 16
// bytes at least): what lies too near the end comes from the last 16 bytes, moved down.
__device__ __forceinline__ uint4 load_edge(const char *p, const char *end, int64_t left)
{
    const char *const from = p + 16 <= end ? p : end - 16;
    const int64_t off = p - from;
    unsigned __int128 v;
    __builtin_memcpy(&v, from, 16);
    v = left <= 0 ? 0 : v >> (8 * (off < 15 ? off : 15));
    if (left < 16) v &= ((unsigned __int128)1 << (8 * (left > 0 ? left : 0))) - 1;
    uint4 r;
    __builtin_memcpy(&r, &v, 16);
    return r;
}
template <typename T> __device__ __forceinline__ uint4 load_whole(const T *p, uint32_t bytes)
{
    uint4 r;
    __builtin_memcpy(&r, __builtin_assume_aligned((const char *)p + bytes, alignof(T)), 16);
    return r;
}

// A wave's sums, in full, to dw (rounded) or to its range's part, on top of those put aside before. Lane l holds channel l % 32 and, in
// register i, output 8 (i / 4) + 4 (l / 32) + i % 4; o1, c1: this lane's first.
template <typename DW, int FO, int FC> __device__ __forceinline__ void store_sums(const WeightArgs &a, const f32x16 (&acc)[FO][FC], const float (&unit)[FC],
                                                                                  float *part, bool aside, bool rounded, int o1, int c1)
{
    asm volatile("" : "+v"(o1), "+v"(c1));                 // (else the compiler keeps all addresses below in registers throughout the sums)
#pragma unroll
    for (int i = 0; i < FO; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) {
            __builtin_amdgcn_sched_barrier(0);             // one accumulator at a time: addresses of all would fill the registers
            const int c = c1 + j * 32;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int o = o1 + i * 32 + 8 * (e / 4) + e % 4;
                if (o >= a.O || c >= a.C) continue;
                const int64_t at = (int64_t)o * a.C + c;
                float v = acc[i][j][e] * unit[j];
                if (aside) v += part[at];
                if (rounded) ((DW *)a.dw)[at] = from_f32<DW>(v);
                else part[at] = v;
            }
        }
}

template <typename T, bool TOKENS, typename DW, int FO, int FC> __global__ void __launch_bounds__(512, 2) k_weight(const WeightArgs a)
{
    using P = typename Operand<T>::type;
    constexpr int NP = Operand<T>::PARTS, BO = 64 * FO, BC = 128 * FC;       // 2 x 4 waves of FO x FC accumulators
    constexpr int STAGE = (BO * NP + BC) * 128;
    extern __shared__ __align__(16) char lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int wo = __builtin_amdgcn_readfirstlane(wave >> 2), wc = wave & 3;
    // workgroups go to the dies in turn; a die takes neighbouring tiles of one range, which read the same dy and q from its L2
    const int n_wg = gridDim.x, die = blockIdx.x % 8, spare = n_wg % 8;
    const int at = die * (n_wg / 8) + min(die, spare) + blockIdx.x / 8;
    const int tile = at % a.tiles, range = at / a.tiles;
    const int o0 = tile / a.tiles_c * BO, c0 = tile % a.tiles_c * BC;
    const int first = range * a.per, last = min(first + a.per, a.blocks);

    // What a thread stages of 64 samples. dy (b, o, n): pieces of 8 samples, eight to a row. dy (b, n, o): pieces of 8 channels x 4 samples;
    // bits 0-1 and 4 up of a piece's number are the channels', so that four lanes read 64 bytes in a row, bits 2 and 3 the lowest and the
    // highest bit of the samples', so that sixteen lanes write 128 bytes of different banks. q: pieces of 16 samples, four to a row.
    constexpr int AV = TOKENS ? (BO * 2 + 511) / 512 : BO * 8 / 512, AK = TOKENS ? 4 : 1, AW = sizeof(T) / 2, BV = BC * 4 / 512;
    constexpr int OH = BO / 64, OHB = OH == 4 ? 2 : 1, EA = 16 / sizeof(T);
    static_assert(OH == 4 || OH == 2, "tile");
    auto group_o = [](int p) { return (p & 3) | ((p >> 4) & (2 * OH - 1)) << 2; };
    auto group_k = [](int p) { return ((p >> 2) & 1) | ((p >> (5 + OHB)) & 3) << 1 | ((p >> 3) & 1) << 3; };
    uint4 da[AV][AK][AW], db[BV];
    // Distances, in bytes, from the first value of a step's tile. Rows beyond the end are the last one's: what comes of them is not stored.
    uint32_t aat[AV], bat[BV];
#pragma unroll
    for (int i = 0; i < AV; ++i) {
        const int p = threadIdx.x + i * 512;
        if constexpr (TOKENS) aat[i] = ((uint32_t)(group_k(p) * 4) * a.O + (o0 + group_o(p) * 8 < a.O ? group_o(p) * 8 : 0)) * sizeof(T);
        else aat[i] = ((uint32_t)(min(o0 + (p >> 3), a.O - 1) - o0) * (uint32_t)a.N + (p & 7) * 8) * sizeof(T);
    }
#pragma unroll
    for (int i = 0; i < BV; ++i) {
        const int p = threadIdx.x + i * 512;
        bat[i] = (uint32_t)(min(c0 + (p >> 2), a.C - 1) - c0) * (uint32_t)a.N + (p & 3) * 16;
    }
    // half h of a run
    auto fetch = [&](int blk, int h) {
        const int b = blk / a.runs, j = blk - b * a.runs;
        const int n0 = j * RUN + h * 64;
        const T *const dy = (const T *)a.dy + (TOKENS ? ((int64_t)b * a.N + n0) * a.O + o0 : ((int64_t)b * a.O + o0) * a.N + n0);
        const int8_t *const q = a.q + ((int64_t)b * a.C + c0) * a.N + n0;
        if (whole_half_run(n0, a.N, a.O, TOKENS)) {
#pragma unroll
            for (int i = 0; i < AV; ++i) {
                if (TOKENS && threadIdx.x + i * 512 >= BO * 2) continue;
#pragma unroll
                for (int r = 0; r < AK; ++r)
#pragma unroll
                    for (int w = 0; w < AW; ++w) da[i][r][w] = load_whole(dy + (int64_t)r * a.O + w * EA, aat[i]);
            }
#pragma unroll
            for (int i = 0; i < BV; ++i) db[i] = load_whole(q, bat[i]);
        } else {
            const char *const dy_end = (const char *)a.dy + (int64_t)a.sequences * a.O * a.N * (int64_t)sizeof(T);
            const char *const q_end = (const char *)a.q + (int64_t)a.sequences * a.C * a.N;
#pragma unroll
            for (int i = 0; i < AV; ++i) {
                const int p = threadIdx.x + i * 512;
                if (TOKENS && p >= BO * 2) continue;
#pragma unroll
                for (int r = 0; r < AK; ++r)
#pragma unroll
                    for (int w = 0; w < AW; ++w) {
                        const int o = TOKENS ? group_o(p) * 8 + w * EA : p >> 3, n = TOKENS ? group_k(p) * 4 + r : (p & 7) * 8 + w * EA;
                        const int64_t left = TOKENS ? (n0 + n < a.N ? a.O - o0 - o : 0) : (o0 + o < a.O ? a.N - n0 - n : 0);
                        da[i][r][w] = load_edge((const char *)(dy + (TOKENS ? (int64_t)n * a.O + o : (int64_t)o * a.N + n)), dy_end, left * (int)sizeof(T));
                    }
            }
#pragma unroll
            for (int i = 0; i < BV; ++i) {
                const int p = threadIdx.x + i * 512;
                db[i] = load_edge((const char *)(q + bat[i]), q_end, a.N - n0 - (p & 3) * 16);
            }
        }
    };
    auto keep = [&](int buf) {
        char *const base = lds + buf * STAGE;
#pragma unroll
        for (int i = 0; i < AV; ++i) {
            const int p = threadIdx.x + i * 512;
            if constexpr (TOKENS) {
                if (p >= BO * 2) continue;
                const int og = group_o(p), kg = group_k(p);
                int at = place(og * 8, kg >> 1) + (kg & 1) * 8;          // row og 8 + e: bits 4-6 turned by e
                asm volatile("" : "+v"(at));                             // (one address kept, not eight)
                T v[4][8];
                __builtin_memcpy(v, da[i], sizeof(v));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    P o[4][NP];
#pragma unroll
                    for (int r = 0; r < 4; ++r) split<T, P>(v[r][e], o[r]);
#pragma unroll
                    for (int s = 0; s < NP; ++s) {
                        const P t[4] = {o[0][s], o[1][s], o[2][s], o[3][s]};
                        __builtin_memcpy(__builtin_assume_aligned(base + s * BO * 128 + e * 128 + (at ^ (e << 4)), 8), t, 8);
                    }
                }
            } else {
                T v[8];
                __builtin_memcpy(v, da[i], sizeof(v));
                P o[8][NP];
#pragma unroll
                for (int e = 0; e < 8; ++e) split<T, P>(v[e], o[e]);
#pragma unroll
                for (int s = 0; s < NP; ++s) {
                    P t[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) t[e] = o[e][s];
                    __builtin_memcpy(__builtin_assume_aligned(base + s * BO * 128 + place(p >> 3, p & 7), 16), t, 16);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BV; ++i) {
            const int p = threadIdx.x + i * 512;
            uint4 t[2];
            Gate<P>().widen(db[i], t);
#pragma unroll
            for (int h = 0; h < 2; ++h) *(uint4 *)(base + NP * BO * 128 + place(p >> 2, (p & 3) * 2 + h)) = t[h];
        }
    };

    // the scales of this lane's channels
    int sat[FC];
#pragma unroll
    for (int j = 0; j < FC; ++j) sat[j] = min(c0 + (wc * FC + j) * 32 + l32, a.C - 1);
    float s[FC];
    auto scales = [&](int blk) {
        const int b = blk / a.runs;
        const float *const p = a.scale + (int64_t)b * a.C * a.runs + (blk - b * a.runs);
#pragma unroll
        for (int j = 0; j < FC; ++j) s[j] = p[(int64_t)sat[j] * a.runs];
    };
    int blk = first;
    if (blk < last) {
        fetch(blk, 0);
        scales(blk);
        keep(0);
        fetch(blk, 1);
        lds_barrier();
    }
    float *const part = a.part + (int64_t)range * a.O * a.C;
    // this lane's first pieces of either operand; piece 2 kk + half is at (... ^ kk << 5)
    const int ro = place(wo * FO * 32 + l32, half), rc = NP * BO * 128 + place(wc * FC * 32 + l32, half);
    bool aside = false;
    do {
        f32x16 acc[FO][FC] = {};
        float unit[FC] = {}, top[FC] = {};         // the scale that the sums are in units of, and the largest so far
        uint32_t zeros = 0;                        // bit j: the run's scale is zero, and so is what its q stands for, whatever that is
        auto products = [&](int buf) {
            if (__builtin_amdgcn_ballot_w64(zeros != 0) != 0) {        // every lane clears what it reads below (two waves the same places)
#pragma unroll
                for (int j = 0; j < FC; ++j) {
                    if (zeros >> j & 1) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) *(uint4 *)(lds + buf * STAGE + (rc ^ (kk << 5)) + j * 32 * 128) = make_uint4(0, 0, 0, 0);
                    }
                }
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const char *const pc = lds + buf * STAGE + (rc ^ (kk << 5)), *const po = lds + buf * STAGE + (ro ^ (kk << 5));
                uint4 fc[FC];
#pragma unroll
                for (int j = 0; j < FC; ++j) fc[j] = *(const uint4 *)(pc + j * 32 * 128);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {        // the smallest parts first
#pragma unroll
                    for (int i = 0; i < FO; ++i) {
                        const uint4 fo = *(const uint4 *)(po + (p * BO + i * 32) * 128);
#pragma unroll
                        for (int j = 0; j < FC; ++j) acc[i][j] = mfma16(fo, fc[j], acc[i][j], P());
                    }
                }
            }
        };
        for (; blk < last; ++blk) {
            // units so much smaller that the sums might leave fp32's range: the sums so far are put aside
            bool small = false;
#pragma unroll
            for (int j = 0; j < FC; ++j) small |= s[j] != 0.f && fabsf(s[j]) < top[j] * 0x1p-60f;
            if (__builtin_amdgcn_ballot_w64(small) != 0) break;
            zeros = 0;
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                // a run of zeros keeps the units; so do the first sums
                zeros |= (s[j] == 0.f ? 1u : 0u) << j;
                const float f = s[j] == 0.f || unit[j] == 0.f ? 1.f : unit[j] / s[j];
                unit[j] = s[j] == 0.f ? unit[j] : s[j];
                top[j] = fmaxf(top[j], fabsf(unit[j]));
#pragma unroll
                for (int i = 0; i < FO; ++i) acc[i][j] *= f;
            }
            // Each half run: what was asked for a half run ago goes to LDS and the next is asked for, on four waves before the products of the
            // half run that is there and on four after them, so that on each SIMD one wave's conversions run beside the other's products.
            const int next = min(blk + 1, last - 1);       // (the last run once more at the end, not used)
            if (wo == 0) keep(1), fetch(next, 0);
            products(0);
            if (wo != 0) keep(1), fetch(next, 0);
            lds_barrier();
            scales(next);
            if (wo == 0) keep(0), fetch(next, 1);
            products(1);
            if (wo != 0) keep(0), fetch(next, 1);
            lds_barrier();
        }
        store_sums<DW, FO, FC>(a, acc, unit, part, aside, a.splits == 1 && blk >= last, o0 + wo * FO * 32 + 4 * half, c0 + wc * FC * 32 + l32);
        aside = true;
    } while (blk < last);
}

// The same for 16-bit dy with everything in pieces of 16 bytes (samples a multiple of 16, channels of dy of 8): tiles go from memory straight
// to LDS, three half runs ahead of the products, as they lie there. dy (b, n, o) is turned over on its way from LDS into the operand: a transposing
// read gives lane i of sixteen the i-th of 16 channels of four samples, each four lanes having pointed at a sample's 16 channels. q is widened
// there too.
//
// Samples of a half run, as operands want them (8 for a lane of either half of the wave): pair u of products, product v of it, takes
// 32 u + 16 half + 8 v ..., so that one read of 16 bytes of q serves both.
//
// Measured: bf16 64 x 4096, 2304 x 768: 0.99 ms and 11 us for the sums, 0.92 PFLOP/s; back to back the socket is at 1382 of 1400 W. Under the profiler,
// which pauses between launches, 0.91 ms at 2.25 GHz, the matrix cores busy 43 % of it and other vector instructions' issue 42. The products alone take
// 574 us (1.6 PFLOP/s); what is brought costs 225 us (70 of them because it comes from beyond the L2), widening q 115, the quotients of the scales 72,
// reading dy from LDS 55: each leaves when it is left out, and waits cost nothing. Taking turns (one wave of a SIMD reads and widens while the other multiplies, a barrier at each turn) was slower, 1.14 ms.
typedef __attribute__((ext_vector_type(4))) short s16x4;
__device__ __forceinline__ uint2 read_transposed(const char *p)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}
template <typename T, bool TOKENS, typename DW, int FO, int FC> __global__ void __launch_bounds__(512, 2) k_weight_async(const WeightArgs a)
{
    constexpr int BO = 64 * FO, BC = 128 * FC, Q_AT = BO * 128, S_AT = Q_AT + BC * 64, STAGE = S_AT + 8 * 256, STAGES = 3;
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int wo = wave >> 2, wc = wave & 3;
    const int n_wg = gridDim.x, die = blockIdx.x % 8, spare = n_wg % 8;
    const int at = die * (n_wg / 8) + min(die, spare) + blockIdx.x / 8;
    const int tile = at % a.tiles, range = at / a.tiles;
    const int o0 = tile / a.tiles_c * BO, c0 = tile % a.tiles_c * BC;
    const int first = range * a.per, last = min(first + a.per, a.blocks);

    // What this lane brings to LDS. dy (b, n, o): rows of BO channels of a sample, their 16-byte pieces moved in pairs by the sample, so that the
    // four samples of a transposing read lie in banks of their own. dy (b, o, n): rows of 64 samples of a channel, pieces moved by
    // the pair of channels (256 bytes, what a clock delivers). q: rows of 64 bytes, pieces moved by the four channels. Channels beyond the end read others: what comes of them is not stored.
    constexpr int LR = BO / 8;                                   // lanes to a row of (b, n, o)
    uint32_t aat[FO], bat[FC];
    int an[FO], bn[FC];                                          // this lane's first sample
#pragma unroll
    for (int i = 0; i < FO; ++i) {
        const int p = (wave * FO + i) * 64 + lane;
        if constexpr (TOKENS) {
            const int n = p / LR, m = n & 3, piece = (p % LR) ^ (2 * (m ^ (m << 1)));
            an[i] = n;
            aat[i] = ((uint32_t)n * (uint32_t)a.O + (o0 + piece * 8 < a.O ? piece * 8 : 0)) * 2;
        } else {
            const int o = p >> 3, piece = (p & 7) ^ ((o >> 1) & 7);
            an[i] = piece * 8;
            aat[i] = ((uint32_t)(min(o0 + o, a.O - 1) - o0) * (uint32_t)a.N + piece * 8) * 2;
        }
    }
#pragma unroll
    for (int i = 0; i < FC; ++i) {
        const int p = (wave * FC + i) * 64 + lane, c = p >> 2, piece = (p & 3) ^ ((c >> 2) & 3);
        bn[i] = piece * 16;
        bat[i] = (uint32_t)(min(c0 + c, a.C - 1) - c0) * (uint32_t)a.N + piece * 16;
    }
    // lane i of a wave's scales is channel i of its 64 (FC = 2) or 32 (FC = 1, twice)
    const uint32_t sat = (uint32_t)(min(c0 + wc * FC * 32 + (FC == 2 ? lane : l32), a.C - 1) - c0) * (uint32_t)a.runs * 4;

    // What is asked for next: the half run from sample `at_n` of sequence `at_b` on (kept, not divided out of the run's number each time).
    const int b0 = first / a.runs;
    int at_b = b0, at_n = (first - b0 * a.runs) * RUN, left = 2 * (last - first);
    const int64_t dy_step = TOKENS ? (int64_t)a.O * 128 : 128;
    const char *dy, *q, *sc;
    auto from_start = [&] {
        dy = ((const char *)a.dy + (TOKENS ? ((int64_t)at_b * a.N + at_n) * a.O + o0 : ((int64_t)at_b * a.O + o0) * a.N + at_n) * 2);
        q = ((const char *)a.q + ((int64_t)at_b * a.C + c0) * a.N + at_n);
        sc = ((const char *)(a.scale + ((int64_t)at_b * a.C + c0) * a.runs + at_n / RUN));
    };
    from_start();
    // (beyond the range's end its last half run once more, not used)
    auto fetch = [&](int h, int stage) {
        const char *const to = lds + stage * STAGE;
        // (the same in all lanes, which the compiler cannot tell)
        dy = uniform(dy), q = uniform(q), sc = uniform(sc);
        if (at_n + 64 <= a.N) {
#pragma unroll
            for (int i = 0; i < FO; ++i) to_lds16(dy, aat[i], to + (wave * FO + i) * 1024);
#pragma unroll
            for (int i = 0; i < FC; ++i) to_lds16(q, bat[i], to + Q_AT + (wave * FC + i) * 1024);
        } else {                                                 // samples beyond the end are zeros
            const char *const zero = (const char *)&zero_piece;
#pragma unroll
            for (int i = 0; i < FO; ++i) to_lds16(at_n + an[i] < a.N ? dy + aat[i] : zero, to + (wave * FO + i) * 1024);
#pragma unroll
            for (int i = 0; i < FC; ++i) to_lds16(at_n + bn[i] < a.N ? q + bat[i] : zero, to + Q_AT + (wave * FC + i) * 1024);
        }
        if (h == 0) to_lds4(sc, sat, to + S_AT + wave * 256);
        if (--left <= 0) return;
        if (h == 0 || at_n + 64 < a.N) {
            at_n += 64, dy += dy_step, q += 64;
            if (h) sc += 4;
        } else {
            at_n = 0, ++at_b;
            from_start();
        }
    };

    // where this lane reads its operands, from a stage's start
    int ra[TOKENS ? FO : 1];
    if constexpr (TOKENS) {
        const int j = lane & 15, m = j >> 2;
#pragma unroll
        for (int i = 0; i < FO; ++i) {
            const int piece = ((wo * FO + i) * 4 + 2 * ((lane >> 4) & 1) + ((j & 3) >> 1)) ^ (2 * (m ^ (m << 1)));
            ra[i] = (16 * half + m) * BO * 2 + piece * 16 + (j & 1) * 8;
        }
    } else {
        ra[0] = (wo * FO * 32 + l32) * 128 + (((2 * half) ^ ((l32 >> 1) & 7)) << 4);
    }
    const int rq = Q_AT + (wc * FC * 32 + l32) * 64 + ((half ^ ((l32 >> 2) & 3)) << 4);

    // The operands of the products of a half run, in four groups 2 u + v: of dy one group ahead of its products, of q a pair of groups.
    uint4 fo[2][FO], fc[2][FC][2], raw[FC];
    auto read_dy = [&](const char *base, int g) {
        const int u = g >> 1, v = g & 1;
#pragma unroll
        for (int i = 0; i < FO; ++i) {
            if constexpr (TOKENS) {
                const char *const p = base + ra[i] + (32 * u + 8 * v) * BO * 2;
                const uint2 x = read_transposed(p), y = read_transposed(p + 4 * BO * 2);
                fo[g & 1][i] = make_uint4(x.x, x.y, y.x, y.y);
            } else {
                fo[g & 1][i] = *(const uint4 *)(base + (ra[0] ^ (u << 6 | v << 4)) + i * 32 * 128);
            }
        }
    };
    auto read_q = [&](const char *base, int u) {
#pragma unroll
        for (int j = 0; j < FC; ++j) raw[j] = *(const uint4 *)(base + (rq ^ (u << 5)) + j * 32 * 64);
    };
    float s[FC] = {};                                            // this lane's scales of the run whose q is widened next
    Gate<T> gate[FC];
    auto widen_q = [&](int u) {
#pragma unroll
        for (int j = 0; j < FC; ++j) gate[j].widen(raw[j], fc[u][j]);
    };
    float *const part = a.part + (int64_t)range * a.O * a.C;
    bool aside = false;
    int blk = first, stage = 0;
    auto read_scales = [&](const char *base) {
#pragma unroll
        for (int j = 0; j < FC; ++j) {
            s[j] = *(const float *)(base + S_AT + wave * 256 + (j * 32 + l32) * 4);
            gate[j] = Gate<T>(s[j]);
        }
    };
    if (blk < last) {
        fetch(0, 0);
        fetch(1, 1);
        fetch(0, 2);
        FC_ARRIVED(2 * (FO + FC) + 1);
        read_scales(lds);
        read_dy(lds, 0);
        read_q(lds, 0);
        widen_q(0);
    }
    do {
        f32x16 acc[FO][FC] = {};
        float unit[FC] = {}, top[FC] = {};
        auto products = [&](int g) {
#pragma unroll
            for (int i = 0; i < FO; ++i)
#pragma unroll
                for (int j = 0; j < FC; ++j) acc[i][j] = mfma16(fo[g & 1][i], fc[g >> 1][j][g & 1], acc[i][j], T());
        };
        // The products of the half run at `stage`. Before the last group every wave has read all of it, and the next half run has arrived: beside that
        // group the next one's first operands are read, and what comes three half runs later is asked for, to the same place.
        auto half_run = [&](auto second) {
            constexpr int H = decltype(second)::value;
            const char *const base = lds + stage * STAGE;
            read_dy(base, 1);
            read_q(base, 1);
            __builtin_amdgcn_sched_barrier(0);
            products(0);
            __builtin_amdgcn_sched_barrier(0);
            read_dy(base, 2);
            __builtin_amdgcn_sched_barrier(0);
            widen_q(1);
            products(1);
            __builtin_amdgcn_sched_barrier(0);
            read_dy(base, 3);
            __builtin_amdgcn_sched_barrier(0);
            products(2);
            __builtin_amdgcn_sched_barrier(0);
            FC_ARRIVED(FO + FC + (H ? 0 : 1));                   // on its way may be the half run after the next
            const int free = stage;
            stage = stage + 1 < STAGES ? stage + 1 : 0;
            const char *const next = lds + stage * STAGE;
            if constexpr (H) read_scales(next);
            read_dy(next, 0);
            read_q(next, 0);
            __builtin_amdgcn_sched_barrier(0);
            fetch(1 - H, free);
            widen_q(0);
            products(3);
            __builtin_amdgcn_sched_barrier(0);
        };
        for (; blk < last; ++blk) {
            bool small = false;
#pragma unroll
            for (int j = 0; j < FC; ++j) small |= s[j] != 0.f && fabsf(s[j]) < top[j] * 0x1p-60f;
            if (__builtin_amdgcn_ballot_w64(small) != 0) break;
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                const float f = s[j] == 0.f || unit[j] == 0.f ? 1.f : unit[j] / s[j];
                unit[j] = s[j] == 0.f ? unit[j] : s[j];
                top[j] = fmaxf(top[j], fabsf(unit[j]));
#pragma unroll
                for (int i = 0; i < FO; ++i) acc[i][j] *= f;
            }
            half_run(std::integral_constant<int, 0>());
            half_run(std::integral_constant<int, 1>());
        }
        store_sums<DW, FO, FC>(a, acc, unit, part, aside, a.splits == 1 && blk >= last, o0 + wo * FO * 32 + 4 * half, c0 + wc * FC * 32 + l32);
        aside = true;
        // stores count as the transfers do; and nothing is on its way to LDS when the workgroup ends
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } while (blk < last);
}

// Tensors of less than the 16 bytes that a load of the kernel above takes (a handful of values): a thread for each of dw's.
template <typename T, bool TOKENS, typename DW> __global__ void __launch_bounds__(64) k_weight_tiny(const WeightArgs a, int64_t first)
{
    const int64_t i = (first + blockIdx.x) * 64 + threadIdx.x;
    if (i >= (int64_t)a.O * a.C) return;
    const int64_t o = i / a.C, c = i - o * a.C;
    float sum = 0.f;
    for (int64_t b = 0; b < a.sequences; ++b)
        for (int64_t n = 0; n < a.N; ++n) {
            const float x = (float)a.q[(b * a.C + c) * a.N + n] * a.scale[(b * a.C + c) * a.runs + n / RUN];
            sum = fmaf(to_f32(((const T *)a.dy)[TOKENS ? (b * a.N + n) * a.O + o : (b * a.O + o) * a.N + n]), x, sum);
        }
    ((DW *)a.dw)[i] = from_f32<DW>(sum);
}

template <typename DW> __global__ void __launch_bounds__(256) k_sum_ranges(const float *__restrict__ part, DW *__restrict__ dw, int splits, int64_t n)
{
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        float s[4];
        load_piece<float, 4>(part + i, n - i, s);
        int k = 1;
        for (; k + 4 <= splits; k += 4) {                  // four loads of a thread on their way at once
            float t[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) load_piece<float, 4>(part + (k + j) * n + i, n - i, t[j]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] += t[j][e];
        }
        for (; k < splits; ++k) {
            float t[4];
            load_piece<float, 4>(part + k * n + i, n - i, t);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += t[e];
        }
        store_rounded<DW, 4>(dw + i, n - i, s);
    }
}

// The tile, and into how many ranges the runs go: as many as fill the compute units once, with a workgroup each, or two of the smaller tile.
struct WeightShape { int fo, fc, splits, per; };
static WeightShape weight_shape(int64_t B, int64_t N, int64_t O, int64_t C, int dtype)
{
    WeightShape w;
    const bool small = dtype == FFTCONV_F32 || ((O + 255) / 256) * ((C + 255) / 256) < 16;
    w.fo = small ? 2 : 4, w.fc = small ? 1 : 2;
    const int64_t tiles = ((O + 64 * w.fo - 1) / (64 * w.fo)) * ((C + 128 * w.fc - 1) / (128 * w.fc));
    const int64_t blocks = B > 0 ? B * ((N + RUN - 1) / RUN) : 1;        // (no sequence: one workgroup a tile writes the zeros)
    int64_t splits = 256 / tiles;
    // (a range of a few runs is over before a second workgroup helps: 2048 samples, 768 -> 768 took 19.5 us with one and 24.8 with two;
    // 1000 sequences of 17, 512 -> 512 take 178 us with two and took 271)
    if (small && dtype != FFTCONV_F32 && splits * 8 < blocks) splits = 512 / tiles;
    splits = splits < 1 ? 1 : splits > blocks ? blocks : splits;
    w.per = (int)((blocks + splits - 1) / splits);
    w.splits = (int)((blocks + w.per - 1) / w.per);
    return w;
}

size_t weight_grad_workspace(int64_t B, int64_t N, int64_t O, int64_t C, int dtype)
{
    return (size_t)weight_shape(B, N, O, C, dtype).splits * (size_t)O * (size_t)C * 4;
}

template <typename T, typename DW> static int run(const WeightShape &w, const WeightArgs &a, bool tokens, hipStream_t s)
{
    auto launch = [&](auto tok, auto fo, auto fc) -> int {
        constexpr int FO = decltype(fo)::value, FC = decltype(fc)::value, NP = Operand<T>::PARTS;
        if constexpr (NP == 1) {
            const bool pieces = a.N % 16 == 0 && (!tokens || a.O % 8 == 0) && ((uintptr_t)a.dy | (uintptr_t)a.q) % 16 == 0;
            if (pieces) {
                constexpr int lds = 3 * (64 * FO * 128 + 128 * FC * 64 + 8 * 256);
                const auto kernel = k_weight_async<T, decltype(tok)::value, DW, FO, FC>;
                FC_TRY(raise_dynamic_lds((const void *)kernel, lds));
                kernel<<<(unsigned)(a.tiles * a.splits), 512, lds, s>>>(a);
                FC_HIP(hipGetLastError());
                return FFTCONV_OK;
            }
        }
        constexpr int lds = 2 * (64 * FO * NP + 128 * FC) * 128;
        const auto kernel = k_weight<T, decltype(tok)::value, DW, FO, FC>;
        FC_TRY(raise_dynamic_lds((const void *)kernel, lds));
        kernel<<<(unsigned)(a.tiles * a.splits), 512, lds, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    };
    using Y = std::true_type;
    using No = std::false_type;
    if ((int64_t)a.sequences * a.N * a.O * (int64_t)sizeof(T) < 16 || (int64_t)a.sequences * a.N * a.C < 16) {
        return in_pieces(((int64_t)a.O * a.C + 63) / 64, 64, [&](int64_t at, unsigned g) -> int {
            if (tokens) k_weight_tiny<T, true, DW><<<g, 64, 0, s>>>(a, at);
            else k_weight_tiny<T, false, DW><<<g, 64, 0, s>>>(a, at);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    }
    if constexpr (sizeof(T) == 2) {
        if (w.fo == 4) {
            const std::integral_constant<int, 4> fo;
            const std::integral_constant<int, 2> fc;
            FC_TRY(tokens ? launch(Y(), fo, fc) : launch(No(), fo, fc));
        }
    }
    if (w.fo == 2) {
        const std::integral_constant<int, 2> fo;
        const std::integral_constant<int, 1> fc;
        FC_TRY(tokens ? launch(Y(), fo, fc) : launch(No(), fo, fc));
    }
    if (a.splits > 1) {
        const int64_t n = (int64_t)a.O * a.C, g = (n + 1023) / 1024;
        k_sum_ranges<DW><<<(unsigned)(g < 65536 ? g : 65536), 256, 0, s>>>(a.part, (DW *)a.dw, a.splits, n);
        FC_HIP(hipGetLastError());
    }
    return FFTCONV_OK;
}

int weight_grad(const void *dy, const int8_t *q, const float *scale, void *dw, int64_t B, int64_t N, int64_t O, int64_t C, bool tokens,
                int dtype_dy, int dtype_dw, void *workspace, hipStream_t s)
{
    const WeightShape w = weight_shape(B, N, O, C, dtype_dy);
    WeightArgs a = {};
    a.dy = dy, a.q = q, a.scale = scale, a.part = (float *)workspace, a.dw = dw, a.sequences = (int)B, a.N = (int)N, a.O = (int)O, a.C = (int)C;
    a.runs = (int)((N + RUN - 1) / RUN), a.blocks = (int)(B * a.runs), a.per = w.per, a.splits = w.splits;
    a.tiles_c = (int)((C + 128 * w.fc - 1) / (128 * w.fc)), a.tiles = (int)((O + 64 * w.fo - 1) / (64 * w.fo)) * a.tiles_c;
    auto by_dw = [&](auto t) -> int {
        using T = decltype(t);
        if (dtype_dw == FFTCONV_F32) return run<T, float>(w, a, tokens, s);
        if constexpr (sizeof(T) == 2) return run<T, T>(w, a, tokens, s);
        return FFTCONV_EUNSUPPORTED;
    };
    if (dtype_dy == FFTCONV_BF16) return by_dw(__bf16());
    if (dtype_dy == FFTCONV_F16) return by_dw(_Float16());
    return by_dw(float());
}

}  // namespace lay
}  // namespace fftconv
