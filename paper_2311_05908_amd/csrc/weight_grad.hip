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
#include "layers_internal.h"

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
    int64_t N;
    int O, C, runs, tiles_c;
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

// Place in LDS of piece c (8 samples, 16 bytes) of a row of 64: moved by the row, so that neither eight rows in a run (an operand's read) nor
// eight rows at steps of eight (the write of a transposed piece) meet in one bank.
__device__ __forceinline__ int place(int row, int c) { return row * 128 + ((c ^ ((row ^ (row >> 3)) & 7)) << 4); }

// One 16-bit part after the other of values in T.
template <typename T, typename P> __device__ __forceinline__ void split(const T &v, P (&o)[Operand<T>::PARTS])
{
    if constexpr (sizeof(T) == 2) {
        o[0] = v;
    } else {
        float left = v;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            o[p] = (P)left;
            left -= (float)o[p];
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
    const int wo = wave >> 2, wc = wave & 3;
    const int o0 = blockIdx.x / a.tiles_c * BO, c0 = blockIdx.x % a.tiles_c * BC;
    const int first = blockIdx.y * a.per, last = min(first + a.per, a.blocks);

    constexpr int AV = TOKENS ? (BO * 2 + 511) / 512 : BO * 8 / 512, AK = TOKENS ? 4 : 1;       // pieces of dy a thread stages; rows of a piece
    constexpr int BV = BC * 4 / 512;
    // TOKENS: a piece is 8 channels x 4 samples. Bits 0-2 of its number are the channels', so that eight lanes read 128 bytes in a row, and bit 3
    // the samples', so that sixteen lanes write 128 bytes of different banks.
    constexpr int OH = BO / 64, OHB = OH == 4 ? 2 : 1;
    static_assert(OH == 4 || OH == 2, "tile");
    auto group_o = [](int p) { return (p & 7) | ((p >> 4) & (OH - 1)) << 3; };
    auto group_k = [](int p) { return ((p >> 3) & 1) | (p >> (4 + OHB)) << 1; };
    T da[AV][AK][8];
    uint4 db[BV];
    // step 2 i + h is half h of run first + i
    auto fetch = [&](int step) {
        const int blk = first + (step >> 1), b = blk / a.runs, j = blk - b * a.runs;
        const int64_t n0 = (int64_t)j * RUN + (step & 1) * 64;
#pragma unroll
        for (int i = 0; i < AV; ++i) {
            const int p = threadIdx.x + i * 512;
            if constexpr (TOKENS) {
                if (p >= BO * 2) continue;
                const int og = group_o(p), kg = group_k(p);
                const int o = o0 + og * 8;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t n = n0 + kg * 4 + r;
                    const int left = n < a.N ? a.O - o : 0;
                    const T *const src = (const T *)a.dy + ((int64_t)b * a.N + n) * a.O + o;
                    if (left >= 8) {
                        __builtin_memcpy(da[i][r], src, sizeof(da[i][r]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) da[i][r][e] = e < left ? src[e] : (T)0.f;
                    }
                }
            } else {
                const int o = o0 + (p >> 3);
                const int64_t n = n0 + (p & 7) * 8, left = o < a.O ? a.N - n : 0;
                const T *const src = (const T *)a.dy + ((int64_t)b * a.O + o) * a.N + n;
                if (left >= 8) {
                    __builtin_memcpy(da[i][0], src, sizeof(da[i][0]));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) da[i][0][e] = e < left ? src[e] : (T)0.f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BV; ++i) {
            const int p = threadIdx.x + i * 512, c = c0 + (p >> 2);
            const int64_t n = n0 + (p & 3) * 16, left = c < a.C ? a.N - n : 0;
            const int8_t *const src = a.q + ((int64_t)b * a.C + c) * a.N + n;
            db[i] = make_uint4(0, 0, 0, 0);
            if (left >= 16) {
                __builtin_memcpy(&db[i], src, 16);
            } else if (left > 0) {
                uint32_t w[4] = {};
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (e < left) w[e / 4] |= (uint32_t)(uint8_t)src[e] << (8 * (e % 4));
                db[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    };
    auto keep = [&](int buf) {
        char *const base = lds + buf * STAGE;
#pragma unroll
        for (int i = 0; i < AV; ++i) {
            const int p = threadIdx.x + i * 512;
            if constexpr (TOKENS) {
                const int og = group_o(p), kg = group_k(p);
                if (p >= BO * 2) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    P o[4][NP];
#pragma unroll
                    for (int r = 0; r < 4; ++r) split<T, P>(da[i][r][e], o[r]);
#pragma unroll
                    for (int s = 0; s < NP; ++s) {
                        const P v[4] = {o[0][s], o[1][s], o[2][s], o[3][s]};
                        __builtin_memcpy(base + s * BO * 128 + place(og * 8 + e, kg >> 1) + (kg & 1) * 8, v, 8);
                    }
                }
            } else {
                P o[8][NP];
#pragma unroll
                for (int e = 0; e < 8; ++e) split<T, P>(da[i][0][e], o[e]);
#pragma unroll
                for (int s = 0; s < NP; ++s) {
                    P v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = o[e][s];
                    __builtin_memcpy(base + s * BO * 128 + place(p >> 3, p & 7), v, 16);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BV; ++i) {
            const int p = threadIdx.x + i * 512;
            int8_t q[16];
            __builtin_memcpy(q, &db[i], 16);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                P v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (P)(float)q[h * 8 + e];
                __builtin_memcpy(base + NP * BO * 128 + place(p >> 2, (p & 3) * 2 + h), v, 16);
            }
        }
    };

    f32x16 acc[FO][FC] = {};
    float unit[FC] = {}, top[FC] = {};             // the scale that the sums are in units of; the largest since they were last put aside
    bool aside = false;
    float *const part = a.part + (int64_t)blockIdx.y * a.O * a.C;
    // sums in full units to `put`; lane l holds channel l % 32 and, in register i, output 8 (i / 4) + 4 (l / 32) + i % 4
    auto each = [&](auto put) {
#pragma unroll
        for (int i = 0; i < FO; ++i)
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                __builtin_amdgcn_sched_barrier(0);          // one accumulator at a time: addresses of all would fill the registers
                const int c = c0 + (wc * FC + j) * 32 + l32;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int o = o0 + (wo * FO + i) * 32 + 8 * (e / 4) + 4 * half + e % 4;
                    if (o < a.O && c < a.C) put((int64_t)o * a.C + c, acc[i][j][e] * unit[j]);
                }
            }
    };
    const int steps = 2 * (last - first);
    if (steps > 0) {
        fetch(0);
        keep(0);
        lds_barrier();
    }
    for (int k = 0; k < steps; ++k) {
        if (k + 1 < steps) fetch(k + 1);
        if ((k & 1) == 0) {
            const int blk = first + (k >> 1), b = blk / a.runs, j0 = blk - b * a.runs;
            float s[FC];
            bool small = false;
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                const int c = min(c0 + (wc * FC + j) * 32 + l32, a.C - 1);
                s[j] = a.scale[((int64_t)b * a.C + c) * a.runs + j0];
                small |= s[j] > 0.f && s[j] < top[j] * 0x1p-60f;
            }
            if (__any(small)) {                    // units so much smaller that the sums might leave fp32's range: the sums are put aside
                each([&](int64_t at, float v) { part[at] = aside ? part[at] + v : v; });
                aside = true;
#pragma unroll
                for (int j = 0; j < FC; ++j) {
                    unit[j] = top[j] = 0.f;
#pragma unroll
                    for (int i = 0; i < FO; ++i) acc[i][j] = 0.f;
                }
            }
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                // a run of zeros keeps the units; so do the first sums
                const float f = s[j] == 0.f || unit[j] == 0.f ? 1.f : unit[j] / s[j];
                unit[j] = s[j] == 0.f ? unit[j] : s[j];
                top[j] = fmaxf(top[j], unit[j]);
#pragma unroll
                for (int i = 0; i < FO; ++i) acc[i][j] *= f;
            }
        }
        const char *const base = lds + (k & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            uint4 fc[FC];
#pragma unroll
            for (int j = 0; j < FC; ++j) fc[j] = *(const uint4 *)(base + NP * BO * 128 + place((wc * FC + j) * 32 + l32, kk * 2 + half));
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) {    // the smallest parts first
#pragma unroll
                for (int i = 0; i < FO; ++i) {
                    const uint4 fo = *(const uint4 *)(base + p * BO * 128 + place((wo * FO + i) * 32 + l32, kk * 2 + half));
#pragma unroll
                    for (int j = 0; j < FC; ++j) acc[i][j] = mfma16(fo, fc[j], acc[i][j], P());
                }
            }
        }
        if (k + 1 < steps) {
            keep((k + 1) & 1);
            lds_barrier();
        }
    }
    if (a.splits > 1) each([&](int64_t at, float v) { part[at] = aside ? part[at] + v : v; });
    else each([&](int64_t at, float v) { ((DW *)a.dw)[at] = from_f32<DW>(aside ? part[at] + v : v); });
}

template <typename DW> __global__ void __launch_bounds__(256) k_sum_ranges(const float *__restrict__ part, DW *__restrict__ dw, int splits, int64_t n)
{
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        float s[4];
        load_piece<float, 4>(part + i, n - i, s);
        for (int k = 1; k < splits; ++k) {
            float t[4];
            load_piece<float, 4>(part + k * n + i, n - i, t);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += t[e];
        }
        store_rounded<DW, 4>(dw + i, n - i, s);
    }
}

// The tile, and into how many ranges the runs go: as many as fill the compute units once, a workgroup each.
struct WeightShape { int fo, fc, splits, per; };
static WeightShape weight_shape(int64_t B, int64_t N, int64_t O, int64_t C, int dtype)
{
    WeightShape w;
    const bool small = dtype == FFTCONV_F32 || ((O + 255) / 256) * ((C + 255) / 256) < 16;
    w.fo = small ? 2 : 4, w.fc = small ? 1 : 2;
    const int64_t tiles = ((O + 64 * w.fo - 1) / (64 * w.fo)) * ((C + 128 * w.fc - 1) / (128 * w.fc));
    const int64_t blocks = B > 0 ? B * ((N + RUN - 1) / RUN) : 1;        // (no sequence: one workgroup a tile writes the zeros)
    int64_t splits = 256 / tiles;
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
        constexpr int lds = 2 * (64 * FO * NP + 128 * FC) * 128;
        const auto kernel = k_weight<T, decltype(tok)::value, DW, FO, FC>;
        FC_TRY(raise_dynamic_lds((const void *)kernel, lds));
        const dim3 grid((unsigned)(((a.O + 64 * FO - 1) / (64 * FO)) * a.tiles_c), (unsigned)a.splits);
        kernel<<<grid, 512, lds, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    };
    using Y = std::true_type;
    using No = std::false_type;
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
    a.dy = dy, a.q = q, a.scale = scale, a.part = (float *)workspace, a.dw = dw, a.N = N, a.O = (int)O, a.C = (int)C;
    a.runs = (int)((N + RUN - 1) / RUN), a.blocks = (int)(B * a.runs), a.per = w.per, a.splits = w.splits;
    a.tiles_c = (int)((C + 128 * w.fc - 1) / (128 * w.fc));
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
