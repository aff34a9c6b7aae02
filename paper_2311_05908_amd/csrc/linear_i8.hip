// Product of rows in 8 bits with a weight in 8 bits, a scale for each token and for each output channel:
//
//   y[t, o] = (sum over k of x[t, k] w[o, k]) xs[t] ws[o] + bias[o]        the sum in 32-bit integers, exact, the rest in fp32, rounded at the store
//
// One kernel serves both layouts of y. Its two operands, both with k contiguous, are R, whose rows lie next to each other in y, and S:
// token by token (t, o) R is the weight, channel by channel (parts, b, o / parts, n) R is the tokens. An accumulator of the matrix cores holds
// four consecutive rows of R for one row of S in a lane, so the values that a lane stores are neighbours in y either way.
//
// Which kernel: up to 64 tokens k_linear_few, bound by the weight's bytes. Above, with k in pieces of 16 bytes (both operands aligned to them),
// k_linear_async: on tiles of 256 x 256 where there is one for every compute unit, else on 128 x 128 where there are 128 of those, and with k in ranges
// where there are 64 or less and k is about 1000 or more. Everything else is k_linear's, which takes any k at any alignment, on up to 128 x 256 (4097 x
// 4097 -> 4097: 0.72 POP/s, where 4096 x 4096 -> 4096 makes 2.1): among it calls of 65 to 127 tiles of 128 x 128, or of fewer with a shorter k, on 64 x 64.
// That last line has not been measured out: 4096 -> 4096 takes 20 us for 256 tokens (ranges), 39 for 257 to 384 (k_linear) and 19 for 385.
#include "layers_index.h"
#include "linear_common.h"

namespace fftconv {
namespace lay {

struct LinArgs {
    const int8_t *r, *s;          // (nr, K), (ns, K)
    const float *rscale, *sscale, *rbias, *sbias;
    void *y;
    int64_t K;
    int nr, ns;
    int channels;                 // y channel by channel: R is b * N + n, S is o
    int beyond_cache;             // y is larger than the memory-side cache (256 MB) by far
    int N, per_part;              // samples of a sequence; output channels of a part
    uint32_t by_n, by_part;       // 2^32 over these, rounded up
    int64_t B;
    int tiles_r, tiles_s;
    int first;                    // tile of a launch's first workgroup (k_linear)
    int ranges, per;              // of k, whose sums of a tile are added up by a second kernel (1: all of k); steps of one
    int *part;                    // (ranges, ns, nr)
};

// First value of y in row s of S: y[column(s) + offset(r)].
__device__ __forceinline__ int64_t column_of(const LinArgs &a, int s)
{
    if (!a.channels) return (int64_t)s * a.nr;
    return (s + quotient(s, a.per_part, a.by_part) * (a.B - 1) * a.per_part) * a.N;
}
// ... and the place of row r of R in it.
__device__ __forceinline__ int64_t row_of(const LinArgs &a, int r)
{
    if (!a.channels) return r;
    const int b = quotient(r, a.N, a.by_n);
    return r + (int64_t)b * (a.per_part - 1) * a.N;
}

template <int FR, int FS> struct Tile {
    static constexpr int BR = 64 * FR, BS = 64 * FS, BK = 64;      // 2 x 2 waves of FR x FS accumulators of 32 x 32
    static constexpr int STAGE = (BR + BS) * BK;
};

__device__ __forceinline__ i32x16 mfma_i8(uint4 a, uint4 b, i32x16 c)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// W values of y in row s of S, from row r of R on (r a multiple of W).
template <typename T, int W> __device__ __forceinline__ void put(const LinArgs &a, int64_t col, int r, const T (&v)[W])
{
    T *const y = (T *)a.y + col;
    if (r + W <= a.nr && (!a.channels || r - quotient(r, a.N, a.by_n) * a.N + W <= a.N)) {
        store_bytes<sizeof(v)>(y + row_of(a, r), v);
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (r + e < a.nr) y[row_of(a, r + e)] = v[e];
    }
}

// One accumulator of 32 x 32: lane l holds column l % 32, register i row 8 (i / 4) + 4 (l / 32) + i % 4.
template <typename T> __device__ __forceinline__ void epilogue(const LinArgs &a, const i32x16 &acc, int r0, int s, const float (&rs)[16],
                                                               const float (&rb)[16], float ss, float sb, int64_t col)
{
    const int half = (threadIdx.x >> 5) & 1;
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaf((float)acc[i] * rs[i], ss, rb[i] + sb);
    if constexpr (sizeof(T) == 4) {
        if (s >= a.ns) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float o[4] = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
            put<float, 4>(a, col, r0 + 8 * j + 4 * half, o);
        }
    } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const T p[2] = {from_f32<T>(v[2 * i]), from_f32<T>(v[2 * i + 1])};
            __builtin_memcpy(&w[i], p, 4);
        }
        // rows 8 j + 4 half ... + 3 of two j: the halves of the wave exchange, so that each lane has eight rows in a run
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto x = __builtin_amdgcn_permlane32_swap(w[2 * j + i], w[2 * j + 2 + i], false, false);
                o[i] = x[0], o[i + 2] = x[1];
            }
            T t[8];
            __builtin_memcpy(t, o, 16);
            if (s < a.ns) put<T, 8>(a, col, r0 + 8 * j + 8 * half, t);
        }
    }
}

// The same where a tile is inside y and its rows' runs of 16 bytes do not end within: by way of 4 KB of LDS of the wave's own, so that a store writes
// 128 bytes in a row of eight columns, whole lines, instead of 32 of thirty-two. 64 rows (32 of fp32) of 32 columns at a time, a row of 128 bytes
// to a column, its 16-byte pieces moved by the pair of columns; the halves of a piece change places in columns 16 up, so that the 32 lanes that
// write at once meet no bank twice.
template <typename T, bool CHANNELS> __device__ __forceinline__ void scaled_to_lds(char *own, const i32x16 &acc, int part, const float *rscale,
                                                                                   const float *rbias, float ss, float sb)
{
    const int half = (threadIdx.x >> 5) & 1, l32 = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float v[4];
        const f32x4 rs = *(const f32x4 *)(rscale + 8 * q + 4 * half);
        if constexpr (CHANNELS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf((float)acc[4 * q + i] * rs[i], ss, sb);
        } else {
            const f32x4 rb = *(const f32x4 *)(rbias + 8 * q + 4 * half);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf((float)acc[4 * q + i] * rs[i], ss, rb[i]);
        }
        if constexpr (sizeof(T) == 4) {
            *(float4 *)(own + l32 * 128 + (((2 * q + half) ^ ((l32 >> 1) & 7)) << 4)) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            const T t[4] = {from_f32<T>(v[0]), from_f32<T>(v[1]), from_f32<T>(v[2]), from_f32<T>(v[3])};
            uint2 w;
            __builtin_memcpy(&w, t, 8);
            *(uint2 *)(own + l32 * 128 + (((4 * part + q) ^ ((l32 >> 1) & 7)) << 4) + ((half ^ (l32 >> 4)) << 3)) = w;
        }
    }
}
// Piece (lane % 8) of column lane / 8 + 8 t of what lies there.
template <typename T> __device__ __forceinline__ uint4 column_piece(const char *own, int t)
{
    const int lane = threadIdx.x & 63, c = (lane >> 3) + 8 * t;
    const uint4 v = *(const uint4 *)(own + c * 128 + (((lane & 7) ^ ((c >> 1) & 7)) << 4));
    return sizeof(T) == 2 && t >= 2 ? make_uint4(v.z, v.w, v.x, v.y) : v;
}

template <typename T, int FR, int FS> __global__ void __launch_bounds__(256, 2) k_linear(const LinArgs a)
{
    using G = Tile<FR, FS>;
    constexpr int PIECES = (G::BR + G::BS) * 4 / 256;             // 16-byte pieces a thread stages
    __shared__ __align__(16) char lds[2 * G::STAGE];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wr = wave >> 1, wsv = wave & 1;
    const int tile = a.first + (int)blockIdx.x, tr = tile / a.tiles_s, ts = tile % a.tiles_s;
    const int r0 = tr * G::BR, s0 = ts * G::BS;
    const int8_t *src[PIECES];
    int dst[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = threadIdx.x + i * 256, row = p >> 2, c = p & 3;
        const bool is_r = row < G::BR;
        const int g = is_r ? min(r0 + row, a.nr - 1) : min(s0 + row - G::BR, a.ns - 1);      // rows beyond the end: the last one, not stored
        src[i] = (is_r ? a.r : a.s) + (int64_t)g * a.K;
        dst[i] = piece_at(row, c);
    }
    uint4 stage[PIECES];
    const int steps = (int)((a.K + G::BK - 1) / G::BK);
    auto fetch = [&](int step) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) stage[i] = load16(src[i], (int64_t)step * G::BK + (threadIdx.x & 3) * 16, a.K);
    };
    auto keep = [&](int buf) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) *(uint4 *)(lds + buf * G::STAGE + dst[i]) = stage[i];
    };
    i32x16 acc[FR][FS] = {};
    fetch(0);
    keep(0);
    lds_barrier();
    const int half = lane >> 5, l32 = lane & 31;
    for (int k = 0; k < steps; ++k) {
        if (k + 1 < steps) fetch(k + 1);
        const char *const base = lds + (k & 1) * G::STAGE;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            uint4 fr[FR], fs[FS];
#pragma unroll
            for (int i = 0; i < FR; ++i) fr[i] = *(const uint4 *)(base + piece_at((wr * FR + i) * 32 + l32, kk * 2 + half));
#pragma unroll
            for (int i = 0; i < FS; ++i) fs[i] = *(const uint4 *)(base + piece_at(G::BR + (wsv * FS + i) * 32 + l32, kk * 2 + half));
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FS; ++j) acc[i][j] = mfma_i8(fr[i], fs[j], acc[i][j]);
        }
        if (k + 1 < steps) {
            keep((k + 1) & 1);
            lds_barrier();
        }
    }
#pragma unroll
    for (int i = 0; i < FR; ++i) {
        const int rbase = r0 + (wr * FR + i) * 32;
        float rs[16], rb[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int r = min(rbase + 8 * (e / 4) + 4 * half + e % 4, a.nr - 1);
            rs[e] = a.rscale[r];
            rb[e] = a.rbias ? a.rbias[r] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < FS; ++j) {
            const int s = s0 + (wsv * FS + j) * 32 + l32, sc = min(s, a.ns - 1);
            epilogue<T>(a, acc[i][j], rbase, s, rs, rb, a.sscale[sc], a.sbias ? a.sbias[sc] : 0.f, column_of(a, sc));
        }
    }
}

// The same for operands in pieces of 16 bytes (K a multiple of 16): 2 x 4 waves, pieces straight to LDS three steps of 64 ahead of the products,
// operands in registers one group ahead. A workgroup takes one tile after the other without a pause in the stream of pieces: what is asked for
// during a tile's last steps is the next tile's, so its first loads are not waited for.
//
// Measured: f16 8192 x 4096 -> 16384 505 us, 2.2 POP/s; bf16 64 x 4096 x 768 -> 3 x 768 613 us, 1.5 POP/s, with 1.2 GB written. Back to back the socket
// is at its cap (1391 and 1398 of 1400 W); under the profiler, which pauses between launches, 492 and 560 us at 1.9 GHz, the matrix cores busy 55 and
// 41 % of it. The matrix cores alone, with nothing brought or stored, take 425 and 330 us; what is brought (70 and 60 us), scaled (100)
// and stored (150) comes on top rather than beside them, for results are written after a tile's products; without any wait for a transfer, or
// without barriers, the time is the same. Hence the large tile (128 x 128: 741 and 917 us), whole lines to a store, and places in y that cost
// no arithmetic.
template <typename T, bool CHANNELS, bool SPLIT, int FR, int FS> __global__ void __launch_bounds__(512, 2) k_linear_async(const LinArgs a, const Walk walk)
{
    constexpr int BR = 64 * FR, BS = 128 * FS, BK = 64, STAGE = (BR + BS) * BK, STAGES = 4, LI = (BR + BS) / 128;
    static_assert(BR == BS, "waves 0-3 bring R, 4-7 bring S");
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int wr = wave >> 2, wsv = wave & 3;
    // tiles first, first + stride, ... below last
    const int wgs = gridDim.x, die = blockIdx.x % 8, dies = min(8, wgs), on_die = (wgs - die + 7) / 8;
    const int begin = (int)((int64_t)walk.tiles * die / dies), last = (int)((int64_t)walk.tiles * (die + 1) / dies);
    const int first = begin + blockIdx.x / 8;
    const int all_steps = (int)((a.K + BK - 1) / BK);
    const bool tail = a.K % BK != 0;
    // item i of the walk: tile i / ranges, range i % ranges of k
    auto item = [&](int i, int &tr, int &ts, int &range) {
        range = SPLIT ? i % a.ranges : 0;
        walk.place(SPLIT ? i / a.ranges : i, tr, ts, a.tiles_r);
    };
    auto steps_of = [&](int range) { return SPLIT ? min(a.per, all_steps - range * a.per) : all_steps; };

    // This wave brings rows 16 LI w' ... of R (waves 0-3) or S (4-7), sixteen with an instruction, a piece of 16 bytes for each lane, moved as
    // piece_at has it.
    const bool is_r = wave < 4;
    const int8_t *const src = is_r ? a.r : a.s;
    const int rows = is_r ? a.nr : a.ns, block = is_r ? BR : BS;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_offset(lds)) + wave * LI * 1024;
    int f_tile = first, f_step = 0, f_steps = 0, f_first = 0;    // what is asked for next; steps of its range, and of those before it
    const char *base = nullptr;
    uint32_t off[LI];
    auto aim = [&] {                                             // at tile f_tile, or, after the last, once more at it
        int tr, ts, range;
        item(min(f_tile, last - 1), tr, ts, range);
        f_steps = steps_of(range), f_first = SPLIT ? range * a.per : 0;
        const int row0 = (is_r ? tr : ts) * block;
        base = (const char *)src + (int64_t)row0 * a.K + (int64_t)f_first * BK - 3072;
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            const int row = (wave & 3) * 16 * LI + i * 16 + (lane >> 2), piece = (lane & 3) ^ ((row >> 2) & 3);
            off[i] = (uint32_t)(min(row0 + row, rows - 1) - row0) * (uint32_t)a.K + piece * 16 + 3072 - i * 1024;
        }
    };
    auto fetch = [&](int stage) {
        if (tail && f_first + f_step == all_steps - 1) {                       // what lies beyond K reads as zeros
#pragma unroll
            for (int i = 0; i < LI; ++i) {
                const int piece = (lane & 3) ^ ((lane >> 4) & 3);
                const char *const from = base + off[i] + i * 1024;
                to_lds16((int64_t)(f_first + f_step) * BK + piece * 16 < a.K ? from : (const char *)&zero_piece, lds + stage * STAGE + (wave * LI + i) * 1024);
            }
        } else {
            to_lds16_rows<LI>(uniform(base), off, __builtin_amdgcn_readfirstlane(to + stage * STAGE));
        }
        base += BK;
        if (++f_step == f_steps) {
            f_step = 0, f_tile += on_die;
            aim();
        }
    };

    if (first >= last) return;
    aim();
    fetch(0);
    fetch(1);
    fetch(2);
    // where this lane's pieces are, from a stage's start: of k 0 ... 31, and of k 32 ... 63 at ^ 32
    const int ro = piece_at(wr * FR * 32 + l32, half), so = BR * 64 + piece_at(wsv * FS * 32 + l32, half);
    uint4 fr[2][FR], fs[2][FS];
    auto read = [&](const char *stage, int kk) {
#pragma unroll
        for (int i = 0; i < FR; ++i) fr[kk][i] = *(const uint4 *)(stage + (ro ^ (kk << 5)) + i * 2048);
#pragma unroll
        for (int j = 0; j < FS; ++j) fs[kk][j] = *(const uint4 *)(stage + (so ^ (kk << 5)) + j * 2048);
    };
    // Scales and biases of this wave's rows of a tile come to LDS at the tile's beginning, to a place of the wave's own, two tiles in turn.
    constexpr int NR = FR / 2, PRIVATE = (2 * NR + 2) * 256;
    const char *const own = lds + STAGES * STAGE + wave * 2 * PRIVATE;
    int tr, ts, range, parity = 0;
    auto fetch_scales = [&] {
        const char *const at = own + parity * PRIVATE;
        // (from the tile's first row on: a tensor may have more rows than 32 bits count bytes)
        const int r0 = tr * BR, s0 = ts * BS, r = r0 + wr * FR * 32 + lane;
        const uint32_t so = (uint32_t)(min(s0 + wsv * FS * 32 + (FS == 2 ? lane : l32), a.ns - 1) - s0) * 4u;
        const char *const zero = (const char *)&zero_piece;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const uint32_t o = (uint32_t)(min(r + i * 64, a.nr - 1) - r0) * 4u;
            to_lds4(uniform((const char *)(a.rscale + r0)), o, at + i * 256);
            if (!CHANNELS) to_lds4(uniform(a.rbias ? (const char *)(a.rbias + r0) : zero), a.rbias ? o : 0, at + (NR + i) * 256);
        }
        to_lds4(uniform((const char *)(a.sscale + s0)), so, at + 2 * NR * 256);
        if (CHANNELS) to_lds4(uniform(a.sbias ? (const char *)(a.sbias + s0) : zero), a.sbias ? so : 0, at + (2 * NR + 1) * 256);
    };
    FC_ARRIVED(2 * LI);
    read(lds, 0);
    int stage = 0;
    for (int tile = first; tile < last; tile += on_die) {
        item(tile, tr, ts, range);
        const int steps = steps_of(range);
        if (!SPLIT) fetch_scales();
        i32x16 acc[FR][FS] = {};
        auto products = [&](int kk) {
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FS; ++j) acc[i][j] = mfma_i8(fr[kk][i], fs[kk][j], acc[i][j]);
        };
        for (int k = 0; k < steps; ++k) {
            const char *const here = lds + stage * STAGE;
            fetch(stage == 0 ? STAGES - 1 : stage - 1);          // (every wave had read that stage before the last barrier)
            read(here, 1);
            __builtin_amdgcn_sched_barrier(0);
            products(0);
            __builtin_amdgcn_sched_barrier(0);
            FC_ARRIVED(2 * LI);                                  // the next step's pieces are there, those of the two after it on their way
            stage = stage + 1 < STAGES ? stage + 1 : 0;
            read(lds + stage * STAGE, 0);
            __builtin_amdgcn_sched_barrier(0);
            products(1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (SPLIT) {
            int *const part = a.part + (int64_t)range * a.ns * a.nr;
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FS; ++j) {
                    const int s = ts * BS + (wsv * FS + j) * 32 + l32, r = tr * BR + (wr * FR + i) * 32 + 4 * half;
                    if (s >= a.ns) continue;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                        store_piece<int, 4>(part + (int64_t)s * a.nr + r + 8 * q, a.nr - r - 8 * q, v);
                    }
                }
            continue;
        }
        // (three steps after they were asked for the scales are there; with fewer steps they are waited for)
        if (steps < 3) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const char *const sc = own + parity * PRIVATE;
        parity ^= 1;
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                         // (else the compiler keeps the places below in registers throughout the sums)
        const int l32 = lane & 31, half = lane >> 5, r0 = tr * BR, s0 = ts * BS;
        constexpr int W = 16 / sizeof(T);
        // All of it inside y, in one sequence and one part of y: places are linear in rows and columns.
        bool whole = r0 + BR <= a.nr && s0 + BS <= a.ns && (CHANNELS ? a.N : a.nr) < 1 << 26;        // (32-bit distances of seven columns)
        if (CHANNELS)
            whole = whole && quotient(r0, a.N, a.by_n) == quotient(r0 + BR - 1, a.N, a.by_n) &&
                    quotient(s0, a.per_part, a.by_part) == quotient(s0 + BS - 1, a.per_part, a.by_part);
        auto column_scale = [&](int j) { return *(const float *)(sc + (2 * NR * 64 + j * 32 + l32) * 4); };
        auto column_bias = [&](int j) { return *(const float *)(sc + ((2 * NR + 1) * 64 + j * 32 + l32) * 4); };
        bool done = false;
        if constexpr (FR == 4) {                                 // (a stage has room for the waves; a smaller tile's has not)
            static_assert(STAGE == 8 * 4096 && LI * 1024 == 4096, "a wave's transfers and its results take the same place");
            if (whole) {
                done = true;
                // The stage of the last step: every wave has read it, and what comes there next is, in a wave's own 4 KB, that wave's own transfers,
                // which it asks for after this.
                char *const mine = lds + (stage == 0 ? STAGES - 1 : stage - 1) * STAGE + wave * 4096;
                constexpr int P = sizeof(T) == 2 ? 2 : 1;        // accumulators to a row of 128 bytes
                const uint32_t stride = CHANNELS ? (uint32_t)a.N : (uint32_t)a.nr;
                const int r1 = r0 + wr * FR * 32, s1 = s0 + wsv * FS * 32;
                const char *const y = uniform((const char *)((T *)a.y + column_of(a, s1) + row_of(a, r1)));
                const uint32_t at = ((uint32_t)(lane >> 3) * stride + (lane & 7) * W) * (uint32_t)sizeof(T);
                auto all = [&](auto beyond) {
#pragma unroll
                for (int i = 0; i < FR; i += P)
#pragma unroll
                    for (int j = 0; j < FS; ++j) {
                        __builtin_amdgcn_sched_barrier(0);
                        const float ss = column_scale(j), sb = CHANNELS ? column_bias(j) : 0.f;
#pragma unroll
                        for (int p = 0; p < P; ++p)
                            scaled_to_lds<T, CHANNELS>(mine, acc[i + p][j], p, (const float *)sc + (i + p) * 32, (const float *)sc + NR * 64 + (i + p) * 32, ss, sb);
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint4 v = column_piece<T>(mine, t);
                            char *const to = (char *)y + ((int64_t)(j * 32 + 8 * t) * stride + i * 32) * (int)sizeof(T) + at;
                            put16<decltype(beyond)::value>(to, v);
                        }
                    }
                };
                if (a.beyond_cache) all(std::true_type());
                else all(std::false_type());
            }
        }
        if (!done) {
#pragma unroll
            for (int i = 0; i < FR; ++i) {
                float rsv[16], rbv[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = i * 32 + 8 * (e / 4) + 4 * half + e % 4;
                    rsv[e] = ((const float *)sc)[r], rbv[e] = CHANNELS ? 0.f : ((const float *)sc)[NR * 64 + r];
                }
#pragma unroll
                for (int j = 0; j < FS; ++j) {
                    __builtin_amdgcn_sched_barrier(0);
                    const int s = s0 + (wsv * FS + j) * 32 + l32;
                    epilogue<T>(a, acc[i][j], r0 + (wr * FR + i) * 32, s, rsv, rbv, column_scale(j), CHANNELS ? column_bias(j) : 0.f, column_of(a, min(s, a.ns - 1)));
                }
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // nothing is on its way to LDS when the workgroup ends
}

// y from the ranges' sums: whole numbers, so their order does not matter.
template <typename T> __global__ void __launch_bounds__(256) k_linear_sums(const LinArgs a)
{
    const int per_row = (a.nr + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int s = (int)(i / per_row), r = (int)(i - (int64_t)s * per_row) * 4;
    if (s >= a.ns) return;
    const int64_t at = (int64_t)s * a.nr + r, size = (int64_t)a.ns * a.nr;
    int sum[4] = {};
#pragma unroll 4
    for (int k = 0; k < a.ranges; ++k) {
        int v[4] = {};
        if (r + 4 <= a.nr) {
            __builtin_memcpy(v, a.part + k * size + at, 16);
        } else {
            for (int e = 0; e < 4; ++e)
                if (r + e < a.nr) v[e] = a.part[k * size + at + e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
    const float ss = a.sscale[s], sb = a.sbias ? a.sbias[s] : 0.f;
    T y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int q = min(r + e, a.nr - 1);
        y[e] = from_f32<T>(fmaf((float)sum[e] * a.rscale[q], ss, (a.rbias ? a.rbias[q] : 0.f) + sb));
    }
    put<T, 4>(a, column_of(a, s), r, y);
}

// Into how many ranges k goes: where few tiles are left for the compute units, as many as give each one, of eight steps of 64 at least.
// (100 tokens, 4096 -> 4096: 32 us on tiles of 64 x 64 with all of k.)
static int k_ranges(int64_t T, int64_t K, int64_t O)
{
    const int64_t tiles = ((T + 127) / 128) * ((O + 127) / 128), steps = (K + 63) / 64;
    if (T <= 64 || K % 16 != 0 || tiles > 64) return 1;
    const int64_t most = 256 / tiles < steps / 8 ? 256 / tiles : steps / 8;
    if (most < 2) return 1;
    const int64_t per = (steps + most - 1) / most;
    return (int)((steps + per - 1) / per);
}

// Few tokens (S, up to 16 NT of them): what counts is how fast the weight streams in, so its rows go from memory straight into the
// operand registers, sixteen rows to a workgroup, whose waves divide k among themselves and add their sums up in LDS. Measured: 1 x 4096 -> 4096
// 5.0 us, 3.3 TB/s of the weight's 16.8 MB; 1 x 8192 -> 16384 25 us with the call, 5.4 TB/s.
struct FewArgs {
    const int8_t *x, *w;
    const float *xs, *ws, *bias;
    void *y;
    int64_t K, B;
    int T, O, channels, N, per_part;
    int first;                    // output of a launch's first workgroup
};

template <typename T, int NT> __global__ void __launch_bounds__(512) k_linear_few(const FewArgs a)
{
    __shared__ i32x4 sums[8][NT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int o0 = a.first + (int)blockIdx.x * 16;
    const int8_t *const w = a.w + (int64_t)min(o0 + l16, a.O - 1) * a.K;
    const int8_t *x[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) x[j] = a.x + (int64_t)min(j * 16 + l16, a.T - 1) * a.K;
    i32x4 acc[NT] = {};
    constexpr int U = NT == 1 ? 4 : 2;
    for (int64_t k0 = (int64_t)wave * 64; k0 < a.K; k0 += 512 * U) {
        uint4 fw[U], fx[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = k0 + 512 * u + quarter * 16;
            fw[u] = load16(w, k, a.K);
#pragma unroll
            for (int j = 0; j < NT; ++j) fx[u][j] = load16(x[j], k, a.K);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < NT; ++j)
                acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, fw[u]), __builtin_bit_cast(i32x4, fx[u][j]), acc[j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) sums[wave][j][lane] = acc[j];
    lds_barrier();
    // lane l holds token l % 16 of the sixteen, outputs 4 (l / 16) ... + 3
    for (int i = threadIdx.x; i < NT * 256; i += 512) {
        const int e = i & 3, l = (i >> 2) & 63, j = i >> 8;
        int sum = 0;
#pragma unroll
        for (int v = 0; v < 8; ++v) sum += sums[v][j][l][e];
        const int t = j * 16 + (l & 15), o = o0 + 4 * (l >> 4) + e;
        if (t >= a.T || o >= a.O) continue;
        const float v = fmaf((float)sum * a.ws[o], a.xs[t], a.bias ? a.bias[o] : 0.f);
        int64_t at = (int64_t)t * a.O + o;
        if (a.channels) {
            const int part = o / a.per_part, b = t / a.N;
            at = ((((int64_t)part * a.B + b) * a.per_part) + (o - part * a.per_part)) * a.N + (t - b * a.N);
        }
        ((T *)a.y)[at] = from_f32<T>(v);
    }
}

template <typename T> static int run(const int8_t *xq, const float *xs, const int8_t *wq, const float *ws, const float *bias, void *y, int64_t B,
                                     int64_t N, int64_t K, int64_t O, int64_t parts, void *workspace, hipStream_t s)
{
    const int64_t t = B * N;
    if (t <= 64) {
        FewArgs a = {xq, wq, xs, ws, bias, y, K, B, (int)t, (int)O, parts > 0, (int)N, (int)(parts ? O / parts : O), 0};
        return in_pieces((O + 15) / 16, 512, [&](int64_t first, unsigned g) -> int {
            a.first = (int)(first * 16);
            if (t <= 16) k_linear_few<T, 1><<<g, 512, 0, s>>>(a);
            else if (t <= 32) k_linear_few<T, 2><<<g, 512, 0, s>>>(a);
            else k_linear_few<T, 4><<<g, 512, 0, s>>>(a);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    }
    LinArgs a = {};
    a.channels = parts > 0;
    a.r = a.channels ? xq : wq, a.s = a.channels ? wq : xq;
    a.rscale = a.channels ? xs : ws, a.sscale = a.channels ? ws : xs;
    (a.channels ? a.sbias : a.rbias) = bias;
    a.y = y, a.K = K, a.nr = (int)(a.channels ? t : O), a.ns = (int)(a.channels ? O : t);
    a.N = (int)N, a.per_part = (int)(parts ? O / parts : O), a.B = B;
    a.beyond_cache = t * O * (int64_t)sizeof(T) > (int64_t)512 << 20;
    a.by_n = reciprocal(a.N), a.by_part = reciprocal(a.per_part);
    auto launch = [&](auto fr, auto fs) -> int {
        constexpr int FR = decltype(fr)::value, FS = decltype(fs)::value;
        using G = Tile<FR, FS>;
        a.tiles_r = (a.nr + G::BR - 1) / G::BR, a.tiles_s = (a.ns + G::BS - 1) / G::BS;
        return in_pieces((int64_t)a.tiles_r * a.tiles_s, 256, [&](int64_t first, unsigned g) -> int {
            a.first = (int)first;
            k_linear<T, FR, FS><<<g, 256, 0, s>>>(a);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    };
    auto launch_async = [&](auto fr, auto fs) -> int {
        constexpr int FR = decltype(fr)::value, FS = decltype(fs)::value, BR = 64 * FR, BS = 128 * FS, lds = 4 * (BR + BS) * 64 + 16 * (FR + 2) * 256;
        a.tiles_r = (a.nr + BR - 1) / BR, a.tiles_s = (a.ns + BS - 1) / BS;
        Walk w = {a.tiles_s, a.tiles_s <= 12 ? a.tiles_s : 8, a.tiles_r * a.tiles_s};
        const auto kernel = a.channels ? k_linear_async<T, true, false, FR, FS> : k_linear_async<T, false, false, FR, FS>;
        FC_TRY(raise_dynamic_lds((const void *)kernel, lds));
        const int most = 256 * (FR == 4 ? 1 : 2);
        kernel<<<(unsigned)(w.tiles < most ? w.tiles : most), 512, lds, s>>>(a, w);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    };
    auto tiles = [&](int br, int bs) { return (int64_t)((a.nr + br - 1) / br) * ((a.ns + bs - 1) / bs); };
    const bool pieces = K % 16 == 0 && ((uintptr_t)xq | (uintptr_t)wq) % 16 == 0;
    a.ranges = k_ranges(t, K, O);
    if (pieces && a.ranges > 1) {
        constexpr int lds = 4 * 256 * 64 + 16 * 4 * 256;
        const int64_t steps = (K + 63) / 64;
        a.per = (int)((steps + a.ranges - 1) / a.ranges), a.part = (int *)workspace;
        a.tiles_r = (a.nr + 127) / 128, a.tiles_s = (a.ns + 127) / 128;
        const Walk w = {a.tiles_s, a.tiles_s <= 12 ? a.tiles_s : 8, a.tiles_r * a.tiles_s * a.ranges};
        const auto kernel = k_linear_async<T, false, true, 2, 1>;
        FC_TRY(raise_dynamic_lds((const void *)kernel, lds));
        kernel<<<(unsigned)w.tiles, 512, lds, s>>>(a, w);
        FC_HIP(hipGetLastError());
        k_linear_sums<T><<<(unsigned)(((int64_t)((a.nr + 3) / 4) * a.ns + 255) / 256), 256, 0, s>>>(a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    }
    // The large tile from one for every compute unit on (8192 x 4096 -> 16384: 575 us, and 741 on the small one); below, the small one: with 144 large
    // ones (4096 x 768 -> 2304) 19.0 us and 20.0, with 128 (2048 x 4096 -> 4096) 46 us and 51.
    if (pieces && tiles(256, 256) >= 256) return launch_async(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
    if (pieces && tiles(128, 128) >= 128) return launch_async(std::integral_constant<int, 2>(), std::integral_constant<int, 1>());
    if (tiles(128, 256) >= 512) return launch(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
    if (tiles(128, 128) >= 256) return launch(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
    return launch(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
}

size_t linear_i8_workspace(int64_t T, int64_t K, int64_t O)
{
    const int ranges = k_ranges(T, K, O);
    return ranges > 1 ? (size_t)ranges * (size_t)T * (size_t)O * 4 : 0;
}

int linear_i8(const int8_t *xq, const float *xs, const int8_t *wq, const float *ws, const float *bias, void *y, int64_t B, int64_t N, int64_t K,
              int64_t O, int64_t parts, int dtype, void *workspace, hipStream_t s)
{
    if (dtype == FFTCONV_BF16) return run<__bf16>(xq, xs, wq, ws, bias, y, B, N, K, O, parts, workspace, s);
    if (dtype == FFTCONV_F16) return run<_Float16>(xq, xs, wq, ws, bias, y, B, N, K, O, parts, workspace, s);
    return run<float>(xq, xs, wq, ws, bias, y, B, N, K, O, parts, workspace, s);
}

}  // namespace lay
}  // namespace fftconv
