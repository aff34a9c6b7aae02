// A gated linear recurrence along the samples of every (sequence, channel), with its gradients, and one token of it.
//
//   a = sigmoid(w), x = (1 - a) u        or, gates by their logarithms, a = exp(min(w, 0)), x = u
//   h_t = a_t h_(t-1) + x_t from `state`;  y_t = v_t h_t
//   backward: p_t = a_t dh_t is what reaches the sample before, dh_t = v_t dy_t + p_(t+1) from `dlast`
//   du = (1 - a) dh, dw = dh (h_(t-1) - u) a (1 - a)    or    du = dh, dw = dh h_(t-1) a;    dv_t = dy_t h_t;  dstate = p_0
//
// A step is a map h -> a h + x; two in a row are one, (a' a, a' x + x'), so lanes compose their own samples, then one another's (sixteen lanes by
// exchanges inside the vector unit, the four rows of a wave one after the other with what comes in), and each walks its samples once more from
// what the lanes before it leave. A wave takes 512 samples of a row at a time, eight in a run for each lane; short rows get part of a wave.
// Everything between the load of u, w, v (and dy) and the store of y (du, dw, dv) is fp32 in registers: every tensor moves once, and that is what
// bounds these kernels: bf16 64 x 768 x 4096 forward 295 us, 5.5 TB/s, backward 510 us, 5.5 TB/s. What comes next is asked for before the samples in
// hand are worked on: 1024 rows of 65536 164 and 202 us, without 261 and 364.
//
// Few rows: a row goes in segments to waves of their own. A first kernel composes each segment to one map, and every wave of the second applies
// those before its own to the row's state (gradients: those behind it to `dlast`).
#include "layers_index.h"
#include "layers_internal.h"

namespace fftconv {
namespace lay {

struct ScanArgs {
    const void *u, *w, *v, *dy;
    const float *state, *dlast, *kept_in;
    const int32_t *lengths;
    void *y, *du, *dw, *dv;
    float *last, *dstate, *kept;
    float2 *maps;                 // (rows, segments): a segment as one map
    int64_t rows, N, first;       // first: row of a launch's first workgroup
    int C, chunks, segments, per; // pieces of 512 samples to a row; segments of a row, pieces of one
    int log_gate, beyond_cache;   // beyond_cache: a result is larger than the memory-side cache (256 MB)
};

constexpr int SE = 8;             // samples of a lane
constexpr float LOG2E = 0x1.715476p+0f, LOG2E_REST = 0x1.4ae0bep-26f, LN2 = 0x1.62e43p-1f;      // log2 e in two parts

// 2^(x log2 e) for x <= 0. What the product rounds away (|x| 2^-24 of the result) is put back where results are fp32.
template <bool CLOSE> __device__ __forceinline__ float exp_below_one(float x)
{
    const float p = x * LOG2E, t = __builtin_amdgcn_exp2f(p);
    if constexpr (!CLOSE) return t;
    const float rest = fmaf(x, LOG2E_REST, fmaf(x, LOG2E, -p)) * LN2;
    return x < -200.f ? 0.f : fmaf(t, rest, t);                  // (from there on the product may be an infinity, and its rest no number)
}

// Gate and its complement: both are exact to rounding however near to one the other is; infinite logits are gates of 0 and 1.
template <typename T> __device__ __forceinline__ void gate_of(float w, bool log_gate, float &a, float &rest)
{
    constexpr bool CLOSE = sizeof(T) == 4;
    if (log_gate) {
        a = exp_below_one<CLOSE>(w > 0.f ? 0.f : w);
        rest = 1.f;
        return;
    }
    // (a state of a long memory meets thousands of gates: the reciprocal is taken to half a unit in the last place, by a step on from the instruction's)
    const float t = exp_below_one<CLOSE>(-fabsf(w)), d = 1.f + t, r0 = __builtin_amdgcn_rcpf(d), r = fmaf(fmaf(-d, r0, 1.f), r0, r0), tr = t * r;
    a = w >= 0.f ? r : tr;
    rest = w >= 0.f ? tr : r;
}

// Eight results of a lane. Past the caches where a tensor is larger than the memory-side one and pushes everything else out of it: bf16 64 x 768 x 4096 305 -> 295 us,
// with the gradients 840 -> 806. (fp32, whose eight are two stores of half a line, goes through them.)
template <typename T> __device__ __forceinline__ void put(T *p, int64_t left, const T (&v)[SE], int beyond_cache)
{
    if (sizeof(T) == 2 && beyond_cache && left >= SE) {
        typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4;
        u32x4 w;
        __builtin_memcpy(&w, v, sizeof(w));
        __builtin_nontemporal_store(w, (u32x4 *)p);
    } else {
        store_piece<T, SE>(p, left, v);
    }
}

template <int CTRL, bool ZERO> __device__ __forceinline__ float dpp_f32(float outside, float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, outside), __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, ZERO));
}
__device__ __forceinline__ float lane_of(float x, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

struct Map {
    float a, x;
};

// One step of the scan over a row of 16 lanes: the map of the lane D before (REVERSE: behind) goes first; lanes in groups of G.
template <bool REVERSE, int D, int G> __device__ __forceinline__ void compose_with(Map &m)
{
    constexpr int CTRL = (REVERSE ? 0x100 : 0x110) + D;
    float a = dpp_f32<CTRL, false>(1.f, m.a), x = dpp_f32<CTRL, false>(0.f, m.x);
    if constexpr (G < 16) {
        const int at = threadIdx.x & (G - 1);
        const bool there = REVERSE ? at + D < G : at >= D;
        a = there ? a : 1.f;
        x = there ? x : 0.f;
    }
    m.x = fmaf(m.a, x, m.x);
    m.a *= a;
}

// From each lane's own map and what comes into its group of G lanes (`in`, the same in all of them): what comes into the lane, and in `in` what leaves the
// group. Samples run up the lanes, or with REVERSE down.
template <bool REVERSE, int G> __device__ __forceinline__ float into_lane(Map m, float &in)
{
    if constexpr (G == 1) {
        const float was = in;
        in = fmaf(m.a, in, m.x);
        return was;
    } else {
        compose_with<REVERSE, 1, G>(m);
        compose_with<REVERSE, 2, G>(m);
        if constexpr (G >= 16) {
            compose_with<REVERSE, 4, G>(m);
            compose_with<REVERSE, 8, G>(m);
        }
        // the lanes before this one, of its row of 16 (or group of 4)
        constexpr int CTRL = REVERSE ? 0x101 : 0x111;
        float a = dpp_f32<CTRL, false>(1.f, m.a), x = dpp_f32<CTRL, false>(0.f, m.x);
        if constexpr (G < 16) {
            const int at = threadIdx.x & (G - 1);
            const bool there = REVERSE ? at + 1 < G : at >= 1;
            a = there ? a : 1.f;
            x = there ? x : 0.f;
        }
        float row_in = in;
        if constexpr (G == 64) {
            // rows one after the other: what comes into each
            constexpr int A = REVERSE ? 48 : 15, B = REVERSE ? 32 : 31, C = REVERSE ? 16 : 47, D = REVERSE ? 0 : 63;
            const float in1 = fmaf(lane_of(m.a, A), in, lane_of(m.x, A)), in2 = fmaf(lane_of(m.a, B), in1, lane_of(m.x, B));
            const float in3 = fmaf(lane_of(m.a, C), in2, lane_of(m.x, C));
            const int row = REVERSE ? 3 - ((threadIdx.x >> 4) & 3) : (threadIdx.x >> 4) & 3;
            row_in = row == 0 ? in : row == 1 ? in1 : row == 2 ? in2 : in3;
            in = fmaf(lane_of(m.a, D), in3, lane_of(m.x, D));
        } else {
            // (the group's whole map is in its last lane, or its first)
            const int whole = (threadIdx.x & 63 & ~(G - 1)) + (REVERSE ? 0 : G - 1);
            in = fmaf(__shfl(m.a, whole), in, __shfl(m.x, whole));
        }
        return fmaf(a, row_in, x);
    }
}

// Eight samples of a lane as they lie in memory, zeros where a row has ended: what is asked for while the 512 samples before are worked on.
template <typename T> struct Raw {
    T v[SE];
    template <bool WHOLE> __device__ __forceinline__ void load(const void *p, int64_t row, int64_t col, int64_t N)
    {
        const T *const x = (const T *)p + row * N;
        if constexpr (WHOLE) {                                   // (a piece that is not there is read at the row's beginning: no branch parts the loads)
            load_bytes<SE * (int)sizeof(T)>(x + (col < N ? col : 0), v);
        } else if (col + SE <= N) {
            load_bytes<SE * (int)sizeof(T)>(x + col, v);
        } else {
#pragma unroll
            for (int e = 0; e < SE; ++e) v[e] = col + e < N ? x[col + e] : (T)0.f;
        }
    }
};

// What a wave's lanes have of G lanes' samples from `col` on: gates and inputs of samples below `len`; behind it the state stays what it is.
template <typename T> struct Piece {
    float a[SE], rest[SE], u[SE], x[SE];
    __device__ __forceinline__ void take(const ScanArgs &g, const Raw<T> &ru, const Raw<T> &rw, int64_t col, int64_t len, bool all)
    {
#pragma unroll
        for (int e = 0; e < SE; ++e) u[e] = to_f32(ru.v[e]);
        if (g.log_gate) {
#pragma unroll
            for (int e = 0; e < SE; ++e) gate_of<T>(to_f32(rw.v[e]), true, a[e], rest[e]), x[e] = u[e];
        } else {
#pragma unroll
            for (int e = 0; e < SE; ++e) gate_of<T>(to_f32(rw.v[e]), false, a[e], rest[e]), x[e] = rest[e] * u[e];
        }
        if (!all) {
#pragma unroll
            for (int e = 0; e < SE; ++e) {
                const bool there = col + e < len;
                a[e] = there ? a[e] : 1.f;
                x[e] = there ? x[e] : 0.f;
                u[e] = there ? u[e] : 0.f;
            }
        }
    }
    __device__ __forceinline__ Map map() const
    {
        Map m = {a[0], x[0]};
#pragma unroll
        for (int e = 1; e < SE; ++e) m.x = fmaf(a[e], m.x, x[e]), m.a *= a[e];
        return m;
    }
};

__device__ __forceinline__ int64_t length_of(const ScanArgs &g, int64_t row)
{
    if (!g.lengths) return g.N;
    const int64_t n = g.lengths[row / g.C];
    return n < 0 ? 0 : n < g.N ? n : g.N;
}

// Maps of `count` of a row's segments, applied to `in` one after the other (REVERSE: from the last): 256 at a time, four in a run for each lane. The first
// 256 are asked for when this is made, so that what else a wave reads is on its way behind them.
template <bool REVERSE> struct Segments {
    const float2 *maps;
    int count;
    float2 m[4];
    __device__ __forceinline__ void load(int base)
    {
        const int k0 = (REVERSE ? count - base - 256 : base) + (int)(threadIdx.x & 63) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = k0 + e >= 0 && k0 + e < count ? maps[k0 + e] : make_float2(1.f, 0.f);
    }
    __device__ __forceinline__ Segments(const float2 *maps, int count) : maps(maps), count(count) { load(0); }
    __device__ __forceinline__ float through(float in)
    {
        for (int base = 0; base < count; base += 256) {
            if (base > 0) load(base);
            Map one = {1.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = REVERSE ? 3 - i : i;
                one.x = fmaf(m[e].x, one.x, m[e].y);
                one.a *= m[e].x;
            }
            into_lane<REVERSE, 64>(one, in);
        }
        return in;
    }
};

// A workgroup's rows: 256 / G of them, or with G = 64 segments of rows, four of them.
template <typename T, int G, bool WHOLE> __global__ void __launch_bounds__(256) k_scan(const ScanArgs g)
{
    const int lane = threadIdx.x & (G - 1);
    int64_t row = g.first + (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    int seg = 0;
    if constexpr (G == 64) {
        if (g.segments > 1) {
            const int64_t i = row;
            row = i / g.segments, seg = (int)(i - row * g.segments);
        }
    }
    if constexpr (G == 64) {
        if (row >= g.rows) return;
    }
    const bool there = row < g.rows;                             // (lanes exchange what they hold: none leaves a wave early)
    row = there ? row : g.rows - 1;
    const int64_t len = length_of(g, row);
    const int end = min((seg + 1) * g.per, g.chunks);
    Raw<T> u, w, v;
    auto ask = [&](int k) {
        const int64_t begin = (int64_t)k * (G * SE), col = begin + lane * SE;
        if (k >= end || begin >= len) return;
        u.template load<WHOLE>(g.u, row, col, g.N);
        w.template load<WHOLE>(g.w, row, col, g.N);
        if (g.v) v.template load<WHOLE>(g.v, row, col, g.N);
    };
    float h = g.state ? g.state[row] : 0.f;
    Segments<false> before(g.maps + row * g.segments, G == 64 ? seg : 0);
    ask(seg * g.per);
    h = before.through(h);
    for (int k = seg * g.per; k < end; ++k) {
        const int64_t begin = (int64_t)k * (G * SE), col = begin + lane * SE;
        if (g.kept && lane == 0 && there) g.kept[row * g.chunks + k] = h;
        T y[SE] = {};
        if (begin < len) {
            Piece<T> p;
            p.take(g, u, w, col, len, begin + G * SE <= len);
            const Raw<T> gate = v;
            ask(k + 1);
            float s = into_lane<false, G>(p.map(), h);
#pragma unroll
            for (int e = 0; e < SE; ++e) {
                s = fmaf(p.a[e], s, p.x[e]);
                const float o = g.v ? s * to_f32(gate.v[e]) : s;
                y[e] = from_f32<T>(col + e < len ? o : 0.f);
            }
        }
        if (there) {
            if (!WHOLE || col < g.N) put<T>((T *)g.y + row * g.N + col, WHOLE ? SE : g.N - col, y, g.beyond_cache);
        }
    }
    if (g.last && lane == 0 && there && seg == g.segments - 1) g.last[row] = h;
}

// A segment as one map: of the state, or with BACK of what reaches the sample before. The last segment's (the first's) is nobody's input.
template <typename T, bool BACK, bool WHOLE> __global__ void __launch_bounds__(256) k_scan_maps(const ScanArgs g)
{
    const int lane = threadIdx.x & 63;
    const int64_t i = g.first + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = i / (g.segments - 1);
    const int seg = (int)(i - row * (g.segments - 1)) + (BACK ? 1 : 0);
    if (row >= g.rows) return;
    const int64_t len = length_of(g, row);
    const int begin = seg * g.per, count = min((seg + 1) * g.per, g.chunks) - begin;
    Map m = {1.f, 0.f};
    for (int j = 0; j < count; ++j) {
        const int k = BACK ? begin + count - 1 - j : begin + j;
        const int64_t at = (int64_t)k * (64 * SE), col = at + lane * SE;
        if (at >= len) continue;
        const bool all = at + 64 * SE <= len;
        Map own;
        if constexpr (!BACK) {
            Raw<T> u, w;
            u.template load<WHOLE>(g.u, row, col, g.N);
            w.template load<WHOLE>(g.w, row, col, g.N);
            Piece<T> p;
            p.take(g, u, w, col, len, all);
            own = p.map();
        } else {
            float w[SE], dy[SE], v[SE];
            load_row_piece<T, SE, WHOLE>((const T *)g.w + row * g.N, col, g.N, w);
            load_row_piece<T, SE, WHOLE>((const T *)g.dy + row * g.N, col, g.N, dy);
            if (g.v) {
                load_row_piece<T, SE, WHOLE>((const T *)g.v + row * g.N, col, g.N, v);
#pragma unroll
                for (int e = 0; e < SE; ++e) dy[e] *= v[e];
            }
            own = {1.f, 0.f};
#pragma unroll
            for (int e = SE - 1; e >= 0; --e) {
                float a, rest;
                gate_of<T>(w[e], g.log_gate, a, rest);
                const bool there = all || col + e < len;
                own.x = there ? a * (dy[e] + own.x) : own.x;
                own.a = there ? own.a * a : own.a;
            }
        }
        // the wave's own map as what it makes of 0, and of the gates alone
        float x = m.x, a = m.a;
        into_lane<BACK, 64>(own, x);
        into_lane<BACK, 64>({own.a, 0.f}, a);
        m = {a, x};
    }
    if (lane == 0) g.maps[row * g.segments + seg] = make_float2(m.a, m.x);
}

template <typename T, int G, bool WHOLE, bool AHEAD> __global__ void __launch_bounds__(256) k_scan_back(const ScanArgs g)
{
    const int lane = threadIdx.x & (G - 1);
    int64_t row = g.first + (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    int seg = 0;
    if constexpr (G == 64) {
        if (g.segments > 1) {
            const int64_t i = row;
            row = i / g.segments, seg = (int)(i - row * g.segments);
        }
        if (row >= g.rows) return;
    }
    const bool there = row < g.rows;
    row = there ? row : g.rows - 1;
    const int64_t len = length_of(g, row);
    const int first = seg * g.per;
    Raw<T> ru, rw, rv, rdy;
    float kept = 0.f;
    auto ask = [&](int k) {
        const int64_t begin = (int64_t)k * (G * SE), col = begin + lane * SE;
        if (k < first || begin >= len) return;
        ru.template load<WHOLE>(g.u, row, col, g.N);
        rw.template load<WHOLE>(g.w, row, col, g.N);
        rdy.template load<WHOLE>(g.dy, row, col, g.N);
        if (g.v) rv.template load<WHOLE>(g.v, row, col, g.N);
        kept = g.kept_in[row * g.chunks + k];
    };
    const int top = min((seg + 1) * g.per, g.chunks) - 1;
    float p = g.dlast ? g.dlast[row] : 0.f;
    Segments<true> behind(g.maps + row * g.segments + seg + 1, G == 64 ? g.segments - 1 - seg : 0);
    ask(top);
    p = behind.through(p);
    for (int k = top; k >= first; --k) {
        const int64_t begin = (int64_t)k * (G * SE), col = begin + lane * SE;
        T du[SE] = {}, dw[SE] = {}, dv[SE] = {};
        if (begin < len) {
            const bool all = begin + G * SE <= len;
            Piece<T> q;
            q.take(g, ru, rw, col, len, all);
            const Raw<T> w = rw, dy = rdy, v = rv;
            float h = kept, d[SE];
            if (AHEAD) ask(k - 1);
            float s = into_lane<false, G>(q.map(), h);
            Map m = {1.f, 0.f};
#pragma unroll
            for (int e = SE - 1; e >= 0; --e) {
                d[e] = g.v ? to_f32(dy.v[e]) * to_f32(v.v[e]) : to_f32(dy.v[e]);
                if (!all) d[e] = col + e < len ? d[e] : 0.f;
                m.x = q.a[e] * (d[e] + m.x);
                m.a *= q.a[e];
            }
            float r = into_lane<true, G>(m, p);
#pragma unroll
            for (int e = SE - 1; e >= 0; --e) {
                d[e] += r;                                       // dh
                r = q.a[e] * d[e];
            }
#pragma unroll
            for (int e = 0; e < SE; ++e) {
                const float before = s;
                s = fmaf(q.a[e], s, q.x[e]);
                float gu, gw;
                if (g.log_gate) {
                    gu = d[e];
                    gw = to_f32(w.v[e]) > 0.f ? 0.f : d[e] * before * q.a[e];
                } else {
                    gu = d[e] * q.rest[e];
                    gw = d[e] * (before - q.u[e]) * (q.a[e] * q.rest[e]);
                }
                const bool in = all || col + e < len;
                du[e] = from_f32<T>(in ? gu : 0.f);
                dw[e] = from_f32<T>(in ? gw : 0.f);
                dv[e] = from_f32<T>(in ? to_f32(dy.v[e]) * s : 0.f);
            }
        } else if (AHEAD) {
            ask(k - 1);
        }
        if (there && (!WHOLE || col < g.N)) {
            const int64_t at = row * g.N + col, left = WHOLE ? SE : g.N - col;
            put<T>((T *)g.du + at, left, du, g.beyond_cache);
            put<T>((T *)g.dw + at, left, dw, g.beyond_cache);
            if (g.v) put<T>((T *)g.dv + at, left, dv, g.beyond_cache);
        }
        if (!AHEAD) ask(k - 1);
    }
    if (g.dstate && lane == 0 && there && seg == 0) g.dstate[row] = p;
}

struct StepArgs {
    const void *u, *w, *v;
    const float *state;
    float *next;
    void *y;
    int64_t T, first;
    int log_gate;
};

// One token: a value a lane. 1 x 768: the call is what it costs.
template <typename T> __global__ void __launch_bounds__(256) k_step(const StepArgs g)
{
    const int64_t i = g.first + (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= g.T) return;
    float a, rest;
    const float u = to_f32(((const T *)g.u)[i]);
    gate_of<T>(to_f32(((const T *)g.w)[i]), g.log_gate, a, rest);
    const float h = fmaf(a, g.state[i], g.log_gate ? u : rest * u);
    g.next[i] = h;
    ((T *)g.y)[i] = from_f32<T>(g.v ? h * to_f32(((const T *)g.v)[i]) : h);
}

// Into how many segments a row goes. A wave takes about 0.9 us for 512 samples (gradients 1.4) however few waves there are; a second kernel costs 2.5 us and
// reads u and w (w, v and dy) again. bf16, forward and backward in us: 500 rows of 2048 in one 5.9 and 7.9, in four 7.8 and 8.8; of 4096 9.1 and
// 13.6, in eight 9.2 and 12.2; of 8192 17 and 24, 13.7 and 19; 1024 rows of 16384 32 and 50, in eight 37 and 55; 256 rows of 4096 8.9 and 13.4, 8.0 and 9.1;
// 16 rows of 65536 110 and 173, in 128 7.9 and 9.5. So: rows of more than 2048 samples, fewer than 1024 of them, and no more than 64 for each 512
// samples, in as many segments as bring 32 waves to a compute unit.
static int scan_segments(int64_t rows, int64_t N)
{
    const int64_t chunks = (N + 64 * SE - 1) / (64 * SE);
    if (rows < 1 || rows >= 1024 || chunks <= 4 || chunks * 64 < rows) return 1;
    const int64_t most = (8192 + rows - 1) / rows, per = most < chunks ? (chunks + most - 1) / most : 1;
    return (int)((chunks + per - 1) / per);
}

size_t gated_scan_workspace(int64_t rows, int64_t N)
{
    const int s = scan_segments(rows, N);
    return s > 1 ? (size_t)rows * s * sizeof(float2) : 0;
}

template <typename T> static int run(ScanArgs &g, bool back, hipStream_t s)
{
    // lanes of a row
    const int lanes = g.N <= SE ? 1 : g.N <= 4 * SE ? 4 : g.N <= 16 * SE ? 16 : 64;
    const bool whole = g.N % SE == 0;
    g.chunks = (int)((g.N + lanes * SE - 1) / (lanes * SE));
    g.segments = scan_segments(g.rows, g.N);
    g.beyond_cache = g.rows * g.N > ((int64_t)256 << 20) / (int64_t)sizeof(T);
    g.per = (g.chunks + g.segments - 1) / g.segments;
    auto launch = [&](auto kernel, int64_t groups) -> int {
        return in_pieces(groups, 256, [&](int64_t first, unsigned n) -> int {
            g.first = first * (256 / lanes);
            kernel<<<n, 256, 0, s>>>(g);
            FC_HIP(hipGetLastError());
            return FFTCONV_OK;
        });
    };
    if (g.segments > 1) {
        const int64_t groups = (g.rows * (g.segments - 1) + 3) / 4;
        FC_TRY(back ? launch(whole ? k_scan_maps<T, true, true> : k_scan_maps<T, true, false>, groups)
                    : launch(whole ? k_scan_maps<T, false, true> : k_scan_maps<T, false, false>, groups));
    }
    const int64_t groups = (g.rows * g.segments + 256 / lanes - 1) / (256 / lanes);
    if (back) {
        if (lanes == 1) return launch(k_scan_back<T, 1, false, false>, groups);
        if (lanes == 4) return launch(k_scan_back<T, 4, false, false>, groups);
        if (lanes == 16) return launch(k_scan_back<T, 16, false, false>, groups);
        // With 64 waves to a compute unit enough is on its way without asking ahead (bf16 64 x 768 x 4096 forward and backward 806 us, with it 818), and waves of
        // one piece have nothing to ask for: without, four of fp32 fit where three do with it (1 x 16 x 131072 12.5 us).
        if (g.per == 1 || g.rows * g.segments >= 16384) return launch(whole ? k_scan_back<T, 64, true, false> : k_scan_back<T, 64, false, false>, groups);
        return launch(whole ? k_scan_back<T, 64, true, true> : k_scan_back<T, 64, false, true>, groups);
    }
    if (lanes == 1) return launch(k_scan<T, 1, false>, groups);
    if (lanes == 4) return launch(k_scan<T, 4, false>, groups);
    if (lanes == 16) return launch(k_scan<T, 16, false>, groups);
    return launch(whole ? k_scan<T, 64, true> : k_scan<T, 64, false>, groups);
}

static int run(ScanArgs &g, bool back, int dtype, hipStream_t s)
{
    return dtype == FFTCONV_BF16 ? run<__bf16>(g, back, s) : dtype == FFTCONV_F16 ? run<_Float16>(g, back, s) : run<float>(g, back, s);
}

int gated_scan(const void *u, const void *w, const void *v, const float *state, const int32_t *lengths, void *y, float *last, float *kept, int64_t B,
               int64_t C, int64_t N, int gate, int dtype, void *workspace, hipStream_t s)
{
    ScanArgs g = {};
    g.u = u, g.w = w, g.v = v, g.state = state, g.lengths = lengths, g.y = y, g.last = last, g.kept = kept;
    g.rows = B * C, g.N = N, g.C = (int)C, g.log_gate = gate == 1, g.maps = (float2 *)workspace;
    return run(g, false, dtype, s);
}

int gated_scan_backward(const void *dy, const void *u, const void *w, const void *v, const float *kept, const float *dlast, const int32_t *lengths,
                        void *du, void *dw, void *dv, float *dstate, int64_t B, int64_t C, int64_t N, int gate, int dtype, void *workspace,
                        hipStream_t s)
{
    ScanArgs g = {};
    g.dy = dy, g.u = u, g.w = w, g.v = v, g.kept_in = kept, g.dlast = dlast, g.lengths = lengths, g.du = du, g.dw = dw, g.dv = dv, g.dstate = dstate;
    g.rows = B * C, g.N = N, g.C = (int)C, g.log_gate = gate == 1, g.maps = (float2 *)workspace;
    return run(g, true, dtype, s);
}

int gated_step(const void *u, const void *w, const void *v, const float *state, float *next, void *y, int64_t T, int gate, int dtype, hipStream_t s)
{
    StepArgs g = {u, w, v, state, next, y, T, 0, gate == 1};
    return in_pieces((T + 255) / 256, 256, [&](int64_t first, unsigned n) -> int {
        g.first = first * 256;
        if (dtype == FFTCONV_BF16) k_step<__bf16><<<n, 256, 0, s>>>(g);
        else if (dtype == FFTCONV_F16) k_step<_Float16><<<n, 256, 0, s>>>(g);
        else k_step<float><<<n, 256, 0, s>>>(g);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    });
}

}  // namespace lay
}  // namespace fftconv
