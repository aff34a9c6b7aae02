// The 2-norm over many tensors together, and the tensors times min(1, limit / (norm + eps)).
//
// Squares are added in 64 bits: bf16 and fp32 numbers of any size stay in range, and a billion of them lose nothing that fp32 shows. Every workgroup adds
// up a stretch of the tensors' pieces in an order of its own, one more adds the workgroups' sums, so results do not depend on timing. Where the tensors
// are comes with the launch (up to 128 of them to one): nothing is copied to the device beforehand.
//
// Bound by bytes: a first pass reads, a second reads again and writes, last pieces first, for what the first read last is still in the memory-side cache.
// Where the factor is one, what would be written in place is left alone. Measured: 604 million values, 403 million of them bf16, the rest fp32, into fp32:
// 285 to 292 us (5.5 to 5.7 TB/s) and 800 (5.0, more than half of it stores); stores past the cache in whole lines give the next call's first pass 30 us and lose 5. A dozen
// tensors of 1.9 MB together: 4.2 and 4.7 us, the call on the host 20.
#include <cstdlib>

#include "layers_internal.h"

namespace fftconv {
namespace lay {

constexpr int TENSORS = 128, PIECE = 8192;       // tensors to a launch; values of a piece

struct Tensors {
    const void *in[TENSORS];
    void *out[TENSORS];
    int64_t count[TENSORS];
    uint32_t start[TENSORS + 1];                 // pieces before a tensor's own
    uint8_t type[TENSORS];                       // of the values, and of those written, times 4
    int n;
};

struct ClipArgs {
    double *sums;                                // of the workgroups of the first pass, one each
    double *total;                               // the norm
    const float *norm;                           // one that came with the call
    float *norm_out;
    double limit, eps;
    int64_t count;                               // sums, where the second pass adds them up itself
};

// f(tensor, first value, values) for this workgroup's pieces: every gridDim.x'th, from the first on, or with DOWN from the last.
template <bool DOWN, typename F> __device__ __forceinline__ void each_piece(const Tensors &t, F f)
{
    const uint32_t all = t.start[t.n];
    int lo = DOWN ? t.n - 1 : 0;
    for (uint32_t i = blockIdx.x; i < all; i += gridDim.x) {
        const uint32_t at = DOWN ? all - 1 - i : i;
        if (DOWN) while (t.start[lo] > at) --lo;
        else while (t.start[lo + 1] <= at) ++lo;
        const int64_t first = (int64_t)(at - t.start[lo]) * PIECE, left = t.count[lo] - first;
        f(lo, first, (int)(left < PIECE ? left : PIECE));
    }
}

template <typename T> __device__ __forceinline__ void add_squares(const void *p, int64_t first, int count, double &sum)
{
    const T *const x = (const T *)p + first;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = (threadIdx.x + i * 256) * 8;
        load_piece<T, 8>(x + at, count - at, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)v[i][e], (double)v[i][e], sum);
}

// The workgroup's sum, in every thread.
__device__ __forceinline__ double group_sum(double x)
{
    __shared__ double part[4];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}
__device__ __forceinline__ double norm_of(const double *sums, int64_t n)
{
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) sum += sums[i];
    return sqrt(group_sum(sum));
}

__global__ void __launch_bounds__(256) k_squares(const Tensors t, const ClipArgs a)
{
    static_assert(PIECE == 256 * 32, "four times eight values to a thread");
    double sum = 0.0;
    each_piece<false>(t, [&](int i, int64_t first, int count) {
        const int type = t.type[i] & 3;
        if (type == FFTCONV_F32) add_squares<float>(t.in[i], first, count, sum);
        else if (type == FFTCONV_F16) add_squares<_Float16>(t.in[i], first, count, sum);
        else add_squares<__bf16>(t.in[i], first, count, sum);
    });
    sum = group_sum(sum);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(256) k_norm(const ClipArgs a)
{
    const double norm = norm_of(a.sums, a.count);
    if (threadIdx.x == 0) {
        *a.total = norm;
        if (a.norm_out) *a.norm_out = (float)norm;
    }
}

// A norm that came with the call, to where the call wants it.
__global__ void k_given(const ClipArgs a) { *a.norm_out = *a.norm; }

template <typename T, typename O> __device__ __forceinline__ void scale_piece(const void *in, void *out, int64_t first, int count, float by)
{
    const T *const x = (const T *)in + first;
    O *const y = (O *)out + first;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = (threadIdx.x + i * 256) * 8;
        load_piece<T, 8>(x + at, count - at, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = (threadIdx.x + i * 256) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] *= by;
        store_rounded<O, 8>(y + at, count - at, v[i]);
    }
}

__global__ void __launch_bounds__(256) k_clip(const Tensors t, const ClipArgs a)
{
    const double norm = a.norm ? (double)*a.norm : a.count ? norm_of(a.sums, a.count) : *a.total;
    if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
    const double c = a.limit / (norm + a.eps);
    const bool all = isinf(a.limit) && !isnan(norm);                 // (by an infinite norm the quotient is no number, and there is nothing to clip)
    const float by = c > 1.0 || all ? 1.f : (float)c;                // (a norm that is no number makes everything so)
    each_piece<true>(t, [&](int i, int64_t first, int count) {
        const int type = t.type[i] & 3;
        const bool wide = t.type[i] >> 2 == FFTCONV_F32;
        if (by == 1.f && t.in[i] == t.out[i]) return;
        if (type == FFTCONV_F32) scale_piece<float, float>(t.in[i], t.out[i], first, count, by);
        else if (type == FFTCONV_F16 && wide) scale_piece<_Float16, float>(t.in[i], t.out[i], first, count, by);
        else if (type == FFTCONV_F16) scale_piece<_Float16, _Float16>(t.in[i], t.out[i], first, count, by);
        else if (wide) scale_piece<__bf16, float>(t.in[i], t.out[i], first, count, by);
        else scale_piece<__bf16, __bf16>(t.in[i], t.out[i], first, count, by);
    });
}

// The launches of a call: f(tensors, workgroups), one after the other, from the last with `down`, until one returns a code.
template <typename F> static int each_launch(const void *const *in, void *const *out, const int64_t *counts, const int *types, const int *types_out,
                                             int64_t tensors, bool down, F f)
{
    for (int64_t i = down ? tensors - 1 : 0; down ? i >= 0 : i < tensors;) {
        Tensors t = {};
        uint32_t pieces = 0;
        // (2^31 pieces to a launch at most)
        for (; (down ? i >= 0 : i < tensors) && t.n < TENSORS; i += down ? -1 : 1) {
            if (counts[i] < 1) continue;
            const uint32_t more = (uint32_t)((counts[i] + PIECE - 1) / PIECE);
            if (pieces + more > 1u << 31) break;
            t.in[t.n] = in ? in[i] : nullptr, t.out[t.n] = out ? out[i] : nullptr, t.count[t.n] = counts[i];
            t.type[t.n] = types ? (uint8_t)(types[i] | (types_out ? types_out[i] : types[i]) << 2) : 0;
            t.start[t.n++] = pieces;
            pieces += more;
        }
        t.start[t.n] = pieces;
        if (t.n == 0) continue;
        if (const int rc = f(t, pieces < 2048 ? pieces : 2048u)) return rc;
    }
    return FFTCONV_OK;
}

size_t clip_workspace(const int64_t *counts, int64_t tensors)
{
    size_t n = 1;
    (void)each_launch(nullptr, nullptr, counts, nullptr, nullptr, tensors, false, [&](const Tensors &, uint32_t groups) { n += groups; return FFTCONV_OK; });
    return n * sizeof(double);
}

struct Span {
    uintptr_t from, to;
    int64_t i;
};
static int by_place(const void *a, const void *b)
{
    const uintptr_t x = ((const Span *)a)->from, y = ((const Span *)b)->from;
    return x < y ? -1 : x > y;
}

// Whether what is written is written once, and read by nothing else: results (each may be its own gradient), the norm and the workspace's sums. A norm that is
// given is read by every workgroup while others write. -1: no memory.
int clip_overlaps(const void *const *in, void *const *out, const int64_t *counts, const int *types, const int *types_out, int64_t tensors,
                  const float *norm_in, const float *norm, const void *workspace)
{
    Span *const s = (Span *)malloc(sizeof(Span) * (size_t)(tensors + 2));
    if (!s) return -1;
    int64_t n = 0;
    for (int64_t i = 0; out && i < tensors; ++i)
        if (counts[i] > 0) s[n++] = {(uintptr_t)out[i], (uintptr_t)out[i] + (uintptr_t)counts[i] * (types_out[i] == FFTCONV_F32 ? 4 : 2), i};
    if (norm && norm != norm_in) s[n++] = {(uintptr_t)norm, (uintptr_t)(norm + 1), -1};
    if (!norm_in) s[n++] = {(uintptr_t)workspace, (uintptr_t)workspace + clip_workspace(counts, tensors), -1};
    qsort(s, (size_t)n, sizeof(Span), by_place);
    int found = 0;
    for (int64_t k = 1; k < n; ++k) found |= s[k].from < s[k - 1].to;
    auto read = [&](uintptr_t from, uintptr_t to, int64_t i) {
        int64_t lo = 0, hi = n;                  // spans before lo end at or before `from`
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (s[mid].to <= from) lo = mid + 1;
            else hi = mid;
        }
        for (; lo < n && s[lo].from < to; ++lo) found |= s[lo].i != i || s[lo].from != from || s[lo].to != to;
    };
    for (int64_t i = 0; i < tensors && !found; ++i)
        if (counts[i] > 0) read((uintptr_t)in[i], (uintptr_t)in[i] + (uintptr_t)counts[i] * (types[i] == FFTCONV_F32 ? 4 : 2), i);
    if (norm_in) read((uintptr_t)norm_in, (uintptr_t)(norm_in + 1), -2);
    free(s);
    return found;
}

int clip_grads(const void *const *in, void *const *out, const int64_t *counts, const int *types, const int *types_out, int64_t tensors, double limit,
               double eps, const float *norm_in, float *norm, void *workspace, hipStream_t s)
{
    // (up to 512 sums are added up by every workgroup of the second pass, and a launch is saved)
    double *const total = (double *)workspace;
    ClipArgs a = {total ? total + 1 : nullptr, total, norm_in, nullptr, limit, eps, 0};
    if (!norm_in) {
        int64_t sums = 0;
        FC_TRY(each_launch(in, nullptr, counts, types, nullptr, tensors, false, [&](const Tensors &t, uint32_t groups) -> int {
            k_squares<<<groups, 256, 0, s>>>(t, a);
            FC_HIP(hipGetLastError());
            a.sums += groups, sums += groups;
            return FFTCONV_OK;
        }));
        a.sums = total + 1, a.count = sums, a.norm_out = norm;
        if (!out || sums == 0 || sums > 512) {
            k_norm<<<1, 256, 0, s>>>(a);
            FC_HIP(hipGetLastError());
            a.count = 0, a.norm_out = nullptr;
        }
    }
    if (norm_in && norm && norm != norm_in) {
        a.norm_out = norm;
        k_given<<<1, 1, 0, s>>>(a);
        FC_HIP(hipGetLastError());
        a.norm_out = nullptr;
    }
    if (!out) return FFTCONV_OK;
    return each_launch(in, out, counts, types, types_out, tensors, true, [&](const Tensors &t, uint32_t groups) -> int {
        k_clip<<<groups, 256, 0, s>>>(t, a);
        FC_HIP(hipGetLastError());
        return FFTCONV_OK;
    });
}

}  // namespace lay
}  // namespace fftconv
