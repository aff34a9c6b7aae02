// Transfers from memory straight to LDS (no register waits for them; vmcnt counts them like loads), written as instructions because the compiler
// waits for all of them before any read of LDS: FC_ARRIVED waits for the right ones. M0, which holds the place in LDS, is used by nothing else
// in the kernels that include this.
#pragma once

#include "layers_internal.h"

namespace fftconv {
namespace lay {

static __device__ const uint4 zero_piece = {0, 0, 0, 0};      // what is brought for places beyond a tensor's end

__device__ __forceinline__ uint32_t lds_offset(const char *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p; }
// An address that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
    return (const char *)(uintptr_t)((uint64_t)hi << 32 | lo);
}
// 16 (or 4) bytes for each lane from base + off to LDS, at `to` + 16 (or 4) * lane.
__device__ __forceinline__ void to_lds16(const char *base, uint32_t off, const char *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds_offset(to))), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void to_lds16(const char *from, const char *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds_offset(to))), "v"(from) : "memory");
}
__device__ __forceinline__ void to_lds4(const char *base, uint32_t off, const char *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds_offset(to))), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void to_lds4(const char *from, const char *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds_offset(to))), "v"(from) : "memory");
}
// N such in a row, 1024 bytes apart in LDS. The instruction's own offset moves both addresses, so off[i] is 1024 i less than the distance from base
// (callers keep base below the first byte by as much as that needs).
template <int N> __device__ __forceinline__ void to_lds16_rows(const char *base, const uint32_t (&off)[N], uint32_t to)
{
    static_assert(N == 2 || N == 4, "rows");
    if constexpr (N == 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                     "global_load_lds_dwordx4 %3, %5 offset:2048\n\tglobal_load_lds_dwordx4 %4, %5 offset:3072" ::"s"(to), "v"(off[0]), "v"(off[1]),
                     "v"(off[2]), "v"(off[3]), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(to), "v"(off[0]),
                     "v"(off[1]), "s"(base) : "memory");
}

// Waits until at most `left` of this wave's transfers are on their way, then for the other waves; this wave's reads of LDS are done by then.
#ifdef FFTCONV_SYNC_CHECK
#define FC_ARRIVED(left) do { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); __syncthreads(); } while (0)
#else
#define FC_ARRIVED(left) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(left) : "memory")
#endif

}  // namespace lay
}  // namespace fftconv
