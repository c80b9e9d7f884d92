// Loads from global memory straight into LDS, and what orders them: of the tile kernels of the products and of attention.
#pragma once
#include <hip/hip_runtime.h>

namespace enc {
namespace tile {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// (M0 holds the LDS address; the instruction may follow M0's write only after a wait state)
__device__ __forceinline__ void load16_to_lds(const void *base, unsigned offset, unsigned lds_addr)
{
    asm volatile("s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(offset), "s"(base), "{m0}"(lds_addr)
                 : "memory");
}
__device__ __forceinline__ void load4_to_lds(const void *base, unsigned offset, unsigned lds_addr)
{
    asm volatile("s_nop 0\n\t"
                 "global_load_lds_dword %0, %1"
                 :
                 : "v"(offset), "s"(base), "{m0}"(lds_addr)
                 : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// A barrier that no access to LDS is moved across.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

} // namespace tile
} // namespace enc
