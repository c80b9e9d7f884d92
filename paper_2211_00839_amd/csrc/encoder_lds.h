// Loads from global memory straight into LDS, and what orders them: of the tile kernels of the products and of attention.
#pragma once
#include <hip/hip_runtime.h>

namespace enc {
namespace tile {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// 16 or 4 bytes of each lane, from a base that all lanes share.  M0 holds the LDS address; the instruction may follow M0's write only after a wait
// state, and the base's by five where a vector instruction wrote it: a register that was held in a lane of another one comes back so, and the
// compiler, which does not see into the asm, puts nothing between.  s_nop 4 is five.
__device__ __forceinline__ void load16_to_lds(const void *base, unsigned offset, unsigned lds_addr)
{
    asm volatile("s_nop 4\n\t"
                 "global_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(offset), "s"(base), "{m0}"(lds_addr)
                 : "memory");
}
__device__ __forceinline__ void load4_to_lds(const void *base, unsigned offset, unsigned lds_addr)
{
    asm volatile("s_nop 4\n\t"
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
