// Direct-to-LDS loads, their waits and LDS addresses.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace realq {

// 16-byte direct-to-LDS load: lane i reads base + off (its own 32-bit byte offset) and fills LDS bytes lds + 16 i ..
// + 15 (base and lds are wave-uniform).  Inline assembly, so that the compiler does not insert conservative waits
// for it: every consumer is ordered by the explicit vmcnt waits and barriers of its loop.  s_nop: the load reads M0
// as its LDS address and needs a wait state behind the scalar write of it, which the compiler does not insert here.
__device__ __forceinline__ void to_lds(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds)
                 : "memory", "m0");
}
// Until at most N vector memory operations of the wave are under way.
template <int N>
__device__ __forceinline__ void vm_wait() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// LDS byte address of a __shared__ object: the low 32 bits of its generic address.
__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(uintptr_t)p; }

}  // namespace realq
