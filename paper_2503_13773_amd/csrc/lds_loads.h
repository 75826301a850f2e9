// Loads from memory straight into LDS, into a stage that one wavefront has for itself: nothing passes through registers, no barrier.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvc {

// 16 bytes per lane from base + off to LDS at lds_addr + 16 * lane; base and lds_addr are uniform.  The compiler does not see these
// accesses: the wavefront waits for them with wait_for_loads().  AGAIN: other wavefronts are about to read the same bytes.
template <bool AGAIN>
__device__ inline void load_to_lds(const unsigned char *base, uint32_t off, uint32_t lds_addr) {
    if constexpr (AGAIN)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds_addr), "v"(off), "s"(base) : "memory");
}
template <bool AGAIN>
__device__ inline void load_to_lds(const unsigned char *addr, uint32_t lds_addr) {
    if constexpr (AGAIN) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(addr) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(lds_addr), "v"(addr) : "memory");
}
// At most N of the wavefront's loads are under way after it.  (Loads that the compiler issued in between make the wait longer, never shorter.)
template <int N>
__device__ inline void wait_for_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// What LDS reads come from may be overwritten after it.
__device__ inline void wait_for_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

}  // namespace kvc
