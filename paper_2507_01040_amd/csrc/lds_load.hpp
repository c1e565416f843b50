// Loads from memory straight to LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cliff {

constexpr uint32_t NOWHERE = 0x80000000u;  // past every descriptor's end: loads zeros

// 16 bytes at a byte offset of each lane from an address of the wave, to LDS from
// `to` on, lane after lane.  Inline asm without outputs: as a builtin, every
// transposing read of LDS, of another buffer too, waits for all of them.
__device__ inline void load_to_lds(const void* from, uint32_t offset, char* to)
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) void lds_void;
    const uint64_t address = (uint64_t)from;
    const u4 d = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)address),
                  (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(address >> 32)) & 0xffffu, 0x7fffffffu,
                  0x00020000u};
    __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"((uint32_t)(uintptr_t)(lds_void*)to), "v"(offset), "s"(d)
                     : "memory", "m0");
}

// Until this wave's loads have arrived (vmcnt 0).
__device__ inline void wait_direct() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Until all but the last N of them have (N < 16).
template <int N>
__device__ inline void wait_direct_but()
{
    __builtin_amdgcn_s_waitcnt(0x0f70 | N);
    __asm__ volatile("" ::: "memory");
}

// A barrier that waits for nothing but the other waves: reads of LDS that are under
// way stay so.
__device__ inline void barrier_alone() { __asm__ volatile("s_barrier" ::: "memory"); }

}  // namespace cliff
