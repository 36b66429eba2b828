// rm_lds.h -- loads from memory to LDS past the registers (prompt.hip, f8.hip).  Not
// part of the C ABI.
#pragma once

#include "rm_decode.h"

namespace rm {

// 16 bytes a lane from base + offset to LDS, lane by lane behind each other.  Not
// the builtin: the compiler would wait for all of it before the next read of LDS.
// m0 is a register that the compiler sets only beside its use.
__device__ inline void to_lds16(uint32_t lds, uint32_t offset, const uint8_t* base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds), "v"(offset), "s"(base) : "memory");
}
// 4 bytes a lane from an address of its own.
__device__ inline void to_lds4(uint32_t lds, const void* from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 :: "s"(lds), "v"(from) : "memory");
}
// An address that all lanes agree on, in scalar registers.
__device__ inline const uint8_t* scalar(const uint8_t* p)
{
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const uint8_t*)(uintptr_t)((uint64_t)hi << 32 | lo);
}
__device__ inline uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

}  // namespace rm
