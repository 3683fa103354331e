// Copies of 16 bytes per lane into LDS at an LDS address (lds_address): no pointer arithmetic or test per copy.
#pragma once

#include "common.h"

namespace pr2 {

__device__ __forceinline__ uint32_t lds_address(const unsigned char* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const lds_void*)p);
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// from an address per lane
__device__ __forceinline__ void dma16_to(const void* src, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 1\n\tglobal_load_lds_dwordx4 %0, off"
                 :
                 : "v"(src), "s"(to)
                 : "memory", "m0");
}
// from a wavefront-uniform base plus a 32-bit byte offset per lane
__device__ __forceinline__ void dma16_to(const void* base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 1\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(off), "s"(base), "s"(to)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

}  // namespace pr2
