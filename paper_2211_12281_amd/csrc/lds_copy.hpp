// Asynchronous copies from memory to the LDS, for the products of 8-bit matrices (matmul_quantized.hip, matmul_rowwise.hip).
#pragma once
#include "kge_internal.h"

__device__ __forceinline__ void kge_copy16(const void *g, uint32_t lds) {
    // lane l's 16 bytes go to LDS address lds + 16 l; tracked by vmcnt, unseen by the compiler
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(g) : "memory");
}
__device__ __forceinline__ void kge_copy4(const void *g, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(g) : "memory");
}
// the same from base + a 32-bit offset of each lane
__device__ __forceinline__ void kge_copy16(const uint8_t *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void kge_copy4(const uint8_t *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
template <int N> __device__ __forceinline__ void kge_wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
