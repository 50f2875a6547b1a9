// Loads from HBM to LDS that pass no registers, and what orders them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "vectors.h"

namespace pase {

typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return (uint32_t) reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)p);
}

// 16 bytes a lane from buffer r, byte offset `at`, to LDS byte dst + 16 * lane (dst
// the same for the wave, through M0, which nothing else here uses).  The load has no register result; whoever reads the
// LDS bytes waits for it by wait_loads().  The builtin of the same instruction
// makes the compiler wait for every such load before each transposing LDS read,
// a step too early: 16384 x 4096 x 4096 rows gradient 510 us with it, 436 without.
__device__ __forceinline__ void load_to_lds(u32x4 r, int at, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(at), "s"(r) : "memory");
}

// The same with 4 bytes a lane.
__device__ __forceinline__ void load_words_to_lds(u32x4 r, int at, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(dst), "v"(at), "s"(r) : "memory");
}

// The descriptor of `bytes` bytes from p on (both the same for the wave): what lies past them reads as 0.
__device__ __forceinline__ u32x4 buffer_of(const void *p, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)at),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xffff),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}

// All but the last N loads and stores of this wave have ended, and its LDS reads.
template <int N> __device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// A barrier alone: what it orders is waited for where it is needed.
__device__ __forceinline__ void barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A transposing LDS read: sixteen lanes read 4 rows x 16 columns of 16 bits, lane l the four columns from its
// address on of row l / 4; it gets the four rows of column l.
__device__ __forceinline__ s16x4 read_across(uint32_t at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)at);
}

}  // namespace pase
