// Tiles that go from memory straight to shared memory, several stages ahead of
// the matrix instructions that read them (linear8.hip, weight_gradient.hip).
//
// A wavefront's load brings 64 pieces of 16 bytes (or 4), each lane's from an
// address of its own, to 64 places in a row of shared memory.  Pieces past the
// range that the descriptor gives become zeros, so tiles need no case for their
// borders.  The loads are counted by the wavefront (vmcnt) and waited for by
// number: `wait_loads<N>` returns when all but the last N have arrived.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace rocket {

typedef int Int4 __attribute__((ext_vector_type(4)));

// A buffer of `bytes` (clamped into [0, 2^31 - 1]) at an address that is the
// same for the whole wavefront; offsets past it read zeros.
//
// A load may read a scalar register only 5 wait states after a vector instruction
// (readfirstlane is one) has written it.  The compiler does not see the loads below, so
// the wait stands here: nothing reads the buffer before it.
__device__ inline Int4 buffer_of(const void *p, int64_t bytes) {
    const uint64_t at = (uint64_t)p;
    const int n = bytes < 0 ? 0 : bytes > INT32_MAX ? INT32_MAX : (int)bytes;
    Int4 buffer = {__builtin_amdgcn_readfirstlane((int)at), __builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xffff),
                   __builtin_amdgcn_readfirstlane(n), 0x00020000};
    asm volatile("s_nop 4" : "+s"(buffer));
    return buffer;
}

// An offset that is past every buffer.
constexpr uint32_t kNowhere = 0x80000000u;

__device__ inline uint32_t shared_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

typedef __attribute__((address_space(3))) char *Shared;

__device__ inline Shared shared_at(uint32_t at) { return (Shared)(uintptr_t)at; }

// 64 pieces of 16 bytes to shared memory from `to` on, a lane's from `offset` and
// `more`, which is the same for all and at most the buffer's bytes (walk.h).  Written in
// assembly since the compiler would wait for every load before the next read of shared
// memory; it has no result, and M0, which it sets, holds nothing of the compiler's here.
__device__ inline void load_stage16(const Int4 &buffer, uint32_t to, uint32_t offset, uint32_t more = 0) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, %3 offen lds"
        :
        : "s"(to), "v"(offset), "s"(buffer), "s"(more)
        : "memory");
}

__device__ inline void load_stage4(const Int4 &buffer, uint32_t to, uint32_t offset) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dword %1, %2, 0 offen lds"
        :
        : "s"(to), "v"(offset), "s"(buffer)
        : "memory");
}

// Until all but the last N loads of this wavefront have arrived, and what it read
// from shared memory is in registers; then every wavefront of the workgroup.
template <int N>
__device__ inline void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace rocket
