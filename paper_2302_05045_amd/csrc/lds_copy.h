// Copies from global memory straight into LDS, the transposing LDS read and the bare barrier: what the matrix kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace samo {
namespace {

#define LDS_AS __attribute__((address_space(3)))
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));

__device__ __attribute__((aligned(16))) const unsigned char zero_row[16] = {0};

// One copy instruction: the wave's 64 x 16 bytes from the lanes' global addresses to LDS at
// lds_byte_addr + 16 * lane.  It writes M0, a register the compiler reserves and does not let an
// asm statement declare as clobbered; nothing else in these kernels makes the compiler use M0 (no
// register arrays indexed at run time, no other LDS-direct or GWS operation).
__device__ __forceinline__ void dma16(const void *g, unsigned lds_byte_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(g), "s"(lds_byte_addr) : "memory");
}

// The same with the global addresses as a scalar base plus a 32-bit offset per lane.  A scalar
// register that a vector instruction has written (the compiler may have parked the base in one) must
// not be read by a memory instruction for five cycles: the wait states in front cover that.
__device__ __forceinline__ void dma16_from(const void *base, unsigned lane_offset, unsigned lds_byte_addr)
{
    asm volatile("s_nop 3\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_offset), "s"(base), "s"(lds_byte_addr)
                 : "memory");
}

// 8 tokens of one feature for an MFMA lane: two transposing reads of one token of four LDS rows each,
// the rows' tokens `step` bytes apart.
__device__ __forceinline__ half8 read_fragment(const unsigned char *p, int step)
{
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS short4v *)(LDS_AS unsigned char *)p);
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS short4v *)(LDS_AS unsigned char *)(p + step));
    const short8v q = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(half8, q);
}

// A pointer all lanes of a wave agree on, told to the compiler.
__device__ __forceinline__ const unsigned char *uniform(const unsigned char *p)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const unsigned char *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a) |
                                                   (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)) << 32);
}

// A bare workgroup barrier: what has to be complete before it is waited for explicitly.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace
}  // namespace samo
