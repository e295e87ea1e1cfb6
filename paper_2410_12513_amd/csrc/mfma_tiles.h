// Pieces that the kernels on the matrix cores share: operand types, splits into bf16 parts, loads that go straight into LDS.
#pragma once
#include "common.h"

namespace first {

constexpr float LOG2E = 1.4426950408889634f;

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16_t;

// hi = bf16(x), lo = bf16(x - hi) for a pair
__device__ __forceinline__ void split_pair(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pk_bf16(a, b);
  lo = pk_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}

// 16 bytes per lane from (descriptor base + voff + soff) to LDS byte lds_off + 16 * lane.  No vector register is written: nothing
// for the compiler to reuse too early; pg_wait / lds_barrier order it.  The LDS offset travels in m0, as an operand: it is the
// compiler that writes the register, so it knows (m0 written in the asm text would be a write it knows nothing of).
typedef int i32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void pg_load_lds(uint32_t lds_off, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(lds_off), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}
__device__ __forceinline__ i32x4_t pg_rsrc(const void* p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  i32x4_t r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff);
  r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
  r[3] = 0x00020000;
  return r;
}
// The same where the descriptor or the offset may come out of a vector register's lanes (v_readlane, v_readfirstlane) right ahead of the load - a kernel that
// holds more scalars than there are registers keeps some there.  The part asks for five wait states between such a write and a memory instruction that reads it; the compiler
// keeps them for its own instructions and does not see one in this text.  (Without them a descriptor's last word was read too early once, and the load faulted.)
__device__ __forceinline__ void pg_load_lds_any(uint32_t lds_off, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(lds_off), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}
template <int N> __device__ __forceinline__ void pg_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// x in both halves of the wave -> (value of lane % 32 in the lower half, in the upper half)
__device__ __forceinline__ void both_halves(float x, float& lower, float& upper) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  lower = __uint_as_float(r[0]); upper = __uint_as_float(r[1]);
}

}  // namespace first
