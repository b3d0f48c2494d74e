// Matrix-core and LDS helpers shared by the attention-block kernels (moe_linear,
// moe_latent, moe_prefill).
//
// Operand layout of mfma_f32_16x16x32_f16 (lane l, c = l % 16, g = l / 16):
//   A: row c, k = 8 g .. 8 g + 7;  B: column c, the same k;
//   D: column c, rows 4 g .. 4 g + 3.
#pragma once

#include "moe_device.h"

namespace moe {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f4 mfma16(h8 a, h8 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// 16 bytes as eight halves, from global memory or LDS.
__device__ __forceinline__ h8 ld_h8(const void* p) { return *reinterpret_cast<const h8*>(p); }

// Four rows of 16 halves in LDS, read by a group of 16 lanes and transposed: lane i of
// the group passes the address of row i / 4, columns 4 (i % 4) .. + 3, and receives
// column i of the four rows.
__device__ __forceinline__ h4 ld_tr(const void* p) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s4*)(__attribute__((address_space(3))) char*)p);
  return __builtin_bit_cast(h4, v);
}
__device__ __forceinline__ h8 join(h4 a, h4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The LDS address of a shared object.
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// Each lane copies 16 bytes from its own global address to LDS address to + 16 * lane (`to`
// the same for the wave). The compiler does not see it as a memory instruction: vm_wait
// orders it, and every wave waits before the barrier behind which the data is read. (`to`
// goes through m0, which nothing else in these kernels uses.)
__device__ __forceinline__ void dma16(const void* g, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(g)
      : "memory");
}
// The same from a base that the wave shares, with a byte offset per lane.
__device__ __forceinline__ void dma16(const void* base, uint32_t off, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base)
      : "memory");
}
// Four bytes a lane, to lds + 4 * lane.
__device__ __forceinline__ void dma4(const void* g, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %1, off"
      :
      : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(g)
      : "memory");
}
// An int that the whole wave reads and nothing writes while the kernel runs, through the
// scalar unit: waited for apart from the copies into LDS.
__device__ __forceinline__ int ld_scalar(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}
template <int N>
__device__ __forceinline__ void vm_wait() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All of this wave's loads and stores, in a form that the compiler counts too: behind it,
// a loop needs no waits for what was asked for before it.
__device__ __forceinline__ void vm_drain() { __builtin_amdgcn_s_waitcnt(0x0F70); }
// Workgroup barrier that leaves copies into LDS in flight: LDS reads and writes of this
// wave are complete, its global loads need not be.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// XOR key of the 16-byte pieces of a tile row of C pieces (C = 4, 8 or a multiple of
// 16). A b128 read of 16 rows is served in four groups of 16 lanes, rows 0-3 and 12-15
// at one k with rows 4-11 at the next (an odd neighbour): with these even keys the 16
// pieces of a group lie on all 64 banks, and so do four consecutive rows of a
// transposed read.
template <int C>
__device__ __forceinline__ int tile_key(int row) {
  static_assert(C == 4 || C == 8 || C % 16 == 0, "pieces of a row");
  if constexpr (C == 4) return ((row >> 2) & 1) << 1;
  if constexpr (C == 8) return ((row >> 1) & 3) << 1;
  return (row & 7) << 1;
}

__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// Sum and largest over the four lanes of a wave that share c = lane % 16: a lane swap
// with a register's own copy leaves the lower and the upper half's values side by side.
__device__ __forceinline__ float col_sum(float v) {
  const uint32_t x = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t y = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float col_max(float v) {
  const uint32_t x = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t y = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace moe
