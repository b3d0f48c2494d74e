// The latent cache held in 4 bits: its pages, and how a word of codes becomes numbers.
//
// A row is the Dc latents and Dr rotated key values of a token, in groups of 64 (the last
// group is the key). A group holds a step s and a middle z (fp16), a value a code q of 0..15
// and stands for s (q - 8) + z: the middle of the range, as the base of the codes, is a small
// number, which fp16 holds more finely than the range's end. A page of P tokens, in bytes:
//   latents' codes [P][Dc / 2], keys' codes [P][Dr / 2]   (two a byte, the first in the low half)
//   s [G][P], z [G][P]   (fp16, G = Dc / 64 + 1: eight tokens' steps of a group are one load)
#pragma once

#include "moe_latent.h"
#include "moe_tile.h"

namespace moe {

constexpr int kStep4 = 64;       // context tokens of a tile of the absorbed form

// Byte offsets of a page's parts.
struct Page4 {
  int keys, steps;               // the latents' codes begin at 0
  int bytes;
};
__host__ __device__ inline Page4 page4(int Dc, int Dr, int P) {
  const int rows = P * (Dc + Dr) / 2;
  return Page4{P * Dc / 2, rows, rows + P * 4 * (Dc / 64 + 1)};
}

// The constants below, opaque to the compiler: mask and base of one v_and_or_b32 have to lie in
// registers (as literals they take two instructions).
struct CodeBits {
  uint32_t even, odd, even_base, odd_base;
};
__device__ __forceinline__ CodeBits code_bits() {
  CodeBits b{0x000F000Fu, 0x00F000F0u, 0x64006400u, 0x54005400u};
  asm("" : "+s"(b.even), "+s"(b.odd), "+v"(b.even_base), "+v"(b.odd_base));
  return b;
}
// The eight codes of a word less 8, exact halves in code order (in_code_order, 0, 4, 1, 5, 2, 6, 3, 7): a
// code in the low bits of the half 1024 is 1024 + q, four bits up in the half 64 it is 64 + q. Nine
// instructions, and four more for the values; with the bases left in, s and z would have to take them
// out again, and z - 1032 s is no half.
__device__ __forceinline__ h8 codes8(uint32_t w, const CodeBits& k) {
  const auto at = [](uint32_t v, float base) {
    const _Float16 b = (_Float16)(base + 8.f);
    return __builtin_bit_cast(h2, v) - h2{b, b};
  };
  const uint32_t u = w >> 8;
  const h2 a = at((w & k.even) | k.even_base, 1024.f), b = at((w & k.odd) | k.odd_base, 64.f);
  const h2 c = at((u & k.even) | k.even_base, 1024.f), d = at((u & k.odd) | k.odd_base, 64.f);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The values, rounded once to fp16, the type of the products (2^-11 of a value, beside a code's half step
// of 1/30 of its group's range; exact, s and z would have to be taken out of the products, group by group).
__device__ __forceinline__ h8 values8(uint32_t w, h8 s, h8 z, const CodeBits& k) {
  return __builtin_elementwise_fma(codes8(w, k), s, z);
}
__device__ __forceinline__ h8 splat8(_Float16 v) { return h8{v, v, v, v, v, v, v, v}; }

}  // namespace moe
