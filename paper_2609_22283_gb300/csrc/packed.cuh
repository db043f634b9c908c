// What the four bits of a packed slot stand for (see packed.h for the layout).
#pragma once

#include <cstdint>

#include "packed.h"
#include "ptx.cuh"

namespace sva {

// The values of a word of eight codes, as four pairs of bf16; `scale` in both halves.
// A code n = code + 8 put behind the exponent of 16 is the bf16 number 16 + n, and
// code * scale = (16 + n) * scale - 24 * scale.  A scale has at most 5 significant
// bits and is below 2^122, so 24 * scale (3 * 2^3) and the result (at most 7 of 3
// bits) are bf16 numbers: the fused multiply-add rounds nothing.  Three instructions
// a pair, two for the first: inside the attention it is their number that counts (with
// words not turned, one shift more of four, 4680 queries over three packed states of 12
// heads took 418 us instead of 384).
__device__ __forceinline__ uint4 packed_values(uint32_t w, uint32_t scale) {
  uint32_t off, o[4];
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(off) : "r"(scale), "r"(0xC1C0C1C0u));  // -24
  const uint32_t at[4] = {w, w >> 4, w >> 8, __funnelshift_r(w, w, 12)};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t v = (at[j] & 0x00780078u) | 0x41804180u;  // 16 + n
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(o[j]) : "r"(v), "r"(scale), "r"(off));
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// One token's row of a packed tile in registers.  A kernel may be resident before the
// one that packs the tile has ended, so these are ordinary loads.
template <int D>
struct PackRow {
  static constexpr int G = D / kPackGroup;
  struct Scales {
    uint32_t w[G / 2];  // two scales a word
  };
  uint4 codes[G];
  Scales scales;
  __device__ __forceinline__ void load_codes(const uint8_t* tile, int row, int g) {
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(codes[g].x), "=r"(codes[g].y), "=r"(codes[g].z), "=r"(codes[g].w)
                 : "l"(tile + g * (kTile * 16) + row * 16));
  }
  __device__ __forceinline__ void load_scales(const uint8_t* tile, int row) {
    const uint8_t* at = tile + G * (kTile * 16) + row * (G * 2);
    if constexpr (G == 4)
      asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(scales.w[0]), "=r"(scales.w[1]) : "l"(at));
    else
      asm volatile("ld.global.u32 %0, [%1];" : "=r"(scales.w[0]) : "l"(at));
  }
  __device__ __forceinline__ void load_all(const uint8_t* tile, int row) {
    load_scales(tile, row);
#pragma unroll
    for (int g = 0; g < G; ++g) load_codes(tile, row, g);
  }
  // The scale of group g, in both halves.
  static __device__ __forceinline__ uint32_t scale(const Scales& s, int g) {
    return __byte_perm(s.w[g >> 1], 0, g & 1 ? 0x3232 : 0x1010);
  }
};

}  // namespace sva
