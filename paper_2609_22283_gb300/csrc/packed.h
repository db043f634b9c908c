// Packed slots: states in 4 bits, their layout, and the launch parameters of the
// kernels that fill and read them (packed.cu) and that copy states (state_copy.cu).
//
// A packed slot is [2 (K, V)][H][tiles of 128 tokens], a tile's bytes
//   codes   [d / 32][128 tokens][16]: the 32 codes of a token's group g of elements
//   scales  [128 tokens][d / 32] bf16
// so that the threads that take a tile's tokens one each read whole lines, and a
// tile is one piece of memory.  Tokens past T have scale 0.
//
// Bit order of a group: 32-bit word k holds elements 8k..8k+7; element 8k + 2j has the
// four bits from 4j on, element 8k + 2j + 1 those from 16 + 4j on, each as its code + 8
// (1..15), and the word is turned left by 3.  So a shift (none for the first pair) and a
// mask leave two neighbouring elements in the two halves of a word, behind the place of a
// bf16 number's exponent (packed_values in packed.cuh).
#pragma once

#include "internal.h"

namespace sva {

constexpr int kMaxMoves = SVA_MAX_NODES;  // states of a launch
constexpr int kPackGroup = 32;  // elements that share a scale

constexpr int pack_tile_bytes(int d) { return kTile * (d / 2 + d / kPackGroup * 2); }
template <int D>
constexpr int kPackTileBytes = pack_tile_bytes(D);

struct PackParams {
  void* pool;       // slots, bf16 [..][2][H][Tpad][d]
  uint8_t* packed;  // packed slots
  int32_t T, Tpad, H;
  int32_t n;
  int32_t pad;      // unpacking: 1: the rows past T become zeros too
  int32_t slot[kMaxMoves];    // state i: its slot
  int32_t number[kMaxMoves];  // and its packed slot, from 0
};

// Slots to packed slots, and back (d = 64 or 128).
cudaError_t launch_pack(const PackParams& p, int d, cudaStream_t s);
cudaError_t launch_unpack(const PackParams& p, int d, cudaStream_t s);

struct StateCopyParams {
  uint32_t plane;        // 32-byte vectors of a plane that are copied
  uint32_t vectors;      // of a state: all its planes'
  int64_t plane_stride;  // bytes
  int32_t n;
  const uint8_t* src[kMaxMoves];
  uint8_t* dst[kMaxMoves];
};

cudaError_t launch_state_copy(const StateCopyParams& p, cudaStream_t s);

}  // namespace sva
