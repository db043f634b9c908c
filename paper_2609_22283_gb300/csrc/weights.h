// Launch parameters of the attention-weight kernel (weights.cu), apart from
// the attention and RoPE declarations in internal.h.
#pragma once

#include "internal.h"

namespace sva {

constexpr int kMaxWeightRefs = SVA_MAX_NODES * (1 + SVA_MAX_CTX);  // (node, key state) pairs of a launch
constexpr int kMaxWeightSplit = 8;  // CTAs (one cluster) that share a unit's queries
constexpr int kMaxQueryTiles = 65536 / kTile;

struct alignas(128) WeightParams {
  CUtensorMap tmap_q;   // as in AttnParams
  CUtensorMap tmap_kv;
  const float* lse;     // [n_nodes][H][T]
  const float* prev;    // [num_slots][H][T], or null
  float* out;           // [num_slots][H][T]
  int* status;
  float decay;          // of prev
  float scale_log2;     // logit scale * log2(e)
  int32_t T, Tpad, H;
  int32_t n_qt;         // query tiles of a node = key tiles of a slot
  int32_t n_pairs;      // pairs of key tiles of a slot
  int32_t units;        // (slot, head, pair of key tiles)
  int32_t n_split;      // CTAs a unit (1: the grid's CTAs take units in turn)
  int32_t frame_tokens;
  int32_t fault_mode;
  uint64_t timeout_ns;
  const uint32_t* tile_mask;  // masks as in AttnParams
  int32_t mask_words;
  const uint32_t* own_mask;
  int32_t own_words;
  const uint32_t* hist_mask;
  int32_t hist_states;
  int32_t hist_words;
  // Key tiles that the token masks leave anything of, as in AttnParams, or null
  const uint8_t* any_tile;
  int32_t any_stride;
  int32_t masked;       // some mask, or a frame-causal node
  int32_t take;     // 1: a masked launch's CTAs take units of CTAs that have not started
  // The distinct slots that the nodes see, those seen by most nodes first, and
  // for slot i the nodes that see it: refs [first[i], first[i + 1]).
  int32_t n_slots;
  int32_t slot[kMaxWeightRefs];
  uint16_t first[kMaxWeightRefs + 1];
  uint16_t ref[kMaxWeightRefs];
};

// A ref: the node, its key state that the slot is (0 own, 1 + j its ctx_slot[j])
// and whether the own chunk is frame-causal.
constexpr int kRefStateShift = 6, kRefCausal = 1 << 11;
static_assert(SVA_MAX_NODES <= 64 && SVA_MAX_CTX < 31, "ref fields");

cudaError_t launch_weights(const WeightParams& p, int head_dim, int grid, cudaStream_t s);

}  // namespace sva
