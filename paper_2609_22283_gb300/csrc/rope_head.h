// Launch parameters of the per-head norm + RoPE + cache write (rope_head.cu).
#pragma once

#include "internal.h"

namespace sva {

struct RopeHeadParams {
  const void* k;  // bf16, token t (of all nodes') at t * k_stride elements, [H][d] each
  const void* v;
  const void* q;  // may be null
  void* q_out;    // bf16 [n_nodes][T][H][d], or null
  int64_t k_stride, v_stride, q_stride;
  void* cache;    // slot pool base, as in RopeParams
  const float2* tab_t;  // rotation tables, as in RopeParams
  const float2* tab_h;
  const float2* tab_w;
  const float* gamma_k;  // null: ones
  const float* gamma_q;
  int32_t gamma_heads;   // 1: one [d] vector for every head; else [H][d]
  float eps;
  int32_t T, H, d, Tpad, Hp, Wp, P0, P1, P2;
  int32_t n_nodes;
  int32_t group;  // lanes that share a token's part: 8, 16 or 32, a multiple of d / 8
  int32_t parts;  // parts of a token
  RopeNode nodes[SVA_MAX_NODES];
};

// Sets p.group and p.parts.
cudaError_t launch_rope_head(RopeHeadParams& p, int num_sms, cudaStream_t s);

}  // namespace sva
