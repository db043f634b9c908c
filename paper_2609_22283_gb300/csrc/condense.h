// Launch parameters of the kernels that condense states (condense.cu).
#pragma once

#include "internal.h"

namespace sva {

struct CondenseParams {
  float* weight;    // [num_slots][H][T]; the destination's part is written
  int32_t* index;   // [H][T], candidate i * T + t: token t of source i
  void* pool;       // slot pool base, bf16 [num_slots][2][H][Tpad][d]
  int32_t T, Tpad, H, d;
  int32_t n_src, dst;
  int32_t hold;     // 1: a CTA's keys stay in shared memory
  int32_t copy;     // 1: the selection copies the rows too
  int32_t slot[SVA_MAX_CTX];
};

// Sets p.hold and p.copy.
cudaError_t launch_condense(CondenseParams& p, int num_sms, cudaStream_t s);

}  // namespace sva
