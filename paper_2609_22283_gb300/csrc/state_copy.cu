// States copied between slots (sva_cache_copy): per state, planes of equally many
// bytes at one stride (the T rows of each K or V and head of a slot; a packed slot is
// one plane).  The planes' vectors are numbered through, so that a block's are
// consecutive whatever T is.
//
// Bound by HBM: every byte read and written once.  Times with sets of states in turn in
// a graph: one state of 4680 x 12 x 128 (57 MB both ways) 9.9 us (5.8 TB/s), six 50.6 (6.8),
// seven of 40 x 128 (1.38 GB) 190 (7.2); four of 2160 x 16 x 64 3.0, of 320 x 12 x 128 2.6.
// One vector a thread: 10.0, 50.4, 189.5, 3.5, 2.4; four: 9.9, 50.6, 189.8, 3.4, 2.6; eight:
// 10.0, 50.4, 189.2, 4.2, 2.6.
#include <cuda_runtime.h>

#include "packed.h"
#include "ptx.cuh"

namespace sva {
namespace {

constexpr int kCopyThreads = 256;
constexpr int kCopyBatch = 2;  // 32-byte vectors of a thread

struct Vec32 {
  uint32_t w[8];
};

__device__ __forceinline__ Vec32 ld_vec(const uint8_t* p) {
  Vec32 v;
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]),
                 "=r"(v.w[7])
               : "l"(p));
  return v;
}

__device__ __forceinline__ void st_vec(uint8_t* p, const Vec32& v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v.w[0]), "r"(v.w[1]),
               "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7])
               : "memory");
}

__global__ void __launch_bounds__(kCopyThreads) state_copy_kernel(const __grid_constant__ StateCopyParams p) {
  const uint32_t v0 = blockIdx.x * (kCopyThreads * kCopyBatch) + threadIdx.x;
  const uint8_t* src = p.src[blockIdx.y];
  uint8_t* dst = p.dst[blockIdx.y];
  int64_t off[kCopyBatch];
  Vec32 x[kCopyBatch];
  ptx::pdl_wait();
#pragma unroll
  for (int k = 0; k < kCopyBatch; ++k) {
    const uint32_t v = v0 + k * kCopyThreads;
    const uint32_t plane = v / p.plane;
    off[k] = (int64_t)plane * p.plane_stride + (int64_t)(v - plane * p.plane) * 32;
    if (v < p.vectors) x[k] = ld_vec(src + off[k]);
  }
#pragma unroll
  for (int k = 0; k < kCopyBatch; ++k)
    if (v0 + k * kCopyThreads < p.vectors) st_vec(dst + off[k], x[k]);
}

}  // namespace

cudaError_t launch_state_copy(const StateCopyParams& p, cudaStream_t s) {
  constexpr uint32_t per_block = kCopyThreads * kCopyBatch;
  LaunchConfig l(dim3((p.vectors + per_block - 1) / per_block, (unsigned)p.n), kCopyThreads, 0, s);
  return cudaLaunchKernelEx(&l.cfg, state_copy_kernel, p);
}

}  // namespace sva
