// Eviction by accumulated attention weight (sva_cache_condense): of the n * T
// tokens of n states, each head keeps the T whose weight is largest, in their
// order, as one state.
//
// Two launches.  condense_select_kernel finds which: a cluster of up to eight
// CTAs per head, each with a contiguous range of the head's candidates in shared
// memory as ordered integer keys, finds the T-th largest key digit by digit (11,
// 11 and 10 bits: a histogram of the candidates that match the digits so far,
// summed over the cluster through distributed shared memory, each CTA picking
// the digit for itself), then ranks what is kept: everything above that key, and
// of those equal to it the first ones in candidate order.  Counts and ranks are
// integers, so the result does not depend on the order of the atomics.
// condense_gather_kernel then copies the kept rows of K and V: bound by HBM.
#include <mutex>

#include <cuda_runtime.h>

#include "condense.h"
#include "ptx.cuh"

namespace sva {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;
// Keys that a CTA holds in shared memory; a longer range is read again for each
// digit.
constexpr int kHeldKeys = 48 * 1024;

// Weights as integers of the same order; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float w) {
  if (w != w) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
  return v;
}

// Exclusive sum over the block of a pair of counts, in thread order; `all` is the
// sum of all.  Every thread calls it.
__device__ __forceinline__ uint2 block_scan(uint2 v, uint2* warp_sum, uint2* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint2 s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, s.x, o), b = __shfl_up_sync(0xffffffffu, s.y, o);
    if (lane >= o) {
      s.x += a;
      s.y += b;
    }
  }
  if (lane == 31) warp_sum[warp] = s;
  __syncthreads();
  uint2 w = warp_sum[lane];  // 32 warps: every warp sums all of them
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, w.x, o), b = __shfl_up_sync(0xffffffffu, w.y, o);
    if (lane >= o) {
      w.x += a;
      w.y += b;
    }
  }
  all->x = __shfl_sync(0xffffffffu, w.x, 31);
  all->y = __shfl_sync(0xffffffffu, w.y, 31);
  const uint32_t bx = __shfl_sync(0xffffffffu, w.x, warp > 0 ? warp - 1 : 0);
  const uint32_t by = __shfl_sync(0xffffffffu, w.y, warp > 0 ? warp - 1 : 0);
  __syncthreads();  // warp_sum may be written again
  return make_uint2(s.x - v.x + (warp > 0 ? bx : 0u), s.y - v.y + (warp > 0 ? by : 0u));
}

__global__ void __launch_bounds__(kSelThreads, 1) condense_select_kernel(const __grid_constant__ CondenseParams p) {
  extern __shared__ uint32_t held[];
  __shared__ uint32_t hist[2][kBins];  // of two digits in turn
  __shared__ uint2 warp_sum[32];
  __shared__ uint32_t digit_sh, above_sh;
  __shared__ uint2 count_sh;           // this CTA's candidates above the line and on it
  const int tid = threadIdx.x;
  const int nc = p.cluster;
  const int h = (int)blockIdx.x / nc, rank = (int)blockIdx.x - h * nc;
  const int n = p.n_src * p.T;
  const int per = (n + nc - 1) / nc;
  const int e0 = min(rank * per, n), count = min(per, n - e0);
  const bool hold = p.hold != 0;

  ptx::pdl_launch_dependents();
  for (int b = tid; b < kBins; b += kSelThreads) hist[0][b] = 0;
  ptx::pdl_wait();
  auto load = [&](int e) {  // candidate e of the head
    const int i = e / p.T;
    return p.weight + ((size_t)p.slot[i] * p.H + h) * p.T + (e - i * p.T);
  };
  auto key_at = [&](int j) { return hold ? held[j] : key_of(*load(e0 + j)); };
  __syncthreads();

  uint32_t prefix = 0;   // the digits found so far
  int need = p.T;        // of the candidates that match them, the ones to keep
  int shift = 32;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass < 2 ? 11 : 10;
    const uint32_t mask = pass == 0 ? 0u : ~0u << shift;
    shift -= bits;
    uint32_t* hs = hist[pass & 1];
    for (int j = tid; j < count; j += kSelThreads) {
      uint32_t k;
      if (pass == 0) {
        k = key_of(*load(e0 + j));
        if (hold) held[j] = k;
      } else {
        k = key_at(j);
      }
      if (((k ^ prefix) & mask) == 0u) atomicAdd(&hs[(k >> shift) & ((1u << bits) - 1u)], 1u);
    }
    __syncthreads();
    if (nc > 1) ptx::cluster_sync();
    // two bins a thread, the largest digits first
    uint2 mine = make_uint2(0u, 0u);
    const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
    if (nc > 1) {
      for (int c = 0; c < nc; ++c) {
        mine.x += ld_cluster_u32(ptx::mapa_shared(ptx::smem_u32(&hs[b1]), c));
        mine.y += ld_cluster_u32(ptx::mapa_shared(ptx::smem_u32(&hs[b0]), c));
      }
    } else {
      mine = make_uint2(hs[b1], hs[b0]);
    }
    // the other histogram was last read before this pass's cluster barrier
    for (int b = tid; b < kBins; b += kSelThreads) hist[(pass + 1) & 1][b] = 0;
    uint2 all;
    const uint32_t before = block_scan(make_uint2(mine.x + mine.y, 0u), warp_sum, &all).x;
    if (before < (uint32_t)need && before + mine.x + mine.y >= (uint32_t)need) {
      const bool first = before + mine.x >= (uint32_t)need;
      digit_sh = (uint32_t)(first ? b1 : b0);
      above_sh = before + (first ? 0u : mine.x);
    }
    __syncthreads();
    prefix |= digit_sh << shift;
    need -= (int)above_sh;
  }

  // `need` (>= 1) of the candidates equal to `prefix` stay, and all above it.  A
  // thread takes consecutive candidates, an odd number of them (no two lanes of a
  // warp on one bank).
  const int run = ((count + kSelThreads - 1) / kSelThreads) | 1;
  const int j0 = min(tid * run, count), j1 = min(j0 + run, count);
  uint2 my = make_uint2(0u, 0u);
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key_at(j);
    my.x += k > prefix;
    my.y += k == prefix;
  }
  uint2 all;
  uint2 at = block_scan(my, warp_sum, &all);
  int kept = 0, level = 0;  // kept and equal candidates of the CTAs before this one
  if (nc > 1) {
    if (tid == 0) count_sh = all;
    ptx::cluster_sync();
    for (int c = 0; c < rank; ++c) {
      const uint32_t a = ptx::mapa_shared(ptx::smem_u32(&count_sh), c);
      kept += (int)ld_cluster_u32(a);
      level += (int)ld_cluster_u32(a + 4);
    }
    kept += min(level, need);
  }
  int eq = level + (int)at.y;                               // equal ones before this thread's
  int out = kept + (int)at.x + min(eq, need) - min(level, need);
  int32_t* index = p.index + (size_t)h * p.T;
  float* weight = p.weight + ((size_t)p.dst * p.H + h) * p.T;
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key_at(j);
    const bool same = k == prefix;
    if (k > prefix || (same && eq < need)) {
      index[out] = e0 + j;
      weight[out] = *load(e0 + j);
      ++out;
    }
    eq += same;
  }
  // no CTA leaves while another may still read its counts
  if (nc > 1) ptx::cluster_sync();
}

// K and V rows of the kept candidates, kRows rows a thread group in flight.
constexpr int kRows = 4;
__global__ void __launch_bounds__(256) condense_gather_kernel(const __grid_constant__ CondenseParams p) {
  const int vpr = p.d >> 3;  // 16-byte vectors of a row
  const int groups = 256 / vpr;
  const int g = threadIdx.x / vpr, c8 = threadIdx.x - g * vpr;
  const int h = blockIdx.y;
  const int row0 = blockIdx.x * groups * kRows + g;
  const size_t kv = (size_t)p.H * p.Tpad * p.d;  // elements between K and V of a slot
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  uint4 k[kRows], v[kRows];
  int32_t e[kRows];
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int row = row0 + j * groups;
    e[j] = row < p.T ? p.index[(size_t)h * p.T + row] : -1;
  }
  auto at = [&](int slot, int row) {
    return static_cast<uint16_t*>(p.pool) + (((size_t)slot * 2 * p.H + h) * p.Tpad + row) * p.d + c8 * 8;
  };
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    if (e[j] < 0) continue;
    const int i = e[j] / p.T;
    const uint16_t* src = at(p.slot[i], e[j] - i * p.T);
    k[j] = *reinterpret_cast<const uint4*>(src);
    v[j] = *reinterpret_cast<const uint4*>(src + kv);
  }
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    if (e[j] < 0) continue;
    uint16_t* dst = at(p.dst, row0 + j * groups);
    *reinterpret_cast<uint4*>(dst) = k[j];
    *reinterpret_cast<uint4*>(dst + kv) = v[j];
  }
}

}  // namespace

cudaError_t launch_condense(CondenseParams& p, cudaStream_t s) {
  static std::mutex mu;
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!configured[dev]) {
      e = cudaFuncSetAttribute(condense_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               kHeldKeys * 4);
      if (e != cudaSuccess) return e;
      configured[dev] = true;
    }
  }
  const int n = p.n_src * p.T;
  p.cluster = n <= 4096 ? 1 : (n <= 8192 ? 2 : (n <= 16384 ? 4 : 8));
  const int per = (n + p.cluster - 1) / p.cluster;
  p.hold = per <= kHeldKeys ? 1 : 0;
  LaunchConfig sel(dim3((unsigned)(p.H * p.cluster)), kSelThreads, p.hold ? (size_t)per * 4 : 0, s,
                   p.cluster > 1 ? p.cluster : 0);
  e = cudaLaunchKernelEx(&sel.cfg, condense_select_kernel, p);
  if (e != cudaSuccess) return e;
  const int rows = 256 / (p.d >> 3) * kRows;
  LaunchConfig copy(dim3((unsigned)((p.T + rows - 1) / rows), (unsigned)p.H), 256, 0, s);
  return cudaLaunchKernelEx(&copy.cfg, condense_gather_kernel, p);
}

}  // namespace sva
