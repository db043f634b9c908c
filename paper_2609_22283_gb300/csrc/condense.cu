// Eviction by accumulated attention weight (sva_cache_condense): of the n * T
// tokens of n states, each head keeps the T whose weight is largest, in their
// order, as one state.
//
// Two launches, one for the smallest states.  condense_select_kernel finds which: a
// cluster of up to eight CTAs per head, each with a contiguous range of the head's candidates in shared
// memory, finds the T-th largest key (the weights as integers of the same order)
// digit by digit, 11, 11 and 10 bits.  The first digit's histogram has few bins in
// use; each CTA adds its own to every CTA's sums through distributed shared
// memory, and each finds the digit for itself.  The candidates with that digit are
// then few and gathered by every CTA, which finds the other digits alone (a cluster
// barrier costs 0.7 us, reading eight histograms of 2048 bins 1.5 to 2 us); or all
// equal (tokens that nothing attended); or the other digits are found like the
// first, each CTA reading all histograms.  Then what stays is ranked: everything
// above the key, and of the candidates equal to it the first ones.  Counts and ranks
// are integers, so the result does not depend on the order of the atomics.  What
// bounds it is the chain of these steps: 28080 candidates in eight CTAs take 10.5 us,
// of which the loads 2.0, three cluster barriers 2.4, what passes between the CTAs
// 2.5, four scans of a block 2.0.  With each digit's eight histograms read by every
// CTA it was 15.6 us.
// condense_gather_kernel then copies the kept rows of K and V: bound by HBM (57 MB
// of the 23.5 us of 28080 candidates of 12 heads, 192 MB of the 46.1 us of 32760 of 40).
#include <algorithm>
#include <mutex>

#include <cuda_runtime.h>

#include "condense.h"
#include "ptx.cuh"

namespace sva {
namespace {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kBins = 2048;
constexpr int kBinsPerThread = kBins / kSelThreads;
static_assert(kBinsPerThread == 4, "a thread takes a vector of bins");
// Weights that a CTA holds in shared memory; a longer range is read again for each
// digit.
constexpr int kHeldKeys = 40 * 1024;
// Candidates that share the first digit with the line, up to this many in all
// CTAs, are gathered by every CTA of the cluster.
constexpr int kListKeys = 4096;

// Weights (their bits) as integers of the same order; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(uint32_t bits) {
  float w = __uint_as_float(bits);
  if (w != w) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint4 ld_cluster_v4(uint32_t cluster_addr) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(cluster_addr));
  return v;
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr));
  return v;
}

__device__ __forceinline__ void add_cluster_u32(uint32_t cluster_addr, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}

// The halves of a cluster barrier.
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Exclusive sum over the block, in thread order; `all`: the sum of all.  Every
// thread calls it.
template <typename Sum>
__device__ __forceinline__ Sum block_scan(Sum v, Sum* warp_sum, Sum* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sum s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sum a = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += a;
  }
  if (lane == 31) warp_sum[warp] = s;
  __syncthreads();
  Sum w = lane < kSelWarps ? warp_sum[lane] : 0;  // every warp sums all of them
#pragma unroll
  for (int o = 1; o < kSelWarps; o <<= 1) {
    const Sum a = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += a;
  }
  *all = __shfl_sync(0xffffffffu, w, kSelWarps - 1);
  const Sum before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return s - v + (warp > 0 ? before : 0);
}

// The digit of a histogram (four bins a thread in `bins`, thread 0 the largest)
// at which the count from the top reaches `need`.
struct Digit {
  uint32_t digit, above, here;  // candidates above the digit, and with it
};
__device__ __forceinline__ Digit find_digit(uint4 bins, int need, uint32_t* warp_sum, Digit* found) {
  uint32_t all;
  const uint32_t total = bins.x + bins.y + bins.z + bins.w;
  uint32_t at = block_scan(total, warp_sum, &all);
  const uint32_t line = (uint32_t)need;
  if (at < line && at + total >= line) {
    uint32_t digit = (uint32_t)(kBins - 1 - 4 * threadIdx.x), here = bins.w;
    if (at + here < line) {
      at += here;
      --digit;
      here = bins.z;
      if (at + here < line) {
        at += here;
        --digit;
        here = bins.y;
        if (at + here < line) {
          at += here;
          --digit;
          here = bins.x;
        }
      }
    }
    *found = {digit, at, here};
  }
  __syncthreads();
  return *found;
}

// Vector c8 of K and of V of head h's kept candidate `row`.
__device__ __forceinline__ void copy_vector(const CondenseParams& p, int h, int row, int c8) {
  const size_t kv = (size_t)p.H * p.Tpad * p.d;  // elements between K and V of a slot
  const int32_t e = p.index[(size_t)h * p.T + row];
  const int i = e / p.T;
  auto at = [&](int slot, int r) {
    return static_cast<uint16_t*>(p.pool) + (((size_t)slot * 2 * p.H + h) * p.Tpad + r) * p.d + c8 * 8;
  };
  const uint16_t* src = at(p.slot[i], e - i * p.T);
  const uint4 k = *reinterpret_cast<const uint4*>(src);
  const uint4 v = *reinterpret_cast<const uint4*>(src + kv);
  uint16_t* dst = at(p.dst, row);
  *reinterpret_cast<uint4*>(dst) = k;
  *reinterpret_cast<uint4*>(dst + kv) = v;
}

// kCluster CTAs a head.
template <int kCluster>
__global__ void __launch_bounds__(kSelThreads, 2) condense_select_kernel(const __grid_constant__ CondenseParams p) {
  extern __shared__ uint32_t held[];               // the range's weights, then this CTA's list
  __shared__ alignas(16) uint32_t hist[2][kBins];  // of this CTA's candidates
  __shared__ alignas(16) uint32_t sums[kBins];     // the first digit's, of the cluster
  __shared__ uint32_t list[kListKeys];             // the cluster's candidates with the first digit
  __shared__ uint32_t warp_sum[5][kSelWarps];      // of each digit
  __shared__ uint64_t warp_count[kSelWarps];
  __shared__ Digit found[5];
  __shared__ alignas(16) uint32_t match_sh[4];     // this CTA's candidates with the first digit: how many, least, largest
  __shared__ alignas(16) uint32_t count_sh[4];     // this CTA's candidates above the line and on it
  const int tid = threadIdx.x, lane = tid & 31;
  const int h = (int)blockIdx.x / kCluster, rank = (int)blockIdx.x - h * kCluster;
  const int n = p.n_src * p.T;
  const int per = (n + kCluster - 1) / kCluster;
  const int e0 = min(rank * per, n), count = min(per, n - e0);
  const bool hold = p.hold != 0;
  uint32_t* mine = held + (hold ? per : 0);
  const int b0 = kBins - 4 - 4 * tid;              // this thread's bins
  const uint4 zero = make_uint4(0, 0, 0, 0);

  ptx::pdl_launch_dependents();
  *reinterpret_cast<uint4*>(&hist[0][tid * 4]) = zero;
  *reinterpret_cast<uint4*>(&hist[1][tid * 4]) = zero;
  *reinterpret_cast<uint4*>(&sums[tid * 4]) = zero;
  if (tid == 0) {
    match_sh[0] = 0;
    match_sh[1] = ~0u;
    match_sh[2] = 0;
  }
  __syncwarp();
  if constexpr (kCluster > 1) cluster_arrive();    // the sums are clear
  ptx::pdl_wait();
  const uint32_t* weight = reinterpret_cast<const uint32_t*>(p.weight);
  const uint32_t inv_t = 0xFFFFFFFFu / (uint32_t)p.T;
  auto load = [&](int e) {  // candidate e of the head
    int i = (int)__umulhi((uint32_t)e, inv_t);  // e / T or one less: e < 2^20
    if ((i + 1) * p.T <= e) ++i;
    return weight[((size_t)p.slot[i] * p.H + h) * p.T + (e - i * p.T)];
  };
  auto bits_at = [&](int j) { return hold ? held[j] : load(e0 + j); };
  __syncthreads();

  // First digit: the few bins in use are added to every CTA's sums.
#pragma unroll 8
  for (int j = tid; j < count; j += kSelThreads) {
    const uint32_t w = load(e0 + j);
    if (hold) held[j] = w;
    atomicAdd(&hist[0][key_of(w) >> 21], 1u);
  }
  __syncthreads();
  if constexpr (kCluster > 1) {
    cluster_wait();
#pragma unroll
    for (int k = 0; k < kBinsPerThread; ++k) {
      const int b = tid + k * kSelThreads;
      const uint32_t v = hist[0][b];
      if (v != 0)
#pragma unroll
        for (int c = 0; c < kCluster; ++c) add_cluster_u32(ptx::mapa_shared(ptx::smem_u32(&sums[b]), (uint32_t)c), v);
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  }
  const uint32_t* first = kCluster > 1 ? sums : hist[0];
  Digit d = find_digit(*reinterpret_cast<const uint4*>(&first[b0]), p.T, warp_sum[0], &found[0]);
  uint32_t prefix = d.digit << 21;   // the digits found so far
  int need = p.T - (int)d.above;     // of the candidates that match them, the ones to keep
  const bool listed = d.here <= (uint32_t)kListKeys;

  // The candidates that match: their keys where they are few, their range.
  uint32_t least = ~0u, most = 0;
  constexpr int kBlock = 8;  // candidates a thread in one step: one count a warp and step
  for (int base = 0; base < count; base += kBlock * kSelThreads) {
    uint32_t key[kBlock], bits = 0;
#pragma unroll
    for (int u = 0; u < kBlock; ++u) {
      const int j = base + u * kSelThreads + tid;
      key[u] = j < count ? key_of(bits_at(j)) : ~prefix;
      if (((key[u] ^ prefix) >> 21) == 0u) {
        bits |= 1u << u;
        least = min(least, key[u]);
        most = max(most, key[u]);
      }
    }
    if (!listed || !__any_sync(0xffffffffu, bits != 0u)) continue;
    uint32_t at = (uint32_t)__popc(bits);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, at, o);
      if (lane >= o) at += x;
    }
    uint32_t first_at = 0;
    if (lane == 31) first_at = atomicAdd(&match_sh[0], at);
    at += __shfl_sync(0xffffffffu, first_at, 31) - (uint32_t)__popc(bits);
#pragma unroll
    for (int u = 0; u < kBlock; ++u)
      if (bits >> u & 1u) mine[at++] = key[u];
  }
  least = __reduce_min_sync(0xffffffffu, least);
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0 && least <= most) {
    atomicMin(&match_sh[1], least);
    atomicMax(&match_sh[2], most);
  }
  uint4 match[kCluster];
  if constexpr (kCluster > 1) {
    __syncwarp();
    cluster_arrive();
    cluster_wait();
#pragma unroll
    for (int c = 0; c < kCluster; ++c)
      match[c] = ld_cluster_v4(ptx::mapa_shared(ptx::smem_u32(match_sh), (uint32_t)c));
  } else {
    __syncthreads();
    match[0] = *reinterpret_cast<const uint4*>(match_sh);
  }
  least = ~0u;
  most = 0;
#pragma unroll
  for (int c = 0; c < kCluster; ++c) {
    least = min(least, match[c].y);
    most = max(most, match[c].z);
  }
  if (least == most) {  // all of them equal (tokens that nothing attended)
    prefix = least;
  } else if (listed) {
    // Every CTA gathers the cluster's and finds the other digits for itself.
    const uint32_t* keys = mine;
    if constexpr (kCluster > 1) {
#pragma unroll 4
      for (uint32_t j = tid; j < d.here; j += kSelThreads) {
        uint32_t c = 0, at = j;  // its CTA, its place there
#pragma unroll
        for (int k = 0; k < kCluster - 1; ++k)
          if (c == (uint32_t)k && at >= match[k].x) {
            at -= match[k].x;
            ++c;
          }
        list[j] = ld_cluster_u32(ptx::mapa_shared(ptx::smem_u32(mine + at), c));
      }
      keys = list;
      __syncthreads();
    }
    const uint32_t m = d.here;
    *reinterpret_cast<uint4*>(&hist[0][tid * 4]) = zero;
    for (uint32_t j = tid; j < m; j += kSelThreads) atomicAdd(&hist[1][(keys[j] >> 10) & 2047u], 1u);
    __syncthreads();
    d = find_digit(*reinterpret_cast<const uint4*>(&hist[1][b0]), need, warp_sum[1], &found[1]);
    prefix |= d.digit << 10;
    need -= (int)d.above;
    for (uint32_t j = tid; j < m; j += kSelThreads) {
      const uint32_t k = keys[j];
      if (((k ^ prefix) >> 10) == 0u) atomicAdd(&hist[0][k & 1023u], 1u);
    }
    __syncthreads();
    d = find_digit(*reinterpret_cast<const uint4*>(&hist[0][b0]), need, warp_sum[2], &found[2]);
    prefix |= d.digit;
    need -= (int)d.above;
  } else {
    // The cluster's histogram of each digit, by every CTA.
    *reinterpret_cast<uint4*>(&hist[0][tid * 4]) = zero;
#pragma unroll 1
    for (int pass = 1; pass < 3; ++pass) {
      const int shift = pass == 1 ? 10 : 0;
      uint32_t* hs = hist[pass & 1];
      for (int j = tid; j < count; j += kSelThreads) {
        const uint32_t k = key_of(bits_at(j));
        if (((k ^ prefix) >> (pass == 1 ? 21 : 10)) == 0u) atomicAdd(&hs[(k >> shift) & (pass == 1 ? 2047u : 1023u)], 1u);
      }
      uint4 bins = zero;
      if constexpr (kCluster > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        uint4 part[kCluster];
#pragma unroll
        for (int c = 0; c < kCluster; ++c)
          part[c] = ld_cluster_v4(ptx::mapa_shared(ptx::smem_u32(&hs[b0]), (uint32_t)c));
#pragma unroll
        for (int c = 0; c < kCluster; ++c) {
          bins.x += part[c].x;
          bins.y += part[c].y;
          bins.z += part[c].z;
          bins.w += part[c].w;
        }
      } else {
        __syncthreads();
        bins = *reinterpret_cast<const uint4*>(&hs[b0]);
      }
      d = find_digit(bins, need, warp_sum[2 + pass], &found[2 + pass]);
      prefix |= d.digit << shift;
      need -= (int)d.above;
    }
  }

  // `need` (>= 1) of the candidates equal to `prefix` stay, and all above it.  A
  // thread takes consecutive candidates, an odd number of them (no two lanes of a
  // warp on one bank).
  const int run = ((count + kSelThreads - 1) / kSelThreads) | 1;
  const int j0 = min(tid * run, count), j1 = min(j0 + run, count);
  uint32_t above = 0, equal = 0;
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key_of(bits_at(j));
    above += k > prefix;
    equal += k == prefix;
  }
  uint64_t all;
  const uint64_t at = block_scan((uint64_t)above << 32 | equal, warp_count, &all);
  int kept = 0, level = 0;  // kept and equal candidates of the CTAs before this one
  if constexpr (kCluster > 1) {
    if (tid == 0) {
      count_sh[0] = (uint32_t)(all >> 32);
      count_sh[1] = (uint32_t)all;
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    uint4 part[kCluster];
#pragma unroll
    for (int c = 0; c < kCluster; ++c) part[c] = ld_cluster_v4(ptx::mapa_shared(ptx::smem_u32(count_sh), (uint32_t)c));
#pragma unroll
    for (int c = 0; c < kCluster; ++c) {
      kept += c < rank ? (int)part[c].x : 0;
      level += c < rank ? (int)part[c].y : 0;
    }
    __syncwarp();
    cluster_arrive();  // no CTA leaves while another may still read its counts
    kept += min(level, need);
  }
  int eq = level + (int)(uint32_t)at;                       // equal ones before this thread's
  int out = kept + (int)(at >> 32) + min(eq, need) - min(level, need);
  int32_t* index = p.index + (size_t)h * p.T;
  uint32_t* kept_weight = reinterpret_cast<uint32_t*>(p.weight) + ((size_t)p.dst * p.H + h) * p.T;
  for (int j = j0; j < j1; ++j) {
    const uint32_t w = bits_at(j), k = key_of(w);
    const bool same = k == prefix;
    if (k > prefix || (same && eq < need)) {
      index[out] = e0 + j;
      kept_weight[out] = w;
      ++out;
    }
    eq += same;
  }
  if constexpr (kCluster > 1) {
    __syncwarp();
    cluster_wait();
  } else if (p.copy) {
    __syncthreads();
    const int vpr = p.d >> 3;
    for (int v = tid; v < p.T * vpr; v += kSelThreads) copy_vector(p, h, v / vpr, v & (vpr - 1));
  }
}

// K and V rows of the kept candidates, a vector of each a thread: more blocks spread the
// misses better than several rows a thread in flight (with rows in HBM the whole call on
// 28080 candidates of 12 heads of 128 takes 23.5 us, with two, three or four rows a thread
// 26.0 to 26.3; 32760 candidates of 40 heads 46.1 either way).  K and V in blocks of their
// own take 26.9 and 52.2 us.  The next kernel is let in only as blocks end: with its blocks
// resident earlier, calls in a row take 25.6 us instead of 23.5, in L2 19.6 instead of 17.0
// (40 heads: 45.6 instead of 46.1).
constexpr int kCopyThreads = 128;
__global__ void __launch_bounds__(kCopyThreads) condense_gather_kernel(const __grid_constant__ CondenseParams p) {
  const int vpr = p.d >> 3;  // 16-byte vectors of a row
  const int row = blockIdx.x * (kCopyThreads / vpr) + threadIdx.x / vpr;
  ptx::pdl_wait();
  if (row < p.T) copy_vector(p, blockIdx.y, row, threadIdx.x & (vpr - 1));
}

}  // namespace

cudaError_t launch_condense(CondenseParams& p, int num_sms, cudaStream_t s) {
  using Kernel = void (*)(const CondenseParams);
  static const Kernel select[4] = {condense_select_kernel<1>, condense_select_kernel<2>, condense_select_kernel<4>,
                                   condense_select_kernel<8>};
  static std::mutex mu;
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!configured[dev]) {
      for (Kernel k : select) {
        e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (kHeldKeys + kListKeys) * 4);
        if (e != cudaSuccess) return e;
      }
      configured[dev] = true;
    }
  }
  const int n = p.n_src * p.T;
  // About 2048 candidates a CTA, at most eight CTAs a head, and no more of them than two
  // an SM.  (A CTA with more than about 14000 candidates has an SM to itself: where there
  // are more such CTAs than SMs, the last ones run after others.)
  int log2_cluster = 0;
  while (log2_cluster < 3 && n > 2048 << log2_cluster && (long long)p.H << (log2_cluster + 1) <= 2ll * num_sms)
    ++log2_cluster;
  const int per = (n + (1 << log2_cluster) - 1) >> log2_cluster;
  p.hold = per <= kHeldKeys ? 1 : 0;
  LaunchConfig sel(dim3((unsigned)(p.H << log2_cluster)), kSelThreads, (size_t)((p.hold ? per : 0) + std::min(per, kListKeys)) * 4, s,
                   log2_cluster > 0 ? 1 << log2_cluster : 0);
  // Up to two vectors a thread are copied where they are selected: 64 tokens of 12 heads
  // of 128 from four states take 5.8 us a call then, 6.7 with a second launch (in a graph
  // 5.6 and 5.2; one token of two states 4.8 and 6.5, 3.9 and 4.7), 128 tokens 6.9 and 6.6.
  p.copy = log2_cluster == 0 && p.T * (p.d >> 3) <= 2 * kSelThreads ? 1 : 0;
  e = cudaLaunchKernelEx(&sel.cfg, select[log2_cluster], p);
  if (p.copy || e != cudaSuccess) return e;
  const int rows = kCopyThreads / (p.d >> 3);
  LaunchConfig copy(dim3((unsigned)((p.T + rows - 1) / rows), (unsigned)p.H), kCopyThreads, 0, s);
  return cudaLaunchKernelEx(&copy.cfg, condense_gather_kernel, p);
}

}  // namespace sva
