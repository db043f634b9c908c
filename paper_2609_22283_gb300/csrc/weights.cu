// How much attention every cached key got from a launch's queries
// (sva_attend_weights): for a slot s, head h and key v
//   w[s][h][v] = decay * prev + sum_i sum_u exp(scale * q_iu . k_v + M(u, v) - lse_iu)
// over the nodes i that see s and their queries u, the log-sum-exps lse being
// the attention's.  With them known no running maximum is needed and no V: one
// product and one exponential a (query, key) pair, and sums over queries.
//
// So the product is taken the other way round, S^T = K Q^T: a key is a TMEM
// lane, its thread holds 32 or 64 of its scores at a time and adds their
// exponentials up in registers.  No score, weight or sum crosses threads; a
// unit's sum over all its queries stays in one register and nothing is added
// atomically, so results do not depend on the order of CTAs.
//
// One unit is (slot, head, pair of 128-key tiles).  K (the A operand) is copied
// to TMEM once a unit, as packed bf16, so that the MMAs read only Q from shared
// memory (with both operands there M = N = 128 needs all of its 128 B a cycle);
// Q tiles of 128 queries stream past it, for every node that sees the slot.
//   warp 0     TMA producer: a unit's K tiles, then its Q tiles (4 stages);
//   warp 2     -lse * log2(e) of a Q tile's rows (-inf past the last row) into
//              the stage; with masks also the tile's visibility words;
//   warps 1, 3 MMA issuers of key tiles 0 and 1;
//   warps 4-11 sums: warps 4-7 key tile 0, warps 8-11 key tile 1, a thread a key.
// TMEM: K0, K1 (d / 2 columns each), then three S buffers of 128 columns that the
// steps (Q tile i, key tile kt) take in turn, n = 2 i + kt in buffer n % 3: the
// two groups work in opposite phase and each S is issued while the group before
// still works.  S barriers are per group, so that their one waiter waits for
// every phase; the buffer of step n was the other group's at step n - 3.
// A CTA takes units in turn, and the pipeline runs through their ends: the next
// unit's K waits in shared memory, and a group copies it to TMEM when the last S
// of the unit is complete, ahead of the sums over that S.
//
// Launches with fewer units than SMs split a unit's Q tiles over a cluster; the
// partial sums go to the first CTA's shared memory and are added in rank order.
// Launches with masks (or frame causality) take one unit a CTA: a bitmap of the
// (node, Q tile) pairs that have any visible tile is built first, and only those
// are loaded and multiplied.
// All waits are bounded as in the attention kernel; a unit whose CTA gave up one
// is not written.
#include <mutex>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"
#include "weights.h"

namespace sva {
namespace {

using namespace ptx;

constexpr int kThreads = 384;
constexpr int kStages = 4;  // Q tiles in flight
constexpr int kGroupWarps = 4;

template <int D>
struct Cfg {
  static constexpr int kBoxBytes = kTile * 64 * 2;  // one 128-row x 64-column bf16 box
  static constexpr int kBoxes = D / 64;
  static constexpr int kTileBytes = kBoxBytes * kBoxes;
  static constexpr int kOffK = kStages * kTileBytes;
  static constexpr int kSmemBytes = kOffK + 2 * kTileBytes + 1024;  // + alignment slack
  static constexpr uint32_t kKCols = D / 2;          // TMEM columns of a K tile
  static constexpr uint32_t kColS = 128;             // first S buffer
};

struct Bars {
  uint64_t q_full[kStages];   // the Q tile has landed
  uint64_t l_full[kStages];   // its log-sum-exps (and mask words) are there
  uint64_t q_empty[kStages];  // both groups are done with the stage
  uint64_t k_full, k_empty;   // K tiles of a unit in shared memory
  uint64_t k_ready[2];        // K tile in TMEM
  uint64_t s_full[2][3], s_empty[2][3];
  uint64_t drain;
};

// Four MMAs over 64 elements of K, A from TMEM, B K-major in shared memory;
// the first accumulates where `accumulate` says.
__device__ __forceinline__ void mma_ts_kmajor_x4(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc,
                                                 uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      " .reg .pred p, t, e;\n"
      " setp.ne.b32 p, %10, 0;\n"
      " setp.eq.b32 t, 0, 0;\n"
      " elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %5, %9, p;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], %6, %9, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%3], %7, %9, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%4], %8, %9, t;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "r"(a_tmem + 8), "r"(a_tmem + 16), "r"(a_tmem + 24), "l"(b_desc), "l"(b_desc + 2),
      "l"(b_desc + 4), "l"(b_desc + 6), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, uint64_t* bar, int32_t c0,
                                            int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1)
      : "memory");
}

// Caller data, by ordinary loads (see ptx.cuh).
__device__ __forceinline__ float ld_f32_if(const float* p, bool load, float other) {
  return __uint_as_float(
      ld_global_u32_if(reinterpret_cast<const uint32_t*>(p), load, __float_as_uint(other)));
}

// The Q tiles of a unit in order: every (ref, query tile), or the marked ones of
// a bitmap over ref * n_qt + tile.
template <bool kMask>
struct Walk {
  const uint32_t* marks;
  int at, end, n_qt, r, qt;
  uint32_t left;
  __device__ __forceinline__ Walk(const uint32_t* marks_, int begin, int end_, int n_qt_)
      : marks(marks_), at(begin), end(end_), n_qt(n_qt_), r(begin / n_qt_), qt(begin - r * n_qt_), left(0) {
    if constexpr (kMask) {
      left = begin < end ? marks[begin >> 5] & (~0u << (begin & 31)) : 0u;
      at = begin >> 5;
    }
  }
  // The next item into (r, qt); false past the last.
  __device__ __forceinline__ bool next(int& r_out, int& qt_out) {
    if constexpr (kMask) {
      const int words = (end + 31) >> 5;
      while (left == 0u) {
        if (++at >= words) return false;
        left = marks[at];
      }
      const int i = (at << 5) + __ffs(left) - 1;
      left &= left - 1u;
      if (i >= end) return false;
      r_out = i / n_qt;
      qt_out = i - r_out * n_qt;
      return true;
    } else {
      if (at >= end) return false;
      r_out = r;
      qt_out = qt;
      ++at;
      if (++qt == n_qt) {
        qt = 0;
        ++r;
      }
      return true;
    }
  }
};

struct Unit {
  int si, h, kp;  // index of the slot in the launch's list, head, pair of key tiles
};
__device__ __forceinline__ Unit unit_of(const WeightParams& p, int u) {
  const int per_slot = p.H * p.n_pairs;
  Unit x;
  x.si = u / per_slot;
  const int r = u - x.si * per_slot;
  x.h = r / p.n_pairs;
  x.kp = r - x.h * p.n_pairs;
  return x;
}

__device__ __forceinline__ void record_timeout(const WeightParams& p, volatile int* abort_flag) {
  *abort_flag = 1;
  atomicCAS(p.status, kStatusOk, kStatusTimeout);
}

template <int D, bool kMask>
__global__ void __launch_bounds__(kThreads, 1) weights_kernel(const __grid_constant__ WeightParams p) {
  using C = Cfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  __shared__ Bars bars;
  __shared__ uint32_t tmem_base_sh;
  __shared__ volatile int abort_flag;
  __shared__ alignas(16) float nl[kStages][kTile];  // -lse * log2(e) of a stage's queries
  // masks: word w of key tile kt for each query of the stage; 0 none, 1 some, 2 all
  // of a tile's pairs visible; the Q tiles that the unit walks
  __shared__ alignas(16) uint32_t vis[kMask ? kStages : 1][2][4][kMask ? kTile : 1];
  __shared__ int seen[kMask ? kStages : 1][2];
  __shared__ uint32_t marks[kMask ? SVA_MAX_NODES * kMaxQueryTiles / 32 : 1];
  __shared__ float part[kMaxWeightSplit][2 * kTile];  // rank 0: the cluster's partial sums
  __shared__ volatile float part_lost;                // rank 0: a CTA of the cluster gave up

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int ns = p.n_split;
  const int rank = ns > 1 ? (int)blockIdx.x % ns : 0;
  // units of this CTA: u0, u0 + u_step, ...
  const int u0 = ns > 1 ? (int)blockIdx.x / ns : (int)blockIdx.x;
  const int u_step = ns > 1 ? p.units : (int)gridDim.x;  // masked launches: one unit a CTA
  const uint64_t tmo = p.timeout_ns;

  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    prefetch_tmap(&p.tmap_q);
    prefetch_tmap(&p.tmap_kv);
    abort_flag = 0;
    part_lost = 0.0f;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&bars.q_full[s], 1);
      mbar_init(&bars.l_full[s], 1);
      mbar_init(&bars.q_empty[s], 2 * kGroupWarps);
    }
    mbar_init(&bars.k_full, 1);
    mbar_init(&bars.k_empty, 2 * kGroupWarps);
    for (int k = 0; k < 2; ++k) {
      mbar_init(&bars.k_ready[k], kGroupWarps);
      for (int j = 0; j < 3; ++j) {
        mbar_init(&bars.s_full[k][j], 1);
        mbar_init(&bars.s_empty[k][j], kGroupWarps);
      }
    }
    mbar_init(&bars.drain, 2);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_base_sh, 512);
    tmem_relinquish();
  }
  pdl_wait();  // everything above is this CTA's own; what follows reads and writes global memory
  if constexpr (kMask) {
    // Which Q tiles of this unit have anything visible, by the tile mask and the
    // frames (token masks are looked at tile by tile, as they are staged).
    const Unit un = unit_of(p, u0);
    const int n_ref = p.first[un.si + 1] - p.first[un.si];
    const int n_all = n_ref * p.n_qt;
    for (int base = warp * 32; base < n_all; base += kThreads) {
      const int i = base + lane;
      bool on = false;
      if (i < n_all) {
        const int r = i / p.n_qt, qt = i - r * p.n_qt;
        const uint32_t ref = p.ref[p.first[un.si] + r];
        const int state = (ref >> kRefStateShift) & 31;
        on = true;
        if (p.tile_mask) {
          const uint32_t* row =
              p.tile_mask + ((size_t)(ref & 63) * p.n_qt + qt) * p.mask_words;
          const int k = state * p.n_qt + 2 * un.kp;
          on = ((row[k >> 5] >> (k & 31)) & 1u) != 0u;
          if (2 * un.kp + 1 < p.n_qt) on = on || ((row[(k + 1) >> 5] >> ((k + 1) & 31)) & 1u) != 0u;
        }
        if (state == 0 && (ref & kRefCausal)) {
          const int last = min((qt + 1) * kTile, p.T) - 1;
          on = on && last / p.frame_tokens >= 2 * un.kp * kTile / p.frame_tokens;
        }
      }
      const uint32_t m = __ballot_sync(0xffffffffu, on);
      if (lane == 0) marks[base >> 5] = m;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (ns > 1) cluster_sync();  // every CTA of the cluster runs, its part_lost is clear
  const uint32_t tbase = tmem_base_sh;

  // The Q tiles [begin, end) of a unit that this CTA takes.
  auto walk_of = [&](const Unit& un) {
    const int n_all = (p.first[un.si + 1] - p.first[un.si]) * p.n_qt;
    return Walk<kMask>(marks, (int)((long long)n_all * rank / ns), (int)((long long)n_all * (rank + 1) / ns),
                       p.n_qt);
  };

  int q_issued = 0, k_issued = 0;  // producer: copies started
  if (warp == 0) {
    // ------------------------------------------------------------ producer
    if (lane == 0) {
      bool ok = true;
      for (int u = u0; ok && u < p.units; u += u_step) {
        const Unit un = unit_of(p, u);
        const int row = ((p.slot[un.si] * 2) * p.H + un.h) * p.Tpad + un.kp * 2 * kTile;
        const bool two = 2 * un.kp + 1 < p.n_qt;
        ok = mbar_wait(&bars.k_empty, ((uint32_t)k_issued & 1u) ^ 1u, &abort_flag, tmo);
        if (!ok) break;
        mbar_arrive_expect_tx(&bars.k_full, (two ? 2 : 1) * C::kTileBytes);
#pragma unroll
        for (int b = 0; b < C::kBoxes; ++b) {
          tma_load_2d(smem + C::kOffK + b * C::kBoxBytes, &p.tmap_kv, &bars.k_full, b * 64, row);
          if (two)
            tma_load_2d(smem + C::kOffK + C::kTileBytes + b * C::kBoxBytes, &p.tmap_kv, &bars.k_full, b * 64,
                        row + kTile);
        }
        ++k_issued;
        Walk<kMask> walk = walk_of(un);
        int r, qt;
        while (walk.next(r, qt)) {
          const int node = p.ref[p.first[un.si] + r] & 63;
          const int st = q_issued % kStages;
          ok = mbar_wait(&bars.q_empty[st], ((uint32_t)(q_issued / kStages) & 1u) ^ 1u, &abort_flag, tmo);
          if (!ok) break;
          // fault_mode 2 (test hook): withhold the copy of the second tile
          if (!(p.fault_mode == 2 && q_issued == 1)) {
            mbar_arrive_expect_tx(&bars.q_full[st], C::kTileBytes);
#pragma unroll
            for (int b = 0; b < C::kBoxes; ++b)
              tma_load_4d(smem + st * C::kTileBytes + b * C::kBoxBytes, &p.tmap_q, &bars.q_full[st], b * 64, un.h,
                          qt * kTile, node);
          }
          ++q_issued;
        }
      }
      if (!ok) record_timeout(p, &abort_flag);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------ log-sum-exps and mask words
    bool ok = true;
    int it = 0;
    for (int u = u0; ok && u < p.units; u += u_step) {
      const Unit un = unit_of(p, u);
      Walk<kMask> walk = walk_of(un);
      int r, qt;
      while (walk.next(r, qt)) {
        const uint32_t ref = p.ref[p.first[un.si] + r];
        const int node = (int)(ref & 63u);
        const float* src = p.lse + ((size_t)node * p.H + un.h) * p.T;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = qt * kTile + k * 32 + lane;
          v[k] = ld_f32_if(src + row, row < p.T, INFINITY);
        }
        const int st = it % kStages;
        uint32_t w[kMask ? 4 : 1][8];  // of query k * 32 + lane: four words of each key tile
        if constexpr (kMask) {
          const int state = (int)(ref >> kRefStateShift) & 31;
          const uint32_t* base = state == 0 ? p.own_mask : p.hist_mask;
          const int words = (p.T + 31) / 32;
          const int w0 = un.kp * 8;  // first word of the pair of key tiles
          bool tile_on[2] = {true, true};
          if (p.tile_mask) {
            const uint32_t* row = p.tile_mask + ((size_t)node * p.n_qt + qt) * p.mask_words;
            const int k = state * p.n_qt + 2 * un.kp;
            tile_on[0] = ((row[k >> 5] >> (k & 31)) & 1u) != 0u;
            if (2 * un.kp + 1 < p.n_qt) tile_on[1] = ((row[(k + 1) >> 5] >> ((k + 1) & 31)) & 1u) != 0u;
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int q = qt * kTile + k * 32 + lane;
            const size_t qrow = (size_t)node * p.T + q;
            const uint32_t* row = state == 0 ? base + qrow * p.own_words
                                             : base + (qrow * p.hist_states + (state - 1)) * p.hist_words;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              w[k][j] = ld_global_u32_if(row + w0 + j, base != nullptr && q < p.T && w0 + j < words, ~0u);
            int upto = p.T;  // keys that the frames leave visible
            if (state == 0 && (ref & kRefCausal)) upto = (q / p.frame_tokens + 1) * p.frame_tokens;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int n = upto - (w0 + j) * 32;
              if (n < 32) w[k][j] &= n <= 0 ? 0u : (1u << n) - 1u;
              // keys past T have no sum: they count as visible so that a whole
              // tile of a ragged slot can be one
              const int past = p.T - (w0 + j) * 32;
              if (past < 32) w[k][j] |= past <= 0 ? ~0u : ~0u << past;
              // a query that saw nothing adds nothing, whatever its row holds,
              // nor do the rows past T to a key that no query sees
              if (!tile_on[j >> 2] || v[k] == -INFINITY || q >= p.T) w[k][j] = 0u;
            }
          }
        }
        if (!__all_sync(0xffffffffu, mbar_wait(&bars.q_empty[st], ((uint32_t)(it / kStages) & 1u) ^ 1u,
                                               &abort_flag, tmo))) {
          ok = false;
          break;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          nl[st][k * 32 + lane] = v[k] == -INFINITY ? -INFINITY : v[k] * -1.4426950408889634f;
        if constexpr (kMask) {
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) {
            uint32_t any = 0u, all = ~0u;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t x = w[k][kt * 4 + j];
                vis[st][kt][j][k * 32 + lane] = x;
                any |= x;
                all &= x;
              }
            any = __reduce_or_sync(0xffffffffu, any);
            all = __reduce_and_sync(0xffffffffu, all);
            if (lane == 0) seen[st][kt] = any == 0u ? 0 : (all == ~0u ? 2 : 1);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.l_full[st]);
        ++it;
      }
    }
    if (!ok && lane == 0) record_timeout(p, &abort_flag);
  } else if (warp < 4) {
    // ------------------------------------------------------------ MMA issuers
    const int kt = warp == 1 ? 0 : 1;
    constexpr uint32_t idesc = idesc_bf16_f32(kTile, kTile, false);
    const uint64_t dQ = sdesc_sw128(smem_u32(smem), 16, 1024);
    const uint32_t kcol = tbase + (uint32_t)kt * C::kKCols;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, &abort_flag, tmo)) != 0;
    };
    bool ok = true;
    int it = 0, n_unit = 0;
    int buf = kt;  // S buffer of step 2 * it + kt
    for (int u = u0; ok && u < p.units; u += u_step, ++n_unit) {
      const Unit un = unit_of(p, u);
      ok = wait(&bars.k_ready[kt], (uint32_t)n_unit & 1u);
      if (!ok) break;
      Walk<kMask> walk = walk_of(un);
      int r, qt;
      while (walk.next(r, qt)) {
        const int st = it % kStages;
        // the buffer's last user: the other group, 1 (kt = 1) or 2 items ago
        const int before = it - (kt == 1 ? 1 : 2);
        ok = wait(&bars.q_full[st], (uint32_t)(it / kStages) & 1u) &&
             (before < 0 || wait(&bars.s_empty[1 - kt][before % 3], (uint32_t)(before / 3) & 1u));
        if (!ok) break;
        tc_fence_after();
        const uint32_t dcol = tbase + C::kColS + (uint32_t)buf * kTile;
        const uint64_t b = dQ + (uint64_t)(st * (C::kTileBytes >> 4));
#pragma unroll
        for (int x = 0; x < C::kBoxes; ++x)
          mma_ts_kmajor_x4(dcol, kcol + x * 32, b + (uint64_t)(x * (C::kBoxBytes >> 4)), idesc, x > 0 ? 1u : 0u);
        mma_commit_warp(&bars.s_full[kt][it % 3]);
        buf = buf == 0 ? 2 : buf - 1;  // two steps on, modulo 3
        ++it;
      }
    }
    if (!ok && lane == 0) record_timeout(p, &abort_flag);
  } else {
    // ------------------------------------------------------------ sums
    const int kt = (warp - 4) >> 2;
    const int q4 = warp & 3;  // TMEM lane quarter this warp may access
    const int row = q4 * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    const uint64_t sl2x2 = f2u(p.scale_log2, p.scale_log2);
    bool ok = true;
    int n_unit = 0, it = 0, buf = kt;
    // This thread's row of the next unit's K, shared memory -> TMEM.
    auto copy_k = [&]() {
      if (!__all_sync(0xffffffffu, mbar_wait(&bars.k_full, (uint32_t)n_unit & 1u, &abort_flag, tmo))) return false;
      const uint32_t at = smem_u32(smem + C::kOffK + kt * C::kTileBytes) + (uint32_t)(row * 128);
#pragma unroll
      for (int b = 0; b < C::kBoxes; ++b) {
        uint32_t w[32];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint4 v = ld_shared_v4(at + (uint32_t)(b * C::kBoxBytes + ((j ^ (row & 7)) << 4)));
          w[4 * j] = v.x; w[4 * j + 1] = v.y; w[4 * j + 2] = v.z; w[4 * j + 3] = v.w;
        }
        tmem_st32(tbase + lane_off + (uint32_t)kt * C::kKCols + b * 32, w);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&bars.k_ready[kt]);
        mbar_arrive(&bars.k_empty);
      }
      ++n_unit;
      return true;
    };
    if (u0 < p.units) ok = copy_k();
    for (int u = u0; ok && u < p.units; u += u_step) {
      const Unit un = unit_of(p, u);
      const int key = (un.kp * 2 + kt) * kTile + row;
      const size_t at = ((size_t)p.slot[un.si] * p.H + un.h) * p.T + key;
      const bool mine = key < p.T;
      const bool has_keys = key - lane < p.T;  // this warp's part of the tile; K is not loaded past the slot
      const float before = ld_f32_if(p.prev + at, p.prev != nullptr && mine && ns == 1, 0.0f);
      float total = 0.0f;
      Walk<kMask> walk = walk_of(un);
      int r, qt;
      bool more = walk.next(r, qt);
      bool next_k = u + u_step < p.units;  // another unit's K is to follow
      if (!more && next_k) {               // no Q tile (masks only): nothing reads this K
        ok = copy_k();
        if (!ok) break;
      }
      while (more) {
        const int st = it % kStages;
        if (!__all_sync(0xffffffffu,
                        mbar_wait(&bars.l_full[st], (uint32_t)(it / kStages) & 1u, &abort_flag, tmo) &&
                            mbar_wait(&bars.s_full[kt][it % 3], (uint32_t)(it / 3) & 1u, &abort_flag, tmo))) {
          ok = false;
          break;
        }
        tc_fence_after();
        more = walk.next(r, qt);
        if (!more && next_k) {  // the unit's last S is complete: no MMA reads its K any more
          ok = copy_k();
          if (!ok) break;
        }
        const int look = !has_keys ? 0 : kMask ? seen[st][kt] : 2;
        const uint32_t scol = tbase + lane_off + C::kColS + (uint32_t)buf * kTile;
        uint64_t acc[4] = {0, 0, 0, 0};
        auto add = [&](const uint32_t (&s)[32], int c) {
          const ulonglong2* nl2 = reinterpret_cast<const ulonglong2*>(&nl[st][c * 32]);
          const uint4* vw = reinterpret_cast<const uint4*>(&vis[kMask ? st : 0][kt][q4][kMask ? c * 32 : 0]);
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const ulonglong2 n = nl2[e >> 2];
            float x0, x1, x2, x3;
            ffma2(x0, x1, __uint_as_float(s[e]), __uint_as_float(s[e + 1]), sl2x2, n.x);
            ffma2(x2, x3, __uint_as_float(s[e + 2]), __uint_as_float(s[e + 3]), sl2x2, n.y);
            if constexpr (kMask) {
              if (look == 1) {
                const uint4 v = vw[e >> 2];
                if (!((v.x >> lane) & 1u)) x0 = -INFINITY;
                if (!((v.y >> lane) & 1u)) x1 = -INFINITY;
                if (!((v.z >> lane) & 1u)) x2 = -INFINITY;
                if (!((v.w >> lane) & 1u)) x3 = -INFINITY;
              }
            }
            acc[(e >> 1) & 3] = fadd2(acc[(e >> 1) & 3], ex2(x0), ex2(x1));
            acc[((e >> 1) + 1) & 3] = fadd2(acc[((e >> 1) + 1) & 3], ex2(x2), ex2(x3));
          }
        };
        uint32_t s0[32], s1[32];
        if (look != 0) {
          tmem_ld32(scol, s0);
          tmem_ld32(scol + 32, s1);
          tmem_wait_ld(s0);
          tmem_wait_ld(s1);
          add(s0, 0);
          add(s1, 1);
          tmem_ld32(scol + 64, s0);
          tmem_ld32(scol + 96, s1);
          tmem_wait_ld(s0);
          tmem_wait_ld(s1);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.s_empty[kt][it % 3]);
        if (look != 0) {
          add(s0, 2);
          add(s1, 3);
          float a[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) u2f(acc[k], a[2 * k], a[2 * k + 1]);
          total += ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.q_empty[st]);
        buf = buf == 0 ? 2 : buf - 1;  // two steps on, modulo 3
        ++it;
      }
      if (!ok) break;
      if (ns == 1) {
        if (mine) p.out[at] = __fmaf_rn(p.decay, before, total);
      } else {
        st_cluster_f32(mapa_shared(smem_u32(&part[rank][kt * kTile + row]), 0), total);
        __syncwarp();
      }
    }
    if (!ok) {
      if (lane == 0) {
        record_timeout(p, &abort_flag);
        if (ns > 1) st_cluster_f32(mapa_shared(smem_u32(const_cast<float*>(&part_lost)), 0), 1.0f);
      }
      __syncwarp();
    }
  }
  __syncwarp();
  if (ns > 1) {
    cluster_sync();  // the partial sums are there
    if (rank == 0 && warp >= 4 && part_lost == 0.0f) {
      const Unit un = unit_of(p, u0);
      const int j = threadIdx.x - 128;
      const int key = un.kp * 2 * kTile + j;
      if (key < p.T) {
        const size_t at = ((size_t)p.slot[un.si] * p.H + un.h) * p.T + key;
        float total = 0.0f;
        for (int k = 0; k < ns; ++k) total += part[k][j];
        const float before = ld_f32_if(p.prev + at, p.prev != nullptr, 0.0f);
        p.out[at] = __fmaf_rn(p.decay, before, total);
      }
    }
  }

  // ---------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (abort_flag) {
    // Some wait expired: wait (bounded, ignoring the abort flag) for the copies
    // and MMAs that this CTA still has in flight.
    const int zero = 0;
    if (warp == 0 && lane == 0) {
      if (k_issued > 0) mbar_wait(&bars.k_full, (uint32_t)(k_issued - 1) & 1u, &zero, tmo);
      for (int i = (q_issued > kStages ? q_issued - kStages : 0); i < q_issued; ++i) {
        if (p.fault_mode == 2 && i == 1) continue;  // the copy the test hook withheld
        mbar_wait(&bars.q_full[i % kStages], (uint32_t)(i / kStages) & 1u, &zero, tmo);
      }
    } else if (warp == 1 || warp == 3) {
      mma_commit_warp(&bars.drain);  // the same elected lane that issued the MMAs
      mbar_wait(&bars.drain, 0, &zero, tmo);
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tbase, 512);
  }
}

template <int D, bool kMask>
cudaError_t launch(const WeightParams& p, int grid, cudaStream_t s) {
  static std::mutex mu;
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!configured[dev]) {
      e = cudaFuncSetAttribute(weights_kernel<D, kMask>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               Cfg<D>::kSmemBytes);
      if (e != cudaSuccess) return e;
      configured[dev] = true;
    }
  }
  LaunchConfig l(dim3((unsigned)grid), kThreads, Cfg<D>::kSmemBytes, s, p.n_split > 1 ? p.n_split : 0);
  return cudaLaunchKernelEx(&l.cfg, weights_kernel<D, kMask>, p);
}

}  // namespace

cudaError_t launch_weights(const WeightParams& p, int head_dim, int grid, cudaStream_t s) {
  if (head_dim == 128) return p.masked ? launch<128, true>(p, grid, s) : launch<128, false>(p, grid, s);
  if (head_dim == 64) return p.masked ? launch<64, true>(p, grid, s) : launch<64, false>(p, grid, s);
  return cudaErrorInvalidValue;
}

}  // namespace sva
