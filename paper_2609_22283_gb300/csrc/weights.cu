// How much attention every cached key got from a launch's queries
// (sva_attend_weights): for a slot s, head h and key v
//   w[s][h][v] = decay * prev + sum_i sum_u exp(scale * q_iu . k_v + M(u, v) - lse_iu)
// over the nodes i that see s and their queries u, the log-sum-exps lse being
// the attention's.  With them known no running maximum is needed and no V: one
// product and one exponential a (query, key) pair, and sums over queries.
//
// So the product is taken the other way round, S^T = K Q^T: a key is a TMEM lane,
// and the threads that hold its scores add their exponentials up in registers.  No
// score crosses threads, a unit's sum over all its queries stays in two registers
// of two threads, and nothing is added atomically: results do not depend on the
// order of CTAs.
//
// One unit is (slot, head, pair of 128-key tiles).  K (the A operand) is copied
// to TMEM once a unit, as packed bf16, so that the MMAs read only Q from shared
// memory (with both operands there M = N = 128 needs all of its 128 B a cycle);
// Q tiles of 128 queries stream past it, for every node that sees the slot.
//   warp 0     TMA producer: a unit's K tiles, then its Q tiles (4 or 8 stages,
//              freed by the MMAs' commits); with masks also the next unit's marks;
//   warp 2     -lse * log2(e) of a Q tile's rows (-inf past the last row); with
//              masks also the tile's token words, by copies that need no register;
//   warps 1, 3 MMA issuers of key tiles 0 and 1;
//   warps 4-19 sums: warps 4-11 key tile 0, warps 12-19 key tile 1; a warp takes 32
//              keys and half of the queries.
// TMEM: K0, K1 (d / 2 columns each), then three S buffers of 128 columns that the
// steps (Q tile i, key tile kt) take in turn, n = 2 i + kt in buffer n % 3: the
// two groups work in opposite phase and each S is issued while the group before
// still works.  S barriers are per group, so that their one waiter waits for
// every phase; the buffer of step n was the other group's at step n - 3.
// A CTA takes units in turn, and the pipeline runs through their ends: the next
// unit's K waits in shared memory, and a group copies it to TMEM when the last S
// of the unit is complete, ahead of the sums over that S.
//
// What bounds it: the sums.  256 keys x 128 queries are 1024 cycles of the tensor
// core at d = 128 (512 at 64) and 1024 of the exponential unit, which shares its
// issue queue with the TMEM and shared-memory loads: that loop alone, without
// barriers or MMAs, takes 1240 cycles, the kernel 1550 at d = 128 (4680 queries over
// 18720 keys, 12 heads: 178 us, 1510 TFLOP/s; four such nodes over 32760 keys 1201
// us, 1570; these in runs of 20 calls, in long runs, where the power limit holds the
// clock down, 189 to 198 and 1285 to 1351), 1500 at 64 (2 x 2160 queries over 10800
// keys, 16 heads: 135 us, of which the last of ten rounds and the empty half of the
// ninth pair of key tiles are a ninth).  Units are whole: 84 of 1560 queries on 152 SMs
// take 15 us, 168 take 25.  Taken
// on the way, each on the first of these cases: eight summing warps with 128 queries
// each 220 us, sixteen 206; ring positions counted instead of divided 195; Q stages
// freed by the MMAs 193; scores read 16 columns at a time (32 leave a thread too few
// of its 96 registers to overlap exponentials) 186; no branch while scores are on
// their way from TMEM (the compiler waits for them at it) 177.  Not kept: eight
// warps in that form 184; the next item's first scores loaded ahead 196 to 230; S in
// halves of 64 queries with six buffers 209; both operands in shared memory 194; 2^x
// by a polynomial for part of the scores (no gain in the loop alone).
//
// Launches with fewer units than SMs split a unit's Q tiles over a cluster; the
// partial sums go to the first CTA's shared memory and are added in rank order.
// Launches with masks (or frame causality) have a bitmap for each key tile of a unit,
// of the (node, Q tile) pairs that have any visible pair as far as the tile mask, the
// frames and the scan of the token masks say; only tiles marked for either are loaded
// and multiplied.  Units then differ in work, so the grid has a CTA for each, and a
// running CTA takes the next that has not started (cluster launch control) and marks
// its tiles while its own unit's last Q tiles are on their way: the pipeline runs
// through, and the SMs that are done first take more.  A CTA for each unit instead
// takes 205 us where that takes 190.  An item marked for one of a unit's key tiles is
// multiplied for both.  Items that no token mask and no frame cuts are
// summed as without masks (tile masks of the history with all bits set: 191 us on the
// first case above, half of them set at random 153, a quarter 112; frame causality alone
// 193); elsewhere a warp without a visible pair in its 32 keys x 32
// queries skips them, and leaves out exponentials by the transposed bits where some are visible
// (4680 queries over own and three history chunks, keys within 6 patch rows and
// columns: 192 us, of which the scan takes 9; random bits 302; all set 259).  The two
// blocks of 32 queries are looked at together, so that their transpositions overlap and
// the sums run through both: one after the other they took 16, 35 and 29 us more.
// All waits are bounded as in the attention kernel; a sum that is not whole when a
// wait runs out is not written.
#include <mutex>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"
#include "weights.h"

namespace sva {
namespace {

using namespace ptx;

constexpr int kThreads = 640;
constexpr int kRing = 3;  // S buffers and stages of log-sum-exps: item i uses number i % 3
constexpr int kMaxStages = 8;
constexpr int kGroupWarps = 8;  // of a key tile: four TMEM lane quarters x two halves of the queries

template <int D>
struct Cfg {
  static constexpr int kBoxBytes = kTile * 64 * 2;  // one 128-row x 64-column bf16 box
  static constexpr int kBoxes = D / 64;
  static constexpr int kTileBytes = kBoxBytes * kBoxes;
  static constexpr int kStages = D == 128 ? 4 : 8;  // Q tiles in flight
  static constexpr int kOffK = kStages * kTileBytes;
  static constexpr int kSmemBytes = kOffK + 2 * kTileBytes + 1024;  // + alignment slack
  static constexpr uint32_t kKCols = D / 2;          // TMEM columns of a K tile
  static constexpr uint32_t kColS = 128;             // first S buffer
};

// Position in the rings of three: i % 3 and the parity of i / 3.
struct Ring {
  int at = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step() {
    ++at;
    if (at == 3) {
      at = 0;
      phase ^= 1u;
    }
  }
};

// The kernel's instances: without masks; tile masks and frame causality, where most
// marked tiles are wholly visible; token masks (with any of them).
enum class Masks { kNone, kTiles, kWords };

// What goes with a Q tile, and the barriers of number i % 3 of the rings.
template <bool kWords>
struct alignas(16) Stage {
  float nl[kTile];      // -lse * log2(e) of its queries
  // token masks: word w of key tile kt for each query (rows of 132: eight words of
  // four queries lie on 32 banks)
  uint32_t word[kWords ? 8 : 1][kWords ? kTile + 4 : 4];
  uint64_t l_full;      // nl, word and info are there
  uint64_t l_empty;     // both groups are done with them
  uint64_t s_full[2], s_empty[2];  // S of each group
  uint32_t info;        // masks: kItem bits, the query tile above them
};
// The item's key tiles that are marked; it has token words; frames hide keys of it;
// every pair of the marked tiles is visible.
constexpr uint32_t kItemOn = 1, kItemWords = 4, kItemCausal = 8, kItemPlain = 16;
constexpr int kItemTileShift = 8;

struct Bars {
  uint64_t q_full[kMaxStages];   // a Q tile has landed
  uint64_t q_empty[kMaxStages];  // both groups' MMAs have read it
  uint64_t k_full, k_empty;   // K tiles of a unit in shared memory
  uint64_t k_ready[2];        // K tile in TMEM
  uint64_t t_full[2], t_empty[2];  // the second half's sums of a unit
  uint64_t drain;
  // masks: the marks of the CTA's n-th unit, number n % 2, are there, are no longer read;
  // the CTA that was taken is known
  uint64_t m_full[2], m_empty[2], claimed;
};
constexpr int kMarkReaders = 3 + 2 * kGroupWarps;  // warps that walk a unit's tiles, but the producer

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Pairs of fp32 in a 64-bit register, two lanes an instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t r, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
// (a0, a1) * b + c
__device__ __forceinline__ void fma2(float& o0, float& o1, float a0, float a1, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair(a0, a1)), "l"(b), "l"(c));
  unpair(r, o0, o1);
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

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

// Each thread reads 16 columns of its lane; not valid until tmem_wait_ld16(r) has run.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_ld16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
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

// One word to shared memory without a register, zero where `load` is false; and an
// arrival on `bar` when this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_u32_if(uint32_t* dst, const uint32_t* src, bool load) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(load ? 4 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_u32(uint32_t* dst, const uint32_t* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Caller data, by ordinary loads (see ptx.cuh).
__device__ __forceinline__ float ld_f32_if(const float* p, bool load, float other) {
  return __uint_as_float(
      ld_global_u32_if(reinterpret_cast<const uint32_t*>(p), load, __float_as_uint(other)));
}

// The Q tiles of a unit in order: every (ref, query tile), or those marked for
// either key tile in bitmaps over ref * n_qt + tile.
constexpr int kMarkWords = SVA_MAX_NODES * kMaxQueryTiles / 32;
template <bool kMask>
struct Walk {
  const uint32_t (*marks)[kMask ? kMarkWords : 1];
  int at, end, n_qt, r, qt;  // kMask: word of the bitmaps, and the first item of ref r in `qt`
  uint32_t left;             // kMask: the word's bits still to come
  __device__ __forceinline__ Walk(const uint32_t (*marks_)[kMask ? kMarkWords : 1], int begin, int end_, int n_qt_)
      : marks(marks_), at(begin), end(end_), n_qt(n_qt_), r(begin > 0 ? begin / n_qt_ : 0), qt(begin - r * n_qt_), left(0) {
    if constexpr (kMask) {
      at = begin >> 5;
      left = begin < end ? word(at) & (~0u << (begin & 31)) : 0u;
      qt = r * n_qt;
    }
  }
  __device__ __forceinline__ uint32_t word(int w) const {
    uint32_t m = marks[0][w] | marks[kMask ? 1 : 0][w];
    if (w == end >> 5) m &= (1u << (end & 31)) - 1u;
    return m;
  }
  // How many there are (before the first next).
  __device__ __forceinline__ int count() const {
    if constexpr (kMask) {
      int n = 0;
      const int words = (end + 31) >> 5;
      for (int w = at; w < words; ++w) n += __popc(w == at ? left : word(w));
      return n;
    } else {
      return end - at;
    }
  }
  // The next item into (r, qt); false past the last.
  __device__ __forceinline__ bool next(int& r_out, int& qt_out) {
    if constexpr (kMask) {
      const int words = (end + 31) >> 5;
      while (left == 0u) {
        if (++at >= words) return false;
        left = word(at);
      }
      const int i = (at << 5) + __ffs(left) - 1;
      left &= left - 1u;
      while (i - qt >= n_qt) {
        qt += n_qt;
        ++r;
      }
      r_out = r;
      qt_out = i - qt;
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
  // Is the item marked for key tile kt?
  __device__ __forceinline__ bool marked(int kt, int r_in, int qt_in) const {
    const int i = r_in * n_qt + qt_in;
    return (marks[kt][i >> 5] >> (i & 31)) & 1u;
  }
};

// Takes a CTA of this launch that has not started: its number goes to `response`, with
// 16 bytes on `bar`.  Not to be called again once there was none.
__device__ __forceinline__ void try_cancel(void* response, uint64_t* bar) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the last response has been read
  mbar_arrive_expect_tx(bar, 16);
  asm volatile(
      "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
          smem_u32(response)),
      "r"(smem_u32(bar))
      : "memory");
}
// The CTA that was taken, -1 where there was none.
__device__ __forceinline__ int canceled_cta(const void* response) {
  const uint4 r = ld_shared_v4(smem_u32(response));
  int cta;
  asm volatile(
      "{\n"
      " .reg .b128 h;\n"
      " .reg .b64 lo, hi;\n"
      " .reg .pred p;\n"
      " mov.b64 lo, {%1, %2};\n"
      " mov.b64 hi, {%3, %4};\n"
      " mov.b128 h, {lo, hi};\n"
      " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n"
      " mov.s32 %0, -1;\n"
      " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, h;\n"
      "}\n"
      : "=&r"(cta)
      : "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w));
  return cta;
}

struct Unit {
  int si, h, kp;  // index of the slot in the launch's list, head, pair of key tiles
};
__device__ __forceinline__ Unit unit_of(const WeightParams& p, int u) {
  const uint32_t per_slot = (uint32_t)(p.H * p.n_pairs);
  Unit x;
  x.si = (int)((uint32_t)u / per_slot);
  const uint32_t r = (uint32_t)u - (uint32_t)x.si * per_slot;
  x.h = (int)(r / (uint32_t)p.n_pairs);
  x.kp = (int)r - x.h * p.n_pairs;
  return x;
}

__device__ __forceinline__ void record_timeout(const WeightParams& p, volatile int* abort_flag) {
  *abort_flag = 1;
  atomicCAS(p.status, kStatusOk, kStatusTimeout);
}

template <int D, Masks kMasks>
__global__ void __launch_bounds__(kThreads, 1) weights_kernel(const __grid_constant__ WeightParams p) {
  using C = Cfg<D>;
  constexpr bool kMask = kMasks != Masks::kNone, kWords = kMasks == Masks::kWords;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  __shared__ Bars bars;
  __shared__ uint32_t tmem_base_sh;
  __shared__ volatile int abort_flag;
  __shared__ Stage<kWords> stage[kRing];
  __shared__ uint32_t marks[2][2][kMask ? kMarkWords : 1];  // of the CTA's units, by turns
  __shared__ int unit_sh[2];                                // their numbers, -1 after the last
  __shared__ uint4 response;
  // rank 0: the cluster's partial sums; a cluster takes one unit, with masks they lie on
  // the second unit's marks
  __shared__ float part_sh[kMask ? 1 : kMaxWeightSplit][2 * kTile];
  static_assert(!kMask || sizeof(marks[1]) == sizeof(float) * kMaxWeightSplit * 2 * kTile, "part");
  float (*part)[2 * kTile] = kMask ? reinterpret_cast<float (*)[2 * kTile]>(marks[1]) : part_sh;
  __shared__ float half_sum[2][kTile];                // the second half's sums of a unit
  __shared__ volatile float part_lost;                // rank 0: a CTA of the cluster gave up

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int ns = p.n_split;
  const int rank = ns > 1 ? (int)blockIdx.x % ns : 0;
  // units of this CTA: u0, u0 + u_step, ...; with masks u0, and those of the CTAs it takes
  const int u0 = ns > 1 ? (int)blockIdx.x / ns : (int)blockIdx.x;
  const int u_step = ns > 1 ? p.units : (int)gridDim.x;
  const uint64_t tmo = p.timeout_ns;

  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    prefetch_tmap(&p.tmap_q);
    prefetch_tmap(&p.tmap_kv);
    abort_flag = 0;
    part_lost = 0.0f;
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&bars.q_full[s], 1);
      mbar_init(&bars.q_empty[s], 2);
    }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(&stage[s].l_full, kWords ? 33 : 1);  // nl, and with masks each lane's copies
      mbar_init(&stage[s].l_empty, 2 * kGroupWarps);
      for (int k = 0; k < 2; ++k) {
        mbar_init(&stage[s].s_full[k], 1);
        mbar_init(&stage[s].s_empty[k], kGroupWarps);
      }
    }
    mbar_init(&bars.k_full, 1);
    mbar_init(&bars.k_empty, 2 * kGroupWarps);
    for (int k = 0; k < 2; ++k) {
      mbar_init(&bars.k_ready[k], kGroupWarps);
      mbar_init(&bars.t_full[k], kGroupWarps / 2 * 32);
      mbar_init(&bars.t_empty[k], kGroupWarps / 2 * 32);
      mbar_init(&bars.m_full[k], 1);
      mbar_init(&bars.m_empty[k], kMarkReaders);
    }
    mbar_init(&bars.claimed, 1);
    unit_sh[0] = u0;
    unit_sh[1] = -1;
    mbar_init(&bars.drain, 2);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_base_sh, 512);
    tmem_relinquish();
  }
  pdl_wait();  // everything above is this CTA's own; what follows reads and writes global memory
  auto tiles_of = [&](const Unit& un) { return (p.first[un.si + 1] - p.first[un.si]) * p.n_qt; };  // < 2^16
  // Which Q tiles have anything visible of either key tile of a unit, by the tile mask,
  // the frames and the scan of the token masks: of 32 tiles, a lane's each.
  auto mark = [&](const Unit& un, uint32_t (&to)[2][kMask ? kMarkWords : 1], int base) {
    const int i = base + lane;
    bool on[2] = {false, false};
    if (i < tiles_of(un)) {
      const int r = i / p.n_qt, qt = i - r * p.n_qt;
      const uint32_t ref = p.ref[p.first[un.si] + r];
      const int state = (ref >> kRefStateShift) & 31;
      const size_t qrow = (size_t)(ref & 63) * p.n_qt + qt;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int t = 2 * un.kp + kt, k = state * p.n_qt + t;
        on[kt] = t < p.n_qt;
        if (on[kt] && p.tile_mask) on[kt] = (p.tile_mask[qrow * p.mask_words + (k >> 5)] >> (k & 31)) & 1u;
        if (on[kt] && p.any_tile) on[kt] = p.any_tile[qrow * p.any_stride + k] != 0;
        if (on[kt] && state == 0 && (ref & kRefCausal)) {
          const int last = min((qt + 1) * kTile, p.T) - 1;
          on[kt] = last / p.frame_tokens >= t * kTile / p.frame_tokens;
        }
      }
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint32_t m = __ballot_sync(0xffffffffu, on[kt]);
      if (lane == 0) to[kt][base >> 5] = m;
    }
  };
  if constexpr (kMask) {
    const Unit un = unit_of(p, u0);
    for (int base = warp * 32; base < tiles_of(un); base += kThreads) mark(un, marks[0], base);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (ns > 1) cluster_sync();  // every CTA of the cluster runs, its part_lost is clear
  const uint32_t tbase = tmem_base_sh;

  // The Q tiles [begin, end) of the CTA's n-th unit that it takes.
  auto walk_of = [&](const Unit& un, int n) {
    const uint32_t n_all = (uint32_t)(p.first[un.si + 1] - p.first[un.si]) * (uint32_t)p.n_qt;  // < 2^16
    uint32_t begin = 0, end = n_all;
    if (ns > 1) {
      begin = n_all * (uint32_t)rank / (uint32_t)ns;
      end = n_all * (uint32_t)(rank + 1) / (uint32_t)ns;
    }
    return Walk<kMask>(marks[kMask ? n & 1 : 0], (int)begin, (int)end, p.n_qt);
  };
  // The CTA's n-th unit, after `u`; -1 past the last, or where a wait expired (`ok`).
  auto unit_after = [&](int u, int n, bool& ok) {
    if constexpr (kMask) {
      ok = mbar_wait(&bars.m_full[n & 1], (uint32_t)(n >> 1) & 1u, &abort_flag, tmo);
      ok = __all_sync(0xffffffffu, ok);
      return ok ? unit_sh[n & 1] : -1;
    } else {
      return u + u_step < p.units ? u + u_step : -1;
    }
  };
  // This warp reads the marks of the n-th unit no more.
  auto walked = [&](int n) {
    if constexpr (kMask) {
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.m_empty[n & 1]);
    }
  };

  int q_issued = 0, k_issued = 0;  // producer: copies started
  if (warp == 0) {
    // ------------------------------------------------------------ producer
    // One lane; with masks the warp, which also takes and marks the next unit.
    if (kMask || lane == 0) {
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        const bool there = mbar_wait(bar, parity, &abort_flag, tmo);
        return kMask ? __all_sync(0xffffffffu, there) != 0 : there;
      };
      const bool first_lane = lane == 0;
      bool ok = true;
      const bool takes = kMask && p.take != 0;
      if (kMask && first_lane) {
        mbar_arrive(&bars.m_full[0]);  // the first unit's marks are there
        if (!takes) mbar_arrive(&bars.m_full[1]);  // and no unit follows
      }
      for (int u = u0, n = 0; u >= 0; ++n) {
        const Unit un = unit_of(p, u);
        const int row = ((p.slot[un.si] * 2) * p.H + un.h) * p.Tpad + un.kp * 2 * kTile;
        const bool two = 2 * un.kp + 1 < p.n_qt;
        ok = wait(&bars.k_empty, ((uint32_t)k_issued & 1u) ^ 1u);
        if (!ok) break;
        if (first_lane) {
          mbar_arrive_expect_tx(&bars.k_full, (two ? 2 : 1) * C::kTileBytes);
#pragma unroll
          for (int b = 0; b < C::kBoxes; ++b) {
            tma_load_2d(smem + C::kOffK + b * C::kBoxBytes, &p.tmap_kv, &bars.k_full, b * 64, row);
            if (two)
              tma_load_2d(smem + C::kOffK + C::kTileBytes + b * C::kBoxBytes, &p.tmap_kv, &bars.k_full, b * 64,
                          row + kTile);
          }
        }
        ++k_issued;
        Walk<kMask> walk = walk_of(un, n);
        // The next unit: a CTA that has not started is taken when few tiles are left to load
        // (late enough that an SM that is done earlier gets it), then 32 of its tiles are
        // marked with every tile loaded: the Q tiles in flight hide that.
        int next = -1, at = 0;   // its number, the next tile to mark
        int left = 0, early = 0;
        enum { kLater, kClaimed, kMarking, kDone } step = takes ? kLater : kDone;
        if constexpr (kMask) {
          left = walk.count();
          early = 4 + (tiles_of(un) >> 5);
        }
        // The unit whose marks are to be free: the one before; or this one where it has no tile
        // (no S makes the sums wait for the MMA warps then, and k_ready has one phase).
        const int free = left == 0 ? n : n - 1;
        auto advance = [&]() {
          if (step == kLater) {
            if (first_lane) try_cancel(&response, &bars.claimed);
            step = kClaimed;
          } else if (step == kClaimed) {
            const int zero = 0;  // the response is waited for in any case
            ok = __all_sync(0xffffffffu, mbar_wait(&bars.claimed, (uint32_t)n & 1u, &zero, tmo)) != 0;
            if (ok) next = canceled_cta(&response);
            ok = ok && wait(&bars.m_empty[free & 1], (uint32_t)(free >> 1) & 1u);
            step = kMarking;
          } else {
            if (next >= 0 && at < tiles_of(unit_of(p, next))) {
              mark(unit_of(p, next), marks[(n + 1) & 1], at);
              at += 32;
              return;
            }
            if (first_lane) {
              unit_sh[(n + 1) & 1] = next;
              mbar_arrive(&bars.m_full[(n + 1) & 1]);
            }
            step = kDone;
          }
        };
        int r, qt;
        while (walk.next(r, qt)) {
          if constexpr (kMask) {
            if (left-- <= early && step != kDone) advance();
            if (!ok) break;
          }
          const int node = p.ref[p.first[un.si] + r] & 63;
          const int st = q_issued % C::kStages;
          ok = wait(&bars.q_empty[st], ((uint32_t)(q_issued / C::kStages) & 1u) ^ 1u);
          if (!ok) break;
          // fault_mode 2 (test hook): withhold the copy of the second tile
          if (first_lane && !(p.fault_mode == 2 && q_issued == 1)) {
            mbar_arrive_expect_tx(&bars.q_full[st], C::kTileBytes);
#pragma unroll
            for (int b = 0; b < C::kBoxes; ++b)
              tma_load_4d(smem + st * C::kTileBytes + b * C::kBoxBytes, &p.tmap_q, &bars.q_full[st], b * 64, un.h,
                          qt * kTile, node);
          }
          ++q_issued;
        }
        if constexpr (kMask) {
          while (ok && step != kDone) advance();
          u = next;
        } else {
          u = unit_after(u, n + 1, ok);
        }
        if (!ok) {
          const int zero = 0;  // no response outlives the CTA
          if (kMask && step == kClaimed) mbar_wait(&bars.claimed, (uint32_t)n & 1u, &zero, tmo);
          break;
        }
      }
      if (!ok && first_lane) record_timeout(p, &abort_flag);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------ log-sum-exps
    // Loaded an item ahead of their stage.
    bool ok = true;
    int u = u0, n = 0;
    Unit un = unit_of(p, u);
    Walk<kMask> walk = walk_of(un, n);
    float v[4];  // of queries k * 32 + lane
    int r = 0, qt = 0;
    auto load = [&]() {  // the next item's; false past the last
      while (!walk.next(r, qt)) {
        walked(n);
        u = unit_after(u, ++n, ok);
        if (u < 0) return false;
        un = unit_of(p, u);
        walk = walk_of(un, n);
      }
      const int node = p.ref[p.first[un.si] + r] & 63;
      const float* src = p.lse + ((size_t)node * p.H + un.h) * p.T;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int row = qt * kTile + k * 32 + lane;
        v[k] = ld_f32_if(src + row, row < p.T, INFINITY);
      }
      return true;
    };
    // What the masks say of an item, and its token words: of each query (a lane's: k * 32 +
    // lane) the four of either key tile.
    auto describe = [&](Stage<kWords>& g) {
      const uint32_t ref = p.ref[p.first[un.si] + r];
      const int state = (int)(ref >> kRefStateShift) & 31;
      const uint32_t* base = state == 0 ? p.own_mask : p.hist_mask;
      const bool on[2] = {walk.marked(0, r, qt), walk.marked(1, r, qt)};
      if (kWords && base != nullptr) {
        const size_t query = state == 0 ? (size_t)p.own_words : (size_t)p.hist_states * p.hist_words;
        const int w0 = un.kp * 8;  // first word of the pair of key tiles
        const int words = (p.T + 31) / 32;
        // eight lanes take the eight words of a query, four queries at a time
        const int j = lane & 7, q = lane >> 3;
        const uint32_t* row = base + ((size_t)(ref & 63u) * p.T + qt * kTile + q) * query + w0 + j +
                              (state == 0 ? 0 : (size_t)(state - 1) * p.hist_words);
        const size_t step = 4 * query;
        uint32_t* dst = &g.word[kWords ? j : 0][q];
        if (on[0] && on[1] && w0 + 8 <= words && (qt + 1) * kTile <= p.T) {  // nothing to leave out
#pragma unroll 16
          for (int k = 0; k < kTile / 4; ++k, row += step) cp_async_u32(dst + 4 * k, row);
        } else {
          const bool load = on[j >> 2] && w0 + j < words;
          const int rows = load ? p.T - qt * kTile : 0;
#pragma unroll 8
          for (int k = 0; k < kTile / 4; ++k, row += step) {
            const bool in = q + 4 * k < rows;
            cp_async_u32_if(dst + 4 * k, in ? row : base, in);
          }
        }
      }
      const bool causal = state == 0 && (ref & kRefCausal);
      // rows past T hold +inf, queries that saw nothing -inf
      const bool plain = !kWords && !causal &&
                         __all_sync(0xffffffffu, isfinite(v[0]) && isfinite(v[1]) && isfinite(v[2]) && isfinite(v[3]));
      if (lane == 0)
        g.info = (plain ? kItemPlain : 0u) | (on[0] ? kItemOn : 0u) | (on[1] ? kItemOn << 1 : 0u) | (base != nullptr ? kItemWords : 0u) |
                 (causal ? kItemCausal : 0u) | (uint32_t)qt << kItemTileShift;
      if constexpr (kWords) cp_async_arrive(&g.l_full);
    };
    bool more = load();
    Ring it;
    while (more) {
      Stage<kWords>& g = stage[it.at];
      ok = __all_sync(0xffffffffu, mbar_wait(&g.l_empty, it.phase ^ 1u, &abort_flag, tmo)) != 0;
      if (!ok) break;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        g.nl[k * 32 + lane] = v[k] == -INFINITY ? -INFINITY : v[k] * -1.4426950408889634f;
      if constexpr (kMask) describe(g);
      __syncwarp();
      if (lane == 0) mbar_arrive(&g.l_full);
      it.step();
      more = load();
    }
    if constexpr (kWords) asm volatile("cp.async.wait_all;" ::: "memory");  // no copy outlives the CTA
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
    int n_unit = 0, qs = 0;
    uint32_t q_phase = 0;
    Ring it, other;             // this item; the other group's item that had the S buffer before
    bool reused = false;        // there was one
    int ahead = kt == 1 ? 1 : 2;  // items until then
    int buf = kt;               // S buffer of step 2 * it + kt
    for (int u = u0; ok && u >= 0;) {
      const Unit un = unit_of(p, u);
      Walk<kMask> walk = walk_of(un, n_unit);
      ok = wait(&bars.k_ready[kt], (uint32_t)n_unit & 1u);
      if (!ok) break;
      int r, qt;
      while (walk.next(r, qt)) {
        if (!reused) reused = ahead-- == 0;
        ok = wait(&bars.q_full[qs], q_phase);
        if (ok && reused) {
          ok = wait(&stage[other.at].s_empty[1 - kt], other.phase);
          other.step();
        }
        if (!ok) break;
        tc_fence_after();
        const uint32_t dcol = tbase + C::kColS + (uint32_t)buf * kTile;
        const uint64_t b = dQ + (uint64_t)(qs * (C::kTileBytes >> 4));
#pragma unroll
        for (int x = 0; x < C::kBoxes; ++x)
          mma_ts_kmajor_x4(dcol, kcol + x * 32, b + (uint64_t)(x * (C::kBoxBytes >> 4)), idesc, x > 0 ? 1u : 0u);
        mma_commit_warp(&stage[it.at].s_full[kt]);
        mma_commit_warp(&bars.q_empty[qs]);
        if (++qs == C::kStages) {
          qs = 0;
          q_phase ^= 1u;
        }
        buf = buf == 0 ? 2 : buf - 1;  // two steps on, modulo 3
        it.step();
      }
      if (!ok) break;
      walked(n_unit);
      u = unit_after(u, ++n_unit, ok);
    }
    if (!ok && lane == 0) record_timeout(p, &abort_flag);
  } else {
    // ------------------------------------------------------------ sums
    const int kt = (warp - 4) >> 3;
    const int half = ((warp - 4) >> 2) & 1;  // which 64 queries of a Q tile
    const int q4 = warp & 3;  // TMEM lane quarter this warp may access
    const int row = q4 * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    // bytes of (own, partner's) word that a step of the bits' transposition keeps
    const uint32_t sel16 = lane & 16 ? 0x3276u : 0x5410u, sel8 = lane & 8 ? 0x3715u : 0x6240u;
    const uint64_t sl2x2 = pair(p.scale_log2, p.scale_log2);
    bool ok = true;
    int n_unit = 0, done = 0, buf = kt;
    Ring it;
    // This thread's row of the next unit's K, shared memory -> TMEM.
    auto copy_k = [&]() {
      if (!__all_sync(0xffffffffu, mbar_wait(&bars.k_full, (uint32_t)n_unit & 1u, &abort_flag, tmo))) return false;
      const uint32_t at = smem_u32(smem + C::kOffK + kt * C::kTileBytes) + (uint32_t)(row * 128);
#pragma unroll
      for (int b = 0; b < C::kBoxes; ++b) {
        if (b != half) continue;
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
    ok = copy_k();
    for (int u = u0; ok && u >= 0;) {
      const Unit un = unit_of(p, u);
      const int key = (un.kp * 2 + kt) * kTile + row;
      const size_t at = ((size_t)p.slot[un.si] * p.H + un.h) * p.T + key;
      const bool mine = key < p.T;
      const bool has_keys = key - lane < p.T;  // the warp's part of the tile (K is not loaded past the slot)
      const float before = ld_f32_if(p.prev + at, p.prev != nullptr && mine && ns == 1, 0.0f);
      float total = 0.0f;
      int left = walk_of(un, done).count();
      walked(done);
      int next = kMask ? -1 : unit_after(u, done + 1, ok);
      // The unit's last S is complete, or it has none (masks only): no MMA reads its K any
      // more, and the next unit's follows.
      auto next_k = [&]() {
        if constexpr (kMask) next = unit_after(u, done + 1, ok);
        if (next >= 0) ok = copy_k();
        return ok;
      };
      if (left == 0 && !next_k()) break;
      const int first_query = key / p.frame_tokens * p.frame_tokens;  // that sees this key under frame causality
      while (left > 0) {
        Stage<kWords>& g = stage[it.at];
        // both normally tested in one round trip
        const bool lok = mbar_try_wait(&g.l_full, it.phase);
        const bool sok = mbar_try_wait(&g.s_full[kt], it.phase);
        if (!__all_sync(0xffffffffu, lok && sok)) {
          ok = __all_sync(0xffffffffu, mbar_wait(&g.l_full, it.phase, &abort_flag, tmo) &&
                                           mbar_wait(&g.s_full[kt], it.phase, &abort_flag, tmo));
          if (!ok) break;
        }
        tc_fence_after();
        --left;
        if (left == 0 && !next_k()) break;
        uint64_t acc[4] = {0, 0, 0, 0};
        // The 16 queries from half * 64 + c * 16 on; with masks those whose bit is set (a
        // test and an addition each: hiding the scores before the exponential instead is two
        // operations of the integer unit a score, and 5 to 7% slower).
        auto add = [&](const uint32_t (&s)[16], int c, bool some, uint32_t bits) {
          const ulonglong2* nl2 = reinterpret_cast<const ulonglong2*>(&g.nl[half * 64 + c * 16]);
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const ulonglong2 n = nl2[e >> 2];
            float x0, x1, x2, x3;
            fma2(x0, x1, __uint_as_float(s[e]), __uint_as_float(s[e + 1]), sl2x2, n.x);
            fma2(x2, x3, __uint_as_float(s[e + 2]), __uint_as_float(s[e + 3]), sl2x2, n.y);
            if (some) {
              float a0, a1, b0, b1;
              unpair(acc[(e >> 1) & 3], a0, a1);
              unpair(acc[((e >> 1) + 1) & 3], b0, b1);
              x0 = ex2(x0);
              x1 = ex2(x1);
              x2 = ex2(x2);
              x3 = ex2(x3);
              if ((bits >> e) & 1u) a0 += x0;
              if ((bits >> (e + 1)) & 1u) a1 += x1;
              if ((bits >> (e + 2)) & 1u) b0 += x2;
              if ((bits >> (e + 3)) & 1u) b1 += x3;
              acc[(e >> 1) & 3] = pair(a0, a1);
              acc[((e >> 1) + 1) & 3] = pair(b0, b1);
            } else {
              acc[(e >> 1) & 3] = add2(acc[(e >> 1) & 3], pair(ex2(x0), ex2(x1)));
              acc[((e >> 1) + 1) & 3] = add2(acc[((e >> 1) + 1) & 3], pair(ex2(x2), ex2(x3)));
            }
          }
        };
        uint32_t s0[16], s1[16];
        const uint32_t scol = tbase + lane_off + C::kColS + (uint32_t)(buf * kTile + half * 64);
        const uint32_t info = kMask ? g.info : 0u;
        // (with token words that test costs the others 3 to 7%)
        const uint32_t plain = kItemPlain | kItemOn << kt;
        if (!kMask || (!kWords && (info & plain) == plain)) {
          // a warp without keys adds what it finds: a test here costs all others 3 to 8%
          tmem_ld16(scol, s0);
          tmem_wait_ld16(s0);
          tmem_ld16(scol + 16, s1);
          add(s0, 0, false, 0u);
          tmem_wait_ld16(s1);
          tmem_ld16(scol + 32, s0);
          add(s1, 1, false, 0u);
          tmem_wait_ld16(s0);
          tmem_ld16(scol + 48, s1);
          add(s0, 2, false, 0u);
          tmem_wait_ld16(s1);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&g.s_empty[kt]);
          add(s1, 3, false, 0u);
        } else {
          const bool worded = kWords && (info & kItemWords), causal = info & kItemCausal;
          const int q0 = (int)(info >> kItemTileShift) * kTile + half * 64;  // this warp's first query
          if (has_keys && (info & (kItemOn << kt))) {
            // this warp's 32 keys for query c * 32 + lane; a query past T, or that saw
            // nothing, adds nothing, whatever its row holds
            uint32_t w[2], bits[2];
            bool any[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int q = half * 64 + c * 32 + lane;
              w[c] = worded ? g.word[kWords ? kt * 4 + q4 : 0][kWords ? q : 0] : ~0u;
              if (g.nl[q] == -INFINITY) w[c] = 0u;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              bits[c] = __ballot_sync(0xffffffffu, w[c] != 0u);  // a bit a query, for this lane's key
              any[c] = bits[c] != 0u;
            }
            if (worded && (any[0] || any[1]) && !__all_sync(0xffffffffu, (w[0] & w[1]) == ~0u)) {
              // the 32 x 32 bits transposed: halves, bytes, then four, two and one of them
#pragma unroll
              for (int c = 0; c < 2; ++c) bits[c] = __byte_perm(w[c], __shfl_xor_sync(0xffffffffu, w[c], 16), sel16);
#pragma unroll
              for (int c = 0; c < 2; ++c) bits[c] = __byte_perm(bits[c], __shfl_xor_sync(0xffffffffu, bits[c], 8), sel8);
#pragma unroll
              for (int j = 4; j > 0; j >>= 1) {
                const uint32_t m = j == 4 ? 0x0F0F0F0Fu : j == 2 ? 0x33333333u : 0x55555555u;
                const uint32_t keep = (lane & j) ? ~m : m;
                const int turn = (lane & j) ? 32 - j : j;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const uint32_t y = __shfl_xor_sync(0xffffffffu, bits[c], j);
                  bits[c] = (bits[c] & keep) | (__funnelshift_l(y, y, turn) & ~keep);
                }
              }
            }
            if (causal) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const int hidden = first_query - (q0 + c * 32);  // queries ahead of the key's frame
                if (hidden > 0) bits[c] = hidden < 32 ? bits[c] & (~0u << hidden) : 0u;
                any[c] = __any_sync(0xffffffffu, bits[c] != 0u);
              }
            }
            if (any[0] && any[1]) {
              // no sum is kept for the keys past the slot's end
              if (__all_sync(0xffffffffu, (bits[0] & bits[1]) == ~0u || !mine)) {
                tmem_ld16(scol, s0);
                tmem_wait_ld16(s0);
                tmem_ld16(scol + 16, s1);
                add(s0, 0, false, 0u);
                tmem_wait_ld16(s1);
                tmem_ld16(scol + 32, s0);
                add(s1, 1, false, 0u);
                tmem_wait_ld16(s0);
                tmem_ld16(scol + 48, s1);
                add(s0, 2, false, 0u);
                tmem_wait_ld16(s1);
                add(s1, 3, false, 0u);
              } else {
                tmem_ld16(scol, s0);
                tmem_wait_ld16(s0);
                tmem_ld16(scol + 16, s1);
                add(s0, 0, true, bits[0]);
                tmem_wait_ld16(s1);
                tmem_ld16(scol + 32, s0);
                add(s1, 1, true, bits[0] >> 16);
                tmem_wait_ld16(s0);
                tmem_ld16(scol + 48, s1);
                add(s0, 2, true, bits[1]);
                tmem_wait_ld16(s1);
                add(s1, 3, true, bits[1] >> 16);
              }
            } else if (any[0] || any[1]) {
              const int c = any[0] ? 0 : 1;
              const uint32_t col = scol + (uint32_t)(c * 32), some = any[0] ? bits[0] : bits[1];
              tmem_ld16(col, s0);
              tmem_wait_ld16(s0);
              tmem_ld16(col + 16, s1);
              add(s0, 2 * c, true, some);
              tmem_wait_ld16(s1);
              add(s1, 2 * c + 1, true, some >> 16);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&g.s_empty[kt]);
        }
        const uint64_t a = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
        float lo, hi;
        unpair(a, lo, hi);
        total += lo + hi;
        __syncwarp();
        if (lane == 0) mbar_arrive(&g.l_empty);
        buf = buf == 0 ? 2 : buf - 1;  // two steps on, modulo 3
        it.step();
      }
      if (!ok) break;
      // the second half's sums to the first
      if (half == 1) {
        ok = __all_sync(0xffffffffu, mbar_wait(&bars.t_empty[kt], ((uint32_t)done & 1u) ^ 1u, &abort_flag, tmo));
        if (!ok) break;
        half_sum[kt][row] = total;
        mbar_arrive(&bars.t_full[kt]);
      } else {
        ok = __all_sync(0xffffffffu, mbar_wait(&bars.t_full[kt], (uint32_t)done & 1u, &abort_flag, tmo));
        if (!ok) break;
        total += half_sum[kt][row];
        mbar_arrive(&bars.t_empty[kt]);
        if (ns == 1) {
          if (mine) p.out[at] = __fmaf_rn(p.decay, before, total);
        } else {
          st_cluster_f32(mapa_shared(smem_u32(&part[rank][kt * kTile + row]), 0), total);
          __syncwarp();
        }
      }
      ++done;
      u = next;
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
    if (rank == 0 && warp >= 4 && warp < 12 && part_lost == 0.0f) {
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
  // The commits that free the last Q stages have arrived before the CTA leaves.
  if (warp == 0 && lane == 0)
    for (int i = (q_issued > C::kStages ? q_issued - C::kStages : 0); !abort_flag && i < q_issued; ++i)
      mbar_wait(&bars.q_empty[i % C::kStages], (uint32_t)(i / C::kStages) & 1u, &abort_flag, tmo);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (abort_flag) {
    // Some wait expired: wait (bounded, ignoring the abort flag) for the copies
    // and MMAs that this CTA still has in flight.
    const int zero = 0;
    if (warp == 0 && lane == 0) {
      if (k_issued > 0) mbar_wait(&bars.k_full, (uint32_t)(k_issued - 1) & 1u, &zero, tmo);
      for (int i = (q_issued > C::kStages ? q_issued - C::kStages : 0); i < q_issued; ++i) {
        if (p.fault_mode == 2 && i == 1) continue;  // the copy the test hook withheld
        mbar_wait(&bars.q_full[i % C::kStages], (uint32_t)(i / C::kStages) & 1u, &zero, tmo);
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

template <int D, Masks kMasks>
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
      e = cudaFuncSetAttribute(weights_kernel<D, kMasks>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               Cfg<D>::kSmemBytes);
      if (e != cudaSuccess) return e;
      configured[dev] = true;
    }
  }
  LaunchConfig l(dim3((unsigned)grid), kThreads, Cfg<D>::kSmemBytes, s, p.n_split > 1 ? p.n_split : 0);
  return cudaLaunchKernelEx(&l.cfg, weights_kernel<D, kMasks>, p);
}

}  // namespace

cudaError_t launch_weights(const WeightParams& p, int head_dim, int grid, cudaStream_t s) {
  const bool words = p.own_mask != nullptr || p.hist_mask != nullptr;
  if (head_dim == 128)
    return words      ? launch<128, Masks::kWords>(p, grid, s)
           : p.masked ? launch<128, Masks::kTiles>(p, grid, s)
                      : launch<128, Masks::kNone>(p, grid, s);
  if (head_dim == 64)
    return words      ? launch<64, Masks::kWords>(p, grid, s)
           : p.masked ? launch<64, Masks::kTiles>(p, grid, s)
                      : launch<64, Masks::kNone>(p, grid, s);
  return cudaErrorInvalidValue;
}

}  // namespace sva
