// RMSNorm of each head's key (and query), 3D RoPE and the KV-cache write in one
// pass (sva_rope_kv_write_headnorm).  Per token u and head h, over the d
// elements x of one row:
//   y = x * gamma / sqrt(mean(x^2) + eps),
//   (y[2p], y[2p+1]) turned by the angle of pair p at the token's (t, h, w),
// in fp32 with one bf16 rounding; V is copied.  Other than the norm over the
// whole H*d vector, a row's sum of squares stays inside d / 8 lanes, so no warp
// waits for another and a token's heads can be spread over as many warps as a
// launch needs to fill the GPU.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"
#include "rope_head.h"

namespace sva {
namespace {

__device__ __forceinline__ uint4 ld_row(const __nv_bfloat16* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

struct Gamma8 {
  float g[8];
};
__device__ __forceinline__ Gamma8 gamma_at(const float* gamma) {
  const float4 a = ptx::ld_global_f4(gamma), b = ptx::ld_global_f4(gamma + 4);
  return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// One vector of a row: normalised by the sum over the `lanes` lanes that hold
// the row, times gamma, turned.
template <bool kGamma>
__device__ __forceinline__ uint4 norm_turn(uint4 v, const Gamma8& g, const float2 (&cs)[4], int lanes, float inv_d,
                                           float eps) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float x[8], sum = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(w[k] << 16);
    x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    sum = __fmaf_rn(x[2 * k], x[2 * k], sum);
    sum = __fmaf_rn(x[2 * k + 1], x[2 * k + 1], sum);
  }
  sum += __shfl_xor_sync(0xffffffffu, sum, 1);
  sum += __shfl_xor_sync(0xffffffffu, sum, 2);
  sum += __shfl_xor_sync(0xffffffffu, sum, 4);
  if (lanes == 16) sum += __shfl_xor_sync(0xffffffffu, sum, 8);
  const float r = __frsqrt_rn(__fmaf_rn(sum, inv_d, eps));
  uint32_t o[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = x[2 * k] * (kGamma ? g.g[2 * k] * r : r);
    const float b = x[2 * k + 1] * (kGamma ? g.g[2 * k + 1] * r : r);
    const __nv_bfloat162 t = __floats2bfloat162_rn(__fmaf_rn(a, cs[k].x, -(b * cs[k].y)), __fmaf_rn(a, cs[k].y, b * cs[k].x));
    o[k] = *reinterpret_cast<const uint32_t*>(&t);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A warp takes parts of tokens: p.group lanes (all 32, or fewer where a token's
// heads have fewer vectors) walk kBatch vectors each of one token's rows, `group`
// apart, all their loads issued before the first store.  `group` is a multiple of
// the d / 8 vectors of a row, so a lane holds the same four pairs in every vector.
//
// Bound by HBM.  Four blocks of eight warps an SM with two vectors a lane keep 98 KB
// of loads in flight an SM; held to 64 registers, so a row's gammas are fetched where
// they are used (from L1), K's before Q's: with both at hand the instances with Q
// spill (18720 tokens of 12 x 128 with Q, gammas a head 61.4 us, 57.0 so; 4680 of 40
// x 128 52.0 and 48.2).  Three vectors at three blocks: 58.1 and 50.0.  The grid is
// at most eight blocks an SM: a block that loops has its gammas and tables in L1 (4680
// tokens of 12 x 128, K and V, 12.3 us, 13.0 at sixteen, 13.0 with a block a part).
// Times with three sets of buffers in a graph: one 4680-token node of 12 x 128 with Q
// 17.3 us (86 MB, 5.0 TB/s; a device copy of its 43 MB takes 20.5 us in such a loop),
// four 57.0 us (6.1 TB/s), K and V of 40 x 128 32.9 us (5.8 TB/s).
template <int kBatch, bool kQ, bool kGamma>
__global__ void __launch_bounds__(256, 4) rope_head_kernel(const __grid_constant__ RopeHeadParams p) {
  const int lane = threadIdx.x & 31;
  const int vpr = p.d >> 3;                      // 16-byte vectors of a row
  const int vshift = vpr == 16 ? 4 : 3;
  const int c8 = lane & (vpr - 1);
  const int per_tok = p.H * vpr;
  const int in_group = lane & (p.group - 1);
  const int step = p.group * kBatch;             // vectors of a part
  const int HpWp = p.Hp * p.Wp;
  const float inv_d = 1.0f / (float)p.d;
  const size_t kv_stride = (size_t)p.H * p.Tpad * p.d;  // elements between K and V of a slot
  const __nv_bfloat16* kin = static_cast<const __nv_bfloat16*>(p.k);
  const __nv_bfloat16* vin = static_cast<const __nv_bfloat16*>(p.v);
  const __nv_bfloat16* qin = static_cast<const __nv_bfloat16*>(p.q);
  __nv_bfloat16* qout = static_cast<__nv_bfloat16*>(p.q_out);
  __nv_bfloat16* cache = static_cast<__nv_bfloat16*>(p.cache);
  ptx::pdl_wait();
  const int per_warp = 32 / p.group;
  const int units = (p.n_nodes * p.T * p.parts + per_warp - 1) / per_warp;  // of a warp
  const int warps = gridDim.x * (blockDim.x >> 5);
  for (int unit = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); unit < units; unit += warps) {
    const int part_of_all = unit * per_warp + lane / p.group;
    const int tok_all = part_of_all / p.parts;
    const bool live = tok_all < p.n_nodes * p.T;  // the last warp may have groups to spare
    const int tok = live ? tok_all : 0;
    const int v0 = live ? (part_of_all - tok * p.parts) * step + in_group : per_tok;
    uint4 kv[kBatch], vv[kBatch], qv[kQ ? kBatch : 1];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int v = v0 + j * p.group;
      kv[j] = make_uint4(0, 0, 0, 0);
      vv[j] = kv[j];
      if constexpr (kQ) qv[j] = kv[j];
      if (v < per_tok) {
        kv[j] = ld_row(kin + tok * p.k_stride + v * 8);
        vv[j] = ld_row(vin + tok * p.v_stride + v * 8);
        if constexpr (kQ) qv[j] = ld_row(qin + tok * p.q_stride + v * 8);
      }
    }
    const int node = tok / p.T;
    const int u = tok - node * p.T;
    const int f = u / HpWp;
    const int hw = u - f * HpWp;
    const int hh = hw / p.Wp;
    const int ww = hw - hh * p.Wp;
    const RopeNode nd = p.nodes[node];
    const int tpos = nd.t_base + f;
    float2 cs[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int pi = c8 * 4 + k;  // pair index within the head dimension
      if (pi < p.P0)
        cs[k] = __ldg(p.tab_t + (size_t)tpos * p.P0 + pi);
      else if (pi < p.P0 + p.P1)
        cs[k] = __ldg(p.tab_h + (size_t)hh * p.P1 + (pi - p.P0));
      else
        cs[k] = __ldg(p.tab_w + (size_t)ww * p.P2 + (pi - p.P0 - p.P1));
    }
    __nv_bfloat16* out = cache + ((size_t)nd.slot * 2 * p.H * p.Tpad + u) * p.d + c8 * 8;  // (slot, K, head 0, u)
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int v = v0 + j * p.group;
      const bool in = v < per_tok;
      const int gv = p.gamma_heads > 1 ? v * 8 : c8 * 8;
      Gamma8 g{};
      if (kGamma && in) g = gamma_at(p.gamma_k + gv);
      // the shuffles inside want every lane, in range or not
      const uint4 k = norm_turn<kGamma>(kv[j], g, cs, vpr, inv_d, p.eps);
      uint4 q{};
      if constexpr (kQ) {
        if (kGamma && in) g = gamma_at(p.gamma_q + gv);
        q = norm_turn<kGamma>(qv[j], g, cs, vpr, inv_d, p.eps);
      }
      if (in) {
        __nv_bfloat16* dst = out + (size_t)(v >> vshift) * p.Tpad * p.d;
        *reinterpret_cast<uint4*>(dst) = k;
        *reinterpret_cast<uint4*>(dst + kv_stride) = vv[j];
        if constexpr (kQ) *reinterpret_cast<uint4*>(qout + ((size_t)tok * per_tok + v) * 8) = q;
      }
    }
  }
}

template <int kBatch>
cudaError_t launch_batch(RopeHeadParams& p, int num_sms, cudaStream_t s) {
  const int per_tok = p.H * (p.d >> 3);
  p.parts = (per_tok + p.group * kBatch - 1) / (p.group * kBatch);
  const long long units = ((long long)p.n_nodes * p.T * p.parts * p.group + 31) / 32;
  const long long blocks = std::min((units + 7) / 8, 8ll * num_sms);
  LaunchConfig l(dim3((unsigned)blocks), 256, 0, s);
  if (p.gamma_k != nullptr)
    return p.q != nullptr ? cudaLaunchKernelEx(&l.cfg, rope_head_kernel<kBatch, true, true>, p)
                          : cudaLaunchKernelEx(&l.cfg, rope_head_kernel<kBatch, false, true>, p);
  return p.q != nullptr ? cudaLaunchKernelEx(&l.cfg, rope_head_kernel<kBatch, true, false>, p)
                        : cudaLaunchKernelEx(&l.cfg, rope_head_kernel<kBatch, false, false>, p);
}

}  // namespace

cudaError_t launch_rope_head(RopeHeadParams& p, int num_sms, cudaStream_t s) {
  const int per_tok = p.H * (p.d >> 3);
  p.group = per_tok >= 32 ? 32 : (per_tok >= 16 ? 16 : 8);
  // A launch that leaves half of the warps idle is as long as one part takes: 320
  // tokens of 12 x 128 with Q 3.2 us at two vectors a lane, 2.8 at one.  Past that
  // two are faster (4680 tokens 17.3 us, 19.4 at one).
  const long long rows = ((long long)p.n_nodes * p.T * per_tok + 31) / 32;
  return rows <= 16ll * num_sms ? launch_batch<1>(p, num_sms, s) : launch_batch<2>(p, num_sms, s);
}

}  // namespace sva
