// Slots to packed slots and back (sva_cache_pack, sva_cache_unpack; the layout is in
// packed.h).  For a group of 32 elements x of one token's K or V row of a head:
//   a = max |x|,   s = a / 7 rounded to 5 significant bits, halves up,
//   code = x / s to the nearest whole number, halves away from zero:  -7..7,
// as s is at most 2^-5 of it below a / 7.  a < 2^-120: s = 0 and zeros; a >= 2^124, an
// infinity or NaN: s = NaN, all of the group reads as NaN.
//
// Division by s is a multiplication: x and s are numbers of 8 and 5 bits, so x / s is
// either half-way between two whole numbers or further from that than 2^-12 of itself,
// and 1 / s a little too large (by 2^-20) takes the halves away from zero and moves
// nothing else across.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "packed.cuh"

namespace sva {
namespace {

constexpr int kPackThreads = 256;
constexpr uint32_t kZeroCodes = 0x44444444u;  // eight codes of 0: 8 in each four bits, turned by 3

struct Words16 {
  uint32_t w[16];
};

// 64 bytes of a bf16 row (32-byte aligned), as two loads.
__device__ __forceinline__ Words16 ld_group(const uint8_t* p) {
  Words16 r;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.w[8 * k]), "=r"(r.w[8 * k + 1]), "=r"(r.w[8 * k + 2]), "=r"(r.w[8 * k + 3]),
                   "=r"(r.w[8 * k + 4]), "=r"(r.w[8 * k + 5]), "=r"(r.w[8 * k + 6]), "=r"(r.w[8 * k + 7])
                 : "l"(p + 32 * k));
  return r;
}

__device__ __forceinline__ void st_half_group(uint8_t* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z),
               "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
               : "memory");
}

// Scale of a group and the bits of its largest magnitude (a bf16 number's without the
// sign, which order as the magnitudes do, infinity and NaN above the rest).
__device__ __forceinline__ float scale_of(uint32_t a) {
  const float m = __uint_as_float(a << 16);
  const uint32_t b = __float_as_uint(__fdiv_rn(m, 7.0f)) + (1u << 18);  // half of the fifth bit's place
  const float s = __uint_as_float(b & ~((1u << 19) - 1u));
  return a >= 0x7D80u ? __uint_as_float(0x7FC00000u) : (a < 0x0380u ? 0.0f : s);  // 2^124, 2^-120
}

// Where a thread's (token, group) of a state lies.
template <int D>
struct Place {
  static constexpr int G = D / kPackGroup;
  static constexpr int kRows = kPackThreads / G;  // tokens of a block, all of one tile
  int plane, token, group;                        // plane: K or V and head
  __device__ __forceinline__ Place(int Tpad) {
    const int per_plane = Tpad / kRows;
    plane = (int)blockIdx.x / per_plane;
    token = ((int)blockIdx.x - plane * per_plane) * kRows + (int)threadIdx.x / G;
    group = (int)threadIdx.x & (G - 1);
  }
  __device__ __forceinline__ uint8_t* row(const PackParams& p, int slot) const {
    return static_cast<uint8_t*>(p.pool) +
           (((size_t)slot * 2 * p.H + plane) * p.Tpad + token) * (D * 2) + group * (kPackGroup * 2);
  }
  __device__ __forceinline__ uint8_t* tile(const PackParams& p, int number) const {
    return p.packed + (((size_t)number * 2 * p.H + plane) * (p.Tpad / kTile) + token / kTile) * kPackTileBytes<D>;
  }
  __device__ __forceinline__ int codes_at() const { return (group * kTile + token % kTile) * 16; }
  __device__ __forceinline__ int scale_at() const { return G * kTile * 16 + (token % kTile * G + group) * 2; }
};

template <int D>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const __grid_constant__ PackParams p) {
  const Place<D> at(p.Tpad);
  ptx::pdl_wait();
  uint8_t* tile = at.tile(p, p.number[blockIdx.y]);
  uint32_t codes[4] = {kZeroCodes, kZeroCodes, kZeroCodes, kZeroCodes};
  uint32_t scale = 0;
  if (at.token < p.T) {
    const Words16 x = ld_group(at.row(p, p.slot[blockIdx.y]));
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = __vmaxu2(m, x.w[k] & 0x7FFF7FFFu);
    const float s = scale_of(max(m & 0xFFFFu, m >> 16));
    scale = __float_as_uint(s) >> 16;
    const float inv = s > 0.0f ? __fdiv_rn(1.0f, s) * (1.0f + 0x1p-20f) : 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        const uint32_t v = x.w[4 * k + j];
        // code + 8 in the low bits of the sum's mantissa
        const float lo = __fmaf_rn(__uint_as_float(v << 16), inv, 0x1p23f + 8.0f);
        const float hi = __fmaf_rn(__uint_as_float(v & 0xFFFF0000u), inv, 0x1p23f + 8.0f);
        w = (w << 4) + __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
      }
      codes[k] = s > 0.0f ? __funnelshift_l(w, w, 3) : kZeroCodes;
    }
  }
  *reinterpret_cast<uint4*>(tile + at.codes_at()) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
  *reinterpret_cast<uint16_t*>(tile + at.scale_at()) = (uint16_t)scale;
}

template <int D>
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const __grid_constant__ PackParams p) {
  const Place<D> at(p.Tpad);
  ptx::pdl_wait();
  if (at.token >= p.T && p.pad == 0) return;  // (a packed slot holds zeros there)
  const uint8_t* tile = at.tile(p, p.number[blockIdx.y]);
  uint32_t c[4];
  uint16_t s;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3])
               : "l"(tile + at.codes_at()));
  asm volatile("ld.global.u16 %0, [%1];" : "=h"(s) : "l"(tile + at.scale_at()));
  const uint32_t scale = (uint32_t)s * 0x10001u;
  uint8_t* row = at.row(p, p.slot[blockIdx.y]);
#pragma unroll
  for (int k = 0; k < 2; ++k)
    st_half_group(row + 32 * k, packed_values(c[2 * k], scale), packed_values(c[2 * k + 1], scale));
}

template <int D>
cudaError_t launch(const PackParams& p, bool pack, cudaStream_t s) {
  LaunchConfig l(dim3((unsigned)(2 * p.H * (p.Tpad / Place<D>::kRows)), (unsigned)p.n), kPackThreads, 0, s);
  return cudaLaunchKernelEx(&l.cfg, pack ? pack_kernel<D> : unpack_kernel<D>, p);
}

}  // namespace

cudaError_t launch_pack(const PackParams& p, int d, cudaStream_t s) {
  return d == 128 ? launch<128>(p, true, s) : launch<64>(p, true, s);
}

cudaError_t launch_unpack(const PackParams& p, int d, cudaStream_t s) {
  return d == 128 ? launch<128>(p, false, s) : launch<64>(p, false, s);
}

}  // namespace sva
