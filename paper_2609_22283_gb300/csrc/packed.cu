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

// Half a group: 16 elements, 32 bytes.
struct Half {
  uint32_t w[8];
};

__device__ __forceinline__ Half ld_half(const uint8_t* p) {
  Half r;
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]),
                 "=r"(r.w[7])
               : "l"(p));
  return r;
}

__device__ __forceinline__ void st_half(uint8_t* p, const uint4& a, const uint4& b) {
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

// A block takes kTokens tokens of one tile (of plane blockIdx.y, K or V and head, of state
// blockIdx.z), a lane half a group of each of kBatch tokens, so that every load and store
// of a warp covers whole rows and all of a thread's loads are in flight at once.
//
// Bound by HBM: 2.56 bytes an element.  Times with sets of states in turn in a graph: one
// state of 4680 x 12 x 128 (37 MB) packed 7.2 us, unpacked 6.8 (5.1, 5.4 TB/s); six of them
// 32.4 and 33.3 (6.8, 6.6); seven of 40 x 128 (860 MB) 119.3 and 124 (7.2, 6.9); four of 320 x
// 12 x 128 2.5 and 2.4.  A thread with a whole group (two loads or stores 64 bytes apart)
// takes 7.1 us for the one state unpacked; four tokens a thread 6.0, but an attention over
// the states then starts later than it gains (unpacking and attention, four states of 320
// tokens: 19.6 us, 18.0 with two).
template <int D, int kBatch>
struct Part {
  static constexpr int G = D / kPackGroup;
  static constexpr int kLanes = 2 * G;                             // of a token
  static constexpr int kTokens = kPackThreads / kLanes * kBatch;   // of a block
  int first, group, half;  // first token (of the tile) of the thread; the others 32 / kLanes apart
  uint8_t *rows, *tile;    // of the state's plane from the tile's first token on; and the packed tile
  int valid;               // tokens of the tile
  __device__ __forceinline__ explicit Part(const PackParams& p) {
    const int lane = (int)threadIdx.x & 31;
    const int start = (int)blockIdx.x * kTokens, tile_of = start / kTile;
    first = start % kTile + ((int)threadIdx.x >> 5) * (kTokens / (kPackThreads / 32)) + lane / kLanes;
    group = lane / 2 % G;
    half = lane & 1;
    const size_t plane = blockIdx.y;
    rows = static_cast<uint8_t*>(p.pool) +
           (((size_t)p.slot[blockIdx.z] * 2 * p.H + plane) * p.Tpad + (size_t)tile_of * kTile) * (D * 2) +
           (group * 2 + half) * kPackGroup;
    tile = p.packed + (((size_t)p.number[blockIdx.z] * 2 * p.H + plane) * (p.Tpad / kTile) + tile_of) * kPackTileBytes<D>;
    valid = p.T - tile_of * kTile;
  }
  __device__ __forceinline__ int token(int b) const { return first + b * (32 / kLanes); }
  __device__ __forceinline__ uint8_t* row(int b) const { return rows + token(b) * (D * 2); }
  __device__ __forceinline__ uint8_t* codes(int b) const { return tile + (group * kTile + token(b)) * 16 + half * 8; }
  __device__ __forceinline__ uint8_t* scale(int b) const { return tile + G * kTile * 16 + (token(b) * G + group) * 2; }
};

template <int D, int B>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const __grid_constant__ PackParams p) {
  const Part<D, B> at(p);
  Half x[B];
  ptx::pdl_wait();
#pragma unroll
  for (int b = 0; b < B; ++b) {
    x[b] = Half{};
    if (at.token(b) < at.valid) x[b] = ld_half(at.row(b));
  }
#pragma unroll
  for (int b = 0; b < B; ++b) {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = __vmaxu2(m, x[b].w[k] & 0x7FFF7FFFu);
    m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const float s = scale_of(max(m & 0xFFFFu, m >> 16));
    const bool on = s > 0.0f;  // (rows past T are zeros)
    const float inv = on ? __fdiv_rn(1.0f, s) * (1.0f + 0x1p-20f) : 0.0f;
    uint32_t codes[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        const uint32_t v = x[b].w[4 * k + j];
        // code + 8 in the low bits of the sum's mantissa
        const float lo = __fmaf_rn(__uint_as_float(v << 16), inv, 0x1p23f + 8.0f);
        const float hi = __fmaf_rn(__uint_as_float(v & 0xFFFF0000u), inv, 0x1p23f + 8.0f);
        w = (w << 4) + __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
      }
      codes[k] = on ? __funnelshift_l(w, w, 3) : kZeroCodes;
    }
    *reinterpret_cast<uint2*>(at.codes(b)) = make_uint2(codes[0], codes[1]);
    if (at.half == 0) *reinterpret_cast<uint16_t*>(at.scale(b)) = (uint16_t)(__float_as_uint(s) >> 16);
  }
}

template <int D, int B>
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const __grid_constant__ PackParams p) {
  const Part<D, B> at(p);
  const int rows = p.pad != 0 ? kTile : at.valid;  // (a packed slot holds zeros behind the last token)
  uint32_t c[B][2];
  uint16_t s[B];
  ptx::pdl_wait();
#pragma unroll
  for (int b = 0; b < B; ++b) {
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(c[b][0]), "=r"(c[b][1]) : "l"(at.codes(b)));
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(s[b]) : "l"(at.scale(b)));
  }
#pragma unroll
  for (int b = 0; b < B; ++b) {
    const uint32_t scale = (uint32_t)s[b] * 0x10001u;
    if (at.token(b) < rows) st_half(at.row(b), packed_values(c[b][0], scale), packed_values(c[b][1], scale));
  }
}

using PackKernel = void (*)(const PackParams);

template <int D, int B>
cudaError_t launch(PackKernel k, const PackParams& p, cudaStream_t s) {
  LaunchConfig l(dim3((unsigned)(p.Tpad / Part<D, B>::kTokens), 2u * (unsigned)p.H, (unsigned)p.n), kPackThreads, 0, s);
  return cudaLaunchKernelEx(&l.cfg, k, p);
}

}  // namespace

cudaError_t launch_pack(const PackParams& p, int d, cudaStream_t s) {
  return d == 128 ? launch<128, 2>(pack_kernel<128, 2>, p, s) : launch<64, 2>(pack_kernel<64, 2>, p, s);
}

cudaError_t launch_unpack(const PackParams& p, int d, cudaStream_t s) {
  return d == 128 ? launch<128, 2>(unpack_kernel<128, 2>, p, s) : launch<64, 2>(unpack_kernel<64, 2>, p, s);
}

}  // namespace sva
