// The attention instances that read packed slots (see attend.cuh).
#include "attend.cuh"

namespace sva {

// With a mask of any kind it is the instance for token masks, however long the launch is:
// whether units unpack is the caller's choice alone (the space, sva_attend_nodes_packed).  A
// tile mask alone so pays for token masks there, and its bits are not those of the tile-mask
// instance.  By the units and with a space, 4680 queries of 12 x 128 over three packed states
// and a whole one: half of the history's tiles kept 537 and 340 us (322 with whole states), a
// tenth 249 and 183 (164); 320 queries over four packed states, half kept, 20.2 and 19.7 (16.6).
AttendKernel attend_packed_kernel(int head_dim, bool masked, bool cluster) {
  if (head_dim == 128) {
    if (masked) return cluster ? attend_kernel<128, true, true, true, true> : attend_kernel<128, true, true, false, true>;
    return cluster ? attend_kernel<128, false, false, true, true> : attend_kernel<128, false, false, false, true>;
  }
  if (masked) return cluster ? attend_kernel<64, true, true, true, true> : attend_kernel<64, true, true, false, true>;
  return cluster ? attend_kernel<64, false, false, true, true> : attend_kernel<64, false, false, false, true>;
}

}  // namespace sva
