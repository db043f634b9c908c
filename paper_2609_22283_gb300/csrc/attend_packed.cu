// The attention instances that read packed slots (see attend.cuh).
#include "attend.cuh"

namespace sva {

// With a mask of any kind it is the instance for token masks: a launch with masks that is
// long enough to care which has its states unpacked first, into a space, and takes the
// ordinary instances.
AttendKernel attend_packed_kernel(int head_dim, bool masked, bool cluster) {
  if (head_dim == 128) {
    if (masked) return cluster ? attend_kernel<128, true, true, true, true> : attend_kernel<128, true, true, false, true>;
    return cluster ? attend_kernel<128, false, false, true, true> : attend_kernel<128, false, false, false, true>;
  }
  if (masked) return cluster ? attend_kernel<64, true, true, true, true> : attend_kernel<64, true, true, false, true>;
  return cluster ? attend_kernel<64, false, false, true, true> : attend_kernel<64, false, false, false, true>;
}

}  // namespace sva
