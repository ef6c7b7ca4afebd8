// The gate's float32 keys as unsigned integers of the same order.  Plain code for the device and the host.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define MOE_KEY_FN __host__ __device__ __forceinline__
#else
#define MOE_KEY_FN inline
#endif

namespace moe {

// float -> uint32 >= 1 with the same order (finite values and infinities; -0 counts as +0).  0 is free for "not
// selectable": the NaN of all ones, whose image it would be, takes the 1 of its neighbour.  (Without that a router bias of
// memory filled with 0xff left nothing to select, and every round chose expert 0 again.)
MOE_KEY_FN uint32_t ordered(float f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.0f);
  const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return o > 1u ? o : 1u;
}

// the float key back from its ordered image (inverse of ordered)
MOE_KEY_FN float unordered(uint32_t o) {
  return __builtin_bit_cast(float, (o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

}  // namespace moe
