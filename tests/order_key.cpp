// The gate's key images as a C library for test_gate_keys.py.
#include "order_key.hpp"

extern "C" {
void images(const uint32_t* bits, uint32_t* image, uint32_t* back, long n) {
  for (long i = 0; i < n; ++i) {
    image[i] = moe::ordered(__builtin_bit_cast(float, bits[i]));
    back[i] = __builtin_bit_cast(uint32_t, moe::unordered(image[i]));
  }
}
}
