// The tile rules of the block-scaled grouped product as a C library for test_mx_tile_rule.py.
#include "mx_tile_rule.hpp"

extern "C" {
int tile(long cus, long max_rows, long groups, long weight_rows) {
  return (int)moe::mx_tile_rule(cus, max_rows, groups, weight_rows);
}
int slices(int e2m1_rows, int tile_weight_rows, long K) {
  return (int)moe::mx_slices(e2m1_rows != 0, tile_weight_rows, K);
}
}
