// The few-token layer's geometry as a C library for test_decode_geometry.py.
#include "decode_geometry.hpp"

extern "C" {
// out: tiles, shared tiles, shared workgroups, split, shared split, room, lds
void geometry(int T, int E, int E_local, int top_k, int features, int K, int features_s, int K_s, int ns, int mx, int* out) {
  const moe::DecodeGeometry g = moe::decode_geometry({T, E, E_local, top_k, features_s > 0}, features, K, features_s, K_s, ns, mx != 0);
  const int v[7] = {g.tiles, g.shared_tiles, g.shared, g.split, g.shared_split, g.room, g.lds};
  for (int i = 0; i < 7; ++i) out[i] = v[i];
}
int most_lds() { return moe::kDecodeMostLds; }
}
