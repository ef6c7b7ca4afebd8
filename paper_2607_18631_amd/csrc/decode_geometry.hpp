// Geometry of the few-token layer's products (decode.hip): who takes which features, and what lies in LDS.  Plain host
// code but for the constants and sizes that the kernels share, so that a test can evaluate the rules without a GPU.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

#ifndef MOE_HOST_DEVICE
#ifdef __HIPCC__
#define MOE_HOST_DEVICE __host__ __device__
#else
#define MOE_HOST_DEVICE
#endif
#endif

namespace moe {

constexpr int kDecodeWaves = 4;                              // of a workgroup
constexpr int kDecodeRedBytes = kDecodeWaves * 2 * 64 * 16;  // the sums of the parts of K at most
constexpr int kDecodeMostLds = 158 * 1024;
// values of K whose loads a wave issues together
MOE_HOST_DEVICE constexpr int decode_unit(bool mx) { return mx ? 256 : 128; }

// One launch's geometry: `split` waves share the same 16 features (each takes every split-th unit of K), so a
// workgroup owns 16 * kDecodeWaves / split features; `room` bytes of LDS hold rows, of `lds` in all.
struct DecodeGeometry {
  int32_t tiles, shared_tiles;     // workgroups per entry of the plan, per 16 tokens of the shared expert
  int32_t shared;                  // workgroups of the shared expert
  int32_t split, shared_split, room, lds;
};
MOE_HOST_DEVICE constexpr int features_of(int split) { return 16 * kDecodeWaves / split; }
// bytes between rows of K values in LDS: 16 past the row, so that the four rows and four q's that a read touches at
// once lie in different banks
MOE_HOST_DEVICE constexpr int row_bytes(int K) { return 2 * K + 16; }

struct DecodeSizes {
  int T, E, E_local, top_k;
  bool shared;                     // there is a shared expert
};

// experts that have rows when every token chooses at random
inline double expected_active(const DecodeSizes& s) {
  const double none = std::pow(1.0 - (double)s.top_k / s.E, s.T);
  return std::max(1.0, s.E_local * (1.0 - none));
}

// `features` x K weights of each expert, ns streams of them (`features_s` x K_s of the shared expert)
inline DecodeGeometry decode_geometry(const DecodeSizes& s, int features, int K, int features_s, int K_s, int ns, bool mx) {
  DecodeGeometry g{};
  auto tiles = [](int features, int split) { return (features + features_of(split) - 1) / features_of(split); };
  // Waves on the same features: fewer where there are many workgroups (rows staged once serve more weights), more
  // where there are few.  `waves`: of 16 features each, one wave on them.  The up-projection's, which stream two rows of
  // weights, are shared out longer than the down-projection's.  Measured in us a call, for 1 / 2 / 4 waves, weights from memory:
  //   up    128 waves (1 token, 48 of 384 experts of 7168 x 2048 in 4 bits) 36.4 / 29.8 / 27.0; 384 (1 token, 128 of 2048 x 768)
  //         bf16 36.7 / 29.9 / 32.3, 4 bits 24.2 / 22.9 / 23.4; 952 (8 tokens of the first) 66 / 60 / 63; 4900 (4 tokens, 8 of
  //         4096 x 14336) 105 / 101 / 101, in bf16 415 / 385 / 364; 6045 (64 tokens of the second) in bf16 253 / 240 / 244;
  //         7168 (64 tokens, 8 of 4096 x 14336) 250 / 278 / 338, in bf16 679 / 698 / 699
  //   down  512 (1 token, 8 of 4096 x 14336) 54 / 46.5 / 45.5; 1024 23.3 / 23.3 / 24.2; 1400 105 / 101 / 101; 3333 58 / 62 / 71;
  //         6607 49 / 52 / 60; 10541 128 / 132 / 153; 16121 102 / 119 / 153
  // The shared expert's rows are all the tokens; its workgroups come first.  2 waves: 4 of 2048 x 2816 in 4 bits with 1
  // token 25.0 / 22.6 / 22.6, 64 tokens 119 / 123 / 130; 7168 x 2048 with 8 tokens 74 / 62 / 63, 64 tokens 208 / 217 / 237.
  const double waves = expected_active(s) * ((features + 15) / 16);
  g.split = waves >= (ns == 2 ? 7000 : 3000) ? 1 : waves >= (ns == 2 ? 256 : 768) ? 2 : 4;
  g.shared_split = 2;
  g.tiles = tiles(features, g.split);
  g.shared_tiles = std::max(1, tiles(features_s, g.shared_split));
  g.shared = s.shared ? g.shared_tiles * ((s.T + 15) / 16) : 0;
  // LDS: scales, and rows: room for all of an expert's rows where that leaves four workgroups per compute unit, else
  // as much as leaves two.  A round of the most rows has to fit.  (38 KB / 76 KB where the mean is above 1.25 rows: long rows
  // gain from 76, 16 of 14336 values each in the down-projection 307 / 278 us a call, 16 tokens through a shared expert of
  // 7168 x 2048 and 32 of 256 experts 107 / 91; short ones lose, 4 rows of 2048 in the up-projection 91 / 102, 2 of 2048 in the
  // down-projection 204 / 218.  At 1.0 to 1.1 rows they are the same but for rows of 7168, 62 / 60.)
  const int widest = std::max(K, s.shared ? K_s : 0), split = std::max(g.split, g.shared_split);
  const int64_t fixed = mx ? (int64_t)ns * std::max(features_of(g.split), features_of(g.shared_split)) * (widest / 32) : 0;
  const double rows = (double)s.T * s.top_k / s.E * s.E_local / expected_active(s);
  const int most = std::min(s.T, 16);
  const int64_t least = (int64_t)most * row_bytes(std::min(split * decode_unit(mx), widest));
  const int64_t all = (int64_t)most * row_bytes((widest + split * 256 - 1) / (split * 256) * (split * 256));
  const int64_t room = std::max(least, (rows > 1.25 ? 76 : 38) * 1024 - fixed);
  g.room = (int)std::min(room, std::max(all, least));
  g.lds = (int)std::max<int64_t>(kDecodeRedBytes, g.room + fixed);
  return g;
}

}  // namespace moe
