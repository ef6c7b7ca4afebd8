// Host-only size arithmetic of the kernels' launches and workspaces (no device code): the
// router-logits tile and K split, and the permutation workspace layout.  Kept apart from the
// device sources so the ABI's validation and workspace layer also builds as plain host C++.
#include "kernels.hpp"

namespace moe {

// Router-logits tile: the whole expert row of 256 or more experts in one tile (128 x 256, 8 waves)
// or 128 of them (64 x 128, 4 waves), with K split only as far as needed to reach one workgroup per
// compute unit.  Measured (logits GEMM + gate, token rows read from HBM): DeepSeek-V3 shape
// (8192 x 256 x 7168) 128 x 256 tiles with 4 partials 59.4 us against 69.2 for 256 x 256 tiles with
// 8; skewed shape (16384 x 128 x 2048) 64 x 128 unsplit 37.5 us against 46.6 for 256 x 256 with 4.
// Fewer rows or experts: 64 x 64.
TileShape f32_tile(int64_t rows, int n) {
  if (rows >= 4096 && n >= 256) return {128, 256, 64};
  if (rows >= 4096 && n >= 128) return {64, 128, 64};
  return {64, 64, 64};
}

int logits_splits(int64_t T, int E, int K) {
  constexpr int64_t kTarget = 256;                         // compute units of an MI355X
  constexpr int64_t kMaxSplits = 16;                       // bounds the partials the gate adds
  const TileShape t = f32_tile(T, E);
  const int64_t base = ((T + t.bm - 1) / t.bm) * ((E + t.bn - 1) / t.bn);
  const int64_t nk = (K + t.bk - 1) / t.bk;
  if (base <= 0 || nk <= 1) return 1;
  int64_t s = (kTarget + base - 1) / base;
  s = s < nk ? s : nk;
  s = s < kMaxSplits ? s : kMaxSplits;
  if (s <= 1) return 1;
  const int64_t chunk = (nk + s - 1) / s;
  return (int)((nk + chunk - 1) / chunk);                // every chunk non-empty
}

int64_t permute_supers(int64_t T) {
  constexpr int64_t sc = (int64_t)kPermChunk * kPermSuper;
  return (T + sc - 1) / sc;
}

PermuteWs permute_ws(int64_t T, int E_local) {
  auto al = [](size_t v) { return (v + 255) / 256 * 256; };
  PermuteWs w;
  const size_t table = al((size_t)permute_supers(T) * E_local * sizeof(int32_t));
  const size_t chunks = (size_t)permute_supers(T) * kPermSuper * E_local;
  w.super_count = 0;
  w.super_base = table;
  w.totals = 2 * table;
  w.chunk_mask = w.totals + al((size_t)E_local * sizeof(int32_t));
  w.chunk_base = w.chunk_mask + al(chunks * sizeof(uint64_t));
  w.bytes = w.chunk_base + al(chunks * sizeof(int32_t));
  return w;
}

// Few-token layer: partials of the logits, which the gate adds.  A workgroup's four waves share one; a wave has 256
// values of K at least.  A call with next to no experts, 1 / 2 / 4 / 8 / 16 partials: 1 token, 384 experts of 7168 values
// 17.5 / 14.0 / 12.2 / 12.0 / 14.8 us; 64 tokens 28.6 / 22.8 / 23.8 / 23.9 / 27.9; 64 tokens, 128 of 2048 17.1 / 15.8 / 15.1 / 15.1;
// only rows of 16384 would gain from more (1 token, 64 experts 27.4 / 18.0 / 13.0 / 10.7 / 9.9).  The number of experts has
// no part in it.
int decode_logits_splits(int /*E*/, int d) {
  const int s = (d + 1023) / 1024;
  return s < 4 ? s : 4;
}

// Norm backward: every workgroup leaves one row of partial sums of dgamma.  A workgroup of four waves takes 4 short rows
// at once, or one long row.  Few rows go to one workgroup, which needs no second launch; up to 256 workgroups each has one
// such round; then 16 rows, up to four workgroups per compute unit of an MI355X.  Forward and backward captured in a graph,
// us a step for numbers of workgroups, the rule's marked:
//   7 rows of 640   *1 6.4, 2 7.6                      100 of 7168     7 25.7, 50 12.5, *100 11.9
//   16 of 2048      *1 11.3, 4 9.9                     1000 of 7168    63 37.6, 128 25.9, *256 22.8, 512 23.7
//   17 of 2048      1 12.1, 2 11.9, *5 10.0            8192 of 7168    256 116, *512 103 - 110, 1024 115
//   1000 of 2048    63 16.6, 125 14.8, *250 14.8       16384 of 2048   256 59.0, 512 60.6, *1024 65.8, 2048 75
//   3001 of 2040    188 22.0, *256 19.6, 512 21.0      100000 of 512   512 103, *1024 93.7, 2048 103
int add_norm_bwd_parts(int64_t rows, int d) {
  const bool is_short = d <= 2048;
  if (rows <= (is_short ? 16 : 2)) return 1;
  const int64_t rounds = is_short ? (rows + 3) / 4 : rows, most = rounds < 256 ? rounds : 256, n = (rows + 15) / 16;
  return (int)(n < most ? most : n < 1024 ? n : 1024);
}

}  // namespace moe
