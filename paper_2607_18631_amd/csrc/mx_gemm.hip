// Grouped products on block-scaled operands: Y[r, n] = sum_k X[r, k] W_g[n, k], X in e4m3 or e2m1, W in
// e2m1, on v_mfma_scale_f32_32x32x64_f8f6f4 (elements multiplied as they are, each block of 32 products
// times both blocks' powers of two, float32 accumulation).
//
// A workgroup owns BM rows of one group and BN weight rows; its K loop runs over slices of 128 or 256
// values in a ring of LDS stages, filled by direct-to-LDS copies.  Each wave multiplies MT x NT tiles of
// 32 x 32: the weights are the first operand, so that a lane holds 16 of the 32 output features of one
// row, its partner lane (l ^ 32) the others.  A group's last rows run on a tile of 64 or 128 rows.
//
// The matrix cores are not to wait for LDS: a slice is multiplied in parts of 64 values, each part's
// operands being read from LDS between the products of the part before it.  The one barrier of a slice
// stands before its last part.  There the whole slice is in registers, so its stage is free and takes the
// copies of the slice STAGES further on; STAGES - 1 slices are on their way or landed.
//
// What bounds it: with many rows the matrix cores, at the clock that their power leaves, and what shares it with them.
// Bare loops of the instruction on random operands run at 3.4 - 4.0 PFLOP/s (e4m3 rows) and 6.2 - 6.6 (e2m1), a fifth to a
// third below those on zeros.  Here they are busy for 62% and 48% of the cycles, at 1.9 GHz, LDS for 19% and 22%.  8192 rows on 8 experts of
// 4096 x 14336 in e2m1: 0.95 ms a call, 3.1 PFLOP/s; with loads that are whole tiles 0.82, of which 0.18 go if nothing is
// copied, 0.09 more if nothing is read from LDS, and 0.44 are the products of a bare loop; the rest are the 5 us in which a
// tile begins and ends.  8192 rows on 32 of 7168 x 2048 in e4m3: 0.45 ms (0.39, 0.06, 0.04, 0.21).  With few rows it is the
// weights' stream: 512 rows on the 32 experts 0.18 ms, 4.1 TB/s; 501 rows on 8 of 2048 x 1408 24 us, a chain of latencies.
//
// What the sums keep: the instruction adds the products of eight neighbouring values of K aligned to the largest of them,
// whatever the shape; with e4m3 rows (products up to 2688, down to 2^-10) it cuts them 2^-13 below that one's power of two,
// then adds in float32.  Measured on normal rows and weights, K = 64 to 7168: 4e-6 of the sum in the mean, 4e-5 at most;
// e2m1 products are exact.  It is the rate of the matrix cores on 8 bits that buys it: products of bf16 would be exact at
// half of it.  The result's error against 64 bits is 1.76e-3 where float32 sums leave 1.66e-3 (bf16's own rounding).
//
// SwiGLU: two weight tiles of a wave are the gate and the up rows of the same 32 features, so the
// activation and the maximum of its block are formed in registers, and the block leaves as elements and
// one scale.
//
// Operand layout of the instruction (lane l: row l % 32, half q = l / 32): e2m1 holds k = 32 q + j in
// nibble j; e4m3 holds k = 16 q + j in bytes j < 16 and k = 32 + 16 q + (j - 16) in the others; the scale
// given by lane l is that of block q of its row for either.

#include "common.hpp"
#include "gemm_device.hpp"
#include "kernels.hpp"
#include "mx_device.hpp"
#include "mx_tile_rule.hpp"

namespace moe {
namespace {

// a 4-bit operand: 16 bytes of the 32 that the instruction's type has room for
__device__ __forceinline__ i32x8 narrow(u32x4 v) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 w = __builtin_bit_cast(i32x4, v);
  return __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
}

// a slice: KS values of K
template <int FMT, int WM, int WN, int MT, int NT, int MOST_STAGES, int KS>
struct MxTile {
  static constexpr int F = FMT, M_WAVES = WM, N_WAVES = WN, M_TILES = MT, N_TILES = NT;
  static constexpr int WAVES = WM * WN;
  static constexpr int NTH = WAVES * 64;
  static constexpr int BM = WM * MT * 32;
  static constexpr int BN = WN * NT * 32;                     // weight rows
  static constexpr int SLICE = KS, PARTS = KS / 64;           // (a part: what one instruction takes)
  static constexpr int XROW = FMT == MX_E4M3 ? KS : KS / 2;   // bytes of a slice's row
  static constexpr int WROW = KS / 2;
  static constexpr int X_BYTES = BM * XROW;
  static constexpr int W_BYTES = BN * WROW;
  static constexpr int STAGE = X_BYTES + W_BYTES;
  // the scales of 512 values: 16 bytes per row (of X, then of W), two sets of them
  static constexpr int GROUP = 512 / KS;                      // slices
  static constexpr int SROWS = (BM + BN + 63) / 64 * 64;
  static constexpr int FIT = (160 * 1024 - 2 * SROWS * 16) / STAGE;
  static constexpr int STAGES = FIT < MOST_STAGES ? FIT : MOST_STAGES;
  static constexpr int LDS = STAGE * STAGES + 2 * SROWS * 16;
  static constexpr int NX = X_BYTES / 1024, NW = W_BYTES / 1024, NS = SROWS / 64;   // wave copies
  // as many waves and weight rows for a group's last rows, where 64 ROWS64 will do
  template <int ROWS64>
  using Low = MxTile<FMT, 2, 4, ROWS64, 2, MOST_STAGES, KS>;
  static constexpr int LOWS = WAVES == 8 && BN == 256 ? (BM - 1) / 128 + (BM > 64) : 0;
  static_assert(X_BYTES % 1024 == 0 && W_BYTES % 1024 == 0, "whole wave copies");
  static_assert(STAGES >= 2, "a slice on its way beside the one in use");
  static_assert(STAGES <= GROUP + 1, "the scales of slice s + STAGES replace those of two groups before");
  static_assert(PARTS % 2 == 0, "a slice begins in the first of two operand buffers");
};

// 16-byte chunk of a row where the stage holds the row's chunk c: rows that share a bank cycle take
// different chunks, so the 16 lanes of a read pass touch every bank once
template <int ROW>
__device__ __forceinline__ int mx_chunk(int row, int c) {
  constexpr int CPR = ROW / 16, RPG = 16 / CPR;
  return c ^ ((row / RPG) % CPR);
}

// rows row0 .. row0 + rows of group g (1 <= rows <= BM), output features feat0 ..
template <class T, bool SWIGLU, bool WHOLE>
__device__ __forceinline__ void mx_tile(const MxGemmProblem& p, char* smem, int g, int64_t row0, int rows, int feat0) {
  constexpr int FMT = T::F, MT = T::M_TILES, NT = T::N_TILES, STEPS = MT * NT / 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = p.K, N = p.N;

  // ---- where the copies come from ----
  const int KB = K / 32;                                       // blocks of a row
  const int nk = (K + T::SLICE - 1) / T::SLICE;
  const int64_t xbytes = FMT == MX_E4M3 ? K : K / 2, wbytes = K / 2;
  // Each wave's share of a stage: copies wave, wave + WAVES, ... of the token rows and the weights.  A lane's source is
  // a base of the wave's plus `from` bytes, 32 bits wide: the host admits no larger group.
  constexpr int MINE = (T::NX + T::NW + T::WAVES - 1) / T::WAVES, LEAST = (T::NX + T::NW) / T::WAVES;
  constexpr int SMINE = (T::NS + T::WAVES - 1) / T::WAVES;
  uint32_t from[MINE];
  const char* sfrom[SMINE];
  const int64_t wrow0 = (int64_t)g * (SWIGLU ? 2 * (int64_t)N : N);
  // weight row (from the group's first) of the stage's row i: plain, or per wave 32 gate and 32 up rows
  auto weight_row = [&](int i) -> uint32_t {
    if constexpr (SWIGLU) {
      const int f = min(feat0 + (i / 64) * 32 + (i & 31), N - 1);
      return (i & 32) ? N + f : f;
    } else {
      return min(feat0 + i, N - 1);
    }
  };
  const char* xb = (const char*)p.X + row0 * xbytes;
  const char* wb = (const char*)p.W + wrow0 * wbytes;
  const char* xs = (const char*)p.X_scales + row0 * KB;
  const char* ws = (const char*)p.W_scales + wrow0 * KB;
#pragma unroll
  for (int c = 0; c < MINE; ++c) {
    const int id = wave + c * T::WAVES;
    if (id < T::NX) {
      const int byte = id * 1024 + lane * 16, r = byte / T::XROW, ch = mx_chunk<T::XROW>(r, (byte % T::XROW) / 16);
      from[c] = (uint32_t)(min(r, rows - 1) * xbytes) + ch * 16;
    } else {
      const int byte = (min(id, T::NX + T::NW - 1) - T::NX) * 1024 + lane * 16, r = byte / T::WROW;
      const int ch = mx_chunk<T::WROW>(r, (byte % T::WROW) / 16);
      from[c] = (uint32_t)(weight_row(r) * wbytes) + ch * 16;
    }
  }
#pragma unroll
  for (int c = 0; c < SMINE; ++c) {
    const int r = (wave + c * T::WAVES) * 64 + lane;
    sfrom[c] = r < T::BM ? xs + (int64_t)min(r, rows - 1) * KB : ws + (int64_t)weight_row(min(r - T::BM, T::BN - 1)) * KB;
  }
  const char* x_end = (const char*)p.X_scales + p.max_rows * KB;
  const char* w_end = (const char*)p.W_scales + (int64_t)p.groups * (SWIGLU ? 2 * (int64_t)N : N) * KB;
  // the slice's value with which this lane's chunks begin, for all its copies: their chunks repeat every 16 rows
  static_assert(WHOLE || (T::WAVES * 1024 / T::XROW % 16 == 0 && 1024 / T::WROW % 16 == 0), "whole periods between copies");
  auto first_value = [&](bool x) {
    int l = lane;
    asm volatile("" : "+v"(l));                                // found again where it is used: in no register of the loop
    return x ? mx_chunk<T::XROW>((wave * 1024 + l * 16) / T::XROW, l * 16 % T::XROW / 16) * (FMT == MX_E4M3 ? 16 : 32)
             : mx_chunk<T::WROW>(l * 16 / T::WROW, l * 16 % T::WROW / 16) * 32;
  };
  // Scales: a row's 4 bytes of one slice are as many cache accesses and requests as its 64 or 128 bytes of values, so
  // they come for a group of slices at a time: 16 bytes per row.  Where rows end inside the last group's 16 bytes, it
  // starts that much earlier.  (WHOLE rows have 16 scales at least.)  Rows that start at any byte are copied from the
  // word that holds their group's first: 16 bytes then hold 3 slices' 12 wherever those start in them.  (Loaded byte by
  // byte they kept every copy behind them waiting: 8192 rows on 32 experts of 4128 x 2080 in e4m3 370 us a call against 518;
  // of 4096 x 2048 273.)
  constexpr int GROUP = WHOLE ? T::GROUP : 3;
  static_assert(WHOLE || (T::SLICE == 128 && T::STAGES <= GROUP + 1), "words of 4 blocks, and two sets");
  char* s_scales = smem + T::STAGES * T::STAGE;
  auto group_start = [&](int s) { return WHOLE ? min(s / GROUP * 16, KB - 16) : s / GROUP * 12; };   // block
  // A stage's copies in pieces, each issued behind two tiles' products: STEPS of them in a slice's last part, and where
  // there are many, as many more in the next slice's first (256 rows in e4m3 397 us a call against 420, of 8192 rows
  // on 32 experts of 7168 x 2048; smaller tiles lose a little, 178 against 175 with 512 rows).
  constexpr int PIECES = STEPS > 2 ? 2 * STEPS : STEPS;
  auto stage_piece = [&](int s, char* base, int piece) {
#pragma unroll
    for (int c = 0; c < MINE; ++c) {
      if (c * PIECES / MINE != piece) continue;
      const int id = wave + c * T::WAVES;                      // wave-uniform
      if (c >= LEAST && id >= T::NX + T::NW) continue;
      const bool x = id < T::NX;
      const char* b = x ? xb + s * T::XROW : wb + s * T::WROW;
      bf16_t* dst = (bf16_t*)(base + id * 1024);
      if (WHOLE || (s + 1) * T::SLICE <= K) {                  // (uniform)
        dma16_sv(b, from[c], dst);
      } else {
        dma16_v(s * T::SLICE + first_value(x) < K ? b + from[c] : (const char*)g_zero_chunk, dst);
      }
    }
    if (piece == STEPS - 1 && s % GROUP == 0) {
      char* set = s_scales + s / GROUP % 2 * (T::SROWS * 16);
      const int at = group_start(s);
#pragma unroll
      for (int c = 0; c < SMINE; ++c) {
        const int id = wave + c * T::WAVES;
        if (id >= T::NS) continue;
        if constexpr (WHOLE) {
          dma16_v(sfrom[c] + at, (bf16_t*)(set + id * 1024));
        } else {
          const int first = (int)((uintptr_t)sfrom[c] & 3);
          const char* word = sfrom[c] - first + at;
          const bool past = word + 16 > (id * 64 + lane < T::BM ? x_end : w_end);
          dma16_v(past ? (const char*)g_zero_chunk : word, (bf16_t*)(set + id * 1024));
          if (__ballot(past)) {                                // the tensor's last rows: byte by byte
            wait_vmcnt<0>();
            if (past) {
              u32x4 v = {0, 0, 0, 0};
              for (int j = 0; j < 12 && at + j < KB; ++j) {
                const uint32_t s = (uint32_t)(uint8_t)sfrom[c][at + j] << (8 * ((first + j) % 4));
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] |= (first + j) / 4 == k ? s : 0u;
              }
              *reinterpret_cast<u32x4*>(set + id * 1024 + lane * 16) = v;
            }
          }
        }
      }
    }
  };
  auto stage = [&](int s, char* base, int pieces) {
#pragma unroll
    for (int piece = 0; piece < pieces; ++piece) stage_piece(s, base, piece);
  };

  // ---- K loop ----
  // the values' copies of the stages that may be on their way (the scales' come on top of them now and then: the wait
  // then asks for a little more than it has to)
  constexpr int AHEAD = (T::STAGES - 2) * LEAST;
  const int wm = wave / T::N_WAVES, wn = wave % T::N_WAVES;
  const int r = lane & 31, q = lane >> 5;
  f32x16 acc[NT][MT];

  struct Part {                        // operands of 64 values of K
    i32x8 w[NT], x[MT];
  };
  struct Scales {                      // of two parts: 4 blocks; shifted by the lane's q, bytes 0 and 2 are its own
    int w[NT], x[MT];
  };
  const int wrow = wn * NT * 32 + r, xrow = wm * MT * 32 + r;
  auto read_w = [&](const char* base, int j, int n, Part& h) {
    const char* W = base + T::X_BYTES + wrow * T::WROW + mx_chunk<T::WROW>(wrow, 2 * j + q) * 16;
    h.w[n] = narrow(ld16(W + n * 32 * T::WROW));
  };
  auto read_x = [&](const char* base, int j, int m, Part& h) {
    if constexpr (FMT == MX_E4M3) {
      const char* lo = base + xrow * T::XROW + mx_chunk<T::XROW>(xrow, 4 * j + q) * 16;
      const char* hi = base + xrow * T::XROW + mx_chunk<T::XROW>(xrow, 4 * j + 2 + q) * 16;
      const u32x4 a = ld16(lo + m * 32 * T::XROW), b = ld16(hi + m * 32 * T::XROW);
      h.x[m] = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
    } else {
      const char* X = base + xrow * T::XROW + mx_chunk<T::XROW>(xrow, 2 * j + q) * 16;
      h.x[m] = narrow(ld16(X + m * 32 * T::XROW));
    }
  };
  // The scales come to the registers 16 bytes of a row at a time, a group of slices: a word of each row, 16 bytes apart,
  // takes LDS as long as all 16 (803 us a call against 813, of 1024 rows on each of 8 experts of 4096 x 14336 in e2m1; the
  // same in e4m3).  For rows that start at any byte it is the two words that hold a slice's four.
  constexpr int HELD = WHOLE ? 4 : 2;
  uint32_t held_w[NT][HELD], held_x[MT][HELD];
  // where in its word a row's group starts (the same for rows 32 apart)
  const int first_w = WHOLE ? 0 : (int)((uintptr_t)(ws + (int64_t)weight_row(wrow) * KB) & 3);
  const int first_x = WHOLE ? 0 : (int)((uintptr_t)(xs + (int64_t)xrow * KB) & 3);
  auto word_of = [&](int i, int j) { return (T::SLICE / 32 * i - group_start(i)) / 4 + j / 2; };   // parts j, j + 1 of slice i
  auto read_scales = [&](int i, int j) {
    const char* S = s_scales + i / GROUP % 2 * (T::SROWS * 16);
    auto one = [&](int row, uint32_t (&v)[HELD]) {
      if constexpr (WHOLE) {
        const u32x4 r = ld16(S + row * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = r[k];
      } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(S + row * 16) + word_of(i, j);
        v[0] = w[0];
        v[1] = w[1];
      }
    };
#pragma unroll
    for (int n = 0; n < NT; ++n) one(T::BM + wrow + n * 32, held_w[n]);
#pragma unroll
    for (int m = 0; m < MT; ++m) one(xrow + m * 32, held_x[m]);
  };
  // (apart from the read: a shift beside it would wait for it, and for the operands read before it)
  auto own_scales = [&](int i, int j, Scales& s) {
    if constexpr (WHOLE) {
      auto take = [&](auto kc) {
        constexpr int k = decltype(kc)::value;
#pragma unroll
        for (int n = 0; n < NT; ++n) s.w[n] = held_w[n][k] >> (8 * q);
#pragma unroll
        for (int m = 0; m < MT; ++m) s.x[m] = held_x[m][k] >> (8 * q);
      };
      const int k = word_of(i, j);
      if (k == 0) take(std::integral_constant<int, 0>{});
      else if (k == 1) take(std::integral_constant<int, 1>{});
      else if (k == 2) take(std::integral_constant<int, 2>{});
      else take(std::integral_constant<int, 3>{});
    } else {
      // blocks past the row's end are zeros, never the next row's (255 would make NaN of zeros)
      const int left = KB - 4 * i;
      const uint32_t exist = left >= 4 ? ~0u : (1u << (8 * left)) - 1;
#pragma unroll
      for (int n = 0; n < NT; ++n) s.w[n] = (__builtin_amdgcn_alignbyte(held_w[n][1], held_w[n][0], first_w) & exist) >> (8 * q);
#pragma unroll
      for (int m = 0; m < MT; ++m) s.x[m] = (__builtin_amdgcn_alignbyte(held_x[m][1], held_x[m][0], first_x) & exist) >> (8 * q);
    }
  };
  // One part's products, with the wave's other work between them: an instruction waits for those before it, so reads or
  // copies in one piece would leave the matrix core idle until the last of all eight waves' had been issued (930 us a
  // call against 887, of 1024 rows on each of 8 experts of 4096 x 14336 in e2m1).  `other(i)` is issued behind the two
  // products of step i, all reads before the last step's.
  // (Matrix instructions are no memory accesses to the compiler, which would move them all behind the barrier.  The empty
  // statement that claims to change their results keeps them where they stand.)
  auto multiply = [&](auto jc, const Part& h, const Scales& s, auto other) {
    constexpr int j = decltype(jc)::value;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int m = 2 * i / NT, n0 = 2 * i % NT;
#pragma unroll
      for (int n = n0; n < n0 + 2; ++n)
        acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(h.w[n], h.x[m], acc[n][m], 4, FMT == MX_E4M3 ? 0 : 4,
                                                                    2 * (j % 2), s.w[n], 2 * (j % 2), s.x[m]);
      asm volatile("" : "+v"(acc[n0][m]), "+v"(acc[n0 + 1][m]));
      __builtin_amdgcn_sched_barrier(0);
      other(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // the next part's operands, weights first, spread over all steps but the last
  auto read_step = [&](const char* base, int j, int i, Part& h) {
#pragma unroll
    for (int k = 0; k < NT + MT; ++k) {
      if (k * (STEPS > 1 ? STEPS - 1 : 1) / (NT + MT) != i) continue;
      if (k < NT) read_w(base, j, k, h);
      else read_x(base, j, k - NT, h);
    }
  };

  char* ring[T::STAGES];
#pragma unroll
  for (int s = 0; s < T::STAGES; ++s) ring[s] = smem + s * T::STAGE;
  auto rotate = [&] {
    char* f = ring[0];
#pragma unroll
    for (int s = 0; s + 1 < T::STAGES; ++s) ring[s] = ring[s + 1];
    ring[T::STAGES - 1] = f;
  };
#pragma unroll
  for (int s = 0; s < T::STAGES; ++s)
    if (s < nk) stage(s, ring[s], s + 1 < T::STAGES ? PIECES : STEPS);
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.f;
  if (nk >= T::STAGES) wait_vmcnt<AHEAD + LEAST * STEPS / PIECES>();
  else wait_vmcnt<0>();
  lds_barrier();
  Part part[2];
  Scales s0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) read_step(ring[0], 0, i, part[0]);
  read_scales(0, 0);
  own_scales(0, 0, s0);
  // ring[0] holds slice s, ring[1] the next, ...
  int s = 0;
  // all parts of a slice but the last; `copy`: with the second half of the copies of the slice STAGES - 1 further on
  auto most_parts = [&](bool copy) {
    auto one = [&](auto jc) {
      constexpr int j = decltype(jc)::value;
      multiply(jc, part[j % 2], s0, [&](int i) {
        read_step(ring[0], j + 1, i, part[(j + 1) % 2]);
        if (!WHOLE && j % 2 && i == 0) read_scales(s, j + 1);
        if (PIECES > STEPS && j == 0 && copy) stage_piece(s + T::STAGES - 1, ring[T::STAGES - 1], STEPS + i);
      });
      if (j % 2) own_scales(s, j + 1, s0);
    };
    one(std::integral_constant<int, 0>{});
    if constexpr (T::PARTS > 2) {
      one(std::integral_constant<int, 1>{});
      one(std::integral_constant<int, 2>{});
    }
  };
  constexpr std::integral_constant<int, T::PARTS - 1> last{};
  for (; s + T::STAGES < nk; ++s) {
    most_parts(true);
    wait_vmcnt<AHEAD>();               // slice s + 1: at most the copies of those behind it are in flight
    lds_barrier();                     // every wave's, and its reads of slice s
    multiply(last, part[1], s0, [&](int i) {
      read_step(ring[1], 0, i, part[0]);
      if (i == 0 && (!WHOLE || (s + 1) % GROUP == 0)) read_scales(s + 1, 0);
      stage_piece(s + T::STAGES, ring[0], i);
    });
    own_scales(s + 1, 0, s0);
    rotate();
  }
  for (; s < nk; ++s) {                // the last slices: nothing more to copy
    most_parts(s + T::STAGES - 1 < nk);
    wait_vmcnt<0>();
    lds_barrier();
    multiply(last, part[1], s0, [&](int i) {
      read_step(ring[1], 0, i, part[0]);   // (behind the last slice: what lies there, not used)
      if (i == 0 && (!WHOLE || (s + 1) % GROUP == 0)) read_scales(min(s + 1, nk - 1), 0);
    });
    own_scales(min(s + 1, nk - 1), 0, s0);
    rotate();
  }

  // ---- results: lane (r, q) holds features 8 g + 4 q + i (g, i < 4) of row r of each tile ----
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int local = (wm * MT + m) * 32 + r;
    const int64_t row = row0 + local;
    if constexpr (SWIGLU) {
#pragma unroll
      for (int n = 0; n < NT; n += 2) {
        const int f0 = feat0 + wn * NT * 16 + n * 16;
        float a[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float h = acc[n][m][i], u = acc[n + 1][m][i];
          // (expf and a division: the up-projection 3 to 12% longer, the result's error the same to 1e-5)
          a[i] = h * __builtin_amdgcn_rcpf(1.0f + __expf(-h)) * u;
        }
        uint32_t most = abs_max_bits(a);
        most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
        const uint32_t s = mx_scale_byte<FMT>(most);
        const bool live = local < rows && f0 < N;               // N is whole blocks
        if constexpr (FMT == MX_E4M3) {
          // groups g of 4 features as dwords; lane q ends up with features 16 q .. 16 q + 15
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = mx_pack4_e4m3(a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3], s);
          const uint32_t o0 = (uint32_t)__shfl_xor((int)(q ? w[0] : w[2]), 32, 64);
          const uint32_t o1 = (uint32_t)__shfl_xor((int)(q ? w[1] : w[3]), 32, 64);
          const u32x4 v = q ? u32x4{o0, w[2], o1, w[3]} : u32x4{w[0], o0, w[1], o1};
          if (live) st16(p.Yq + row * N + f0 + 16 * q, v);
        } else {
          // pairs of groups: 4 half-bytes each, merged with the partner's
          float lo[8], hi[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            lo[i] = a[i];
            hi[i] = a[8 + i];
          }
          const uint32_t w0 = mx_pack8_e2m1(lo, s), w1 = mx_pack8_e2m1(hi, s);   // groups 0, 1 and 2, 3
          const uint32_t o = (uint32_t)__shfl_xor((int)(q ? w0 : w1), 32, 64);
          const uint32_t own = q ? w1 : w0;
          // dword of 8 features = low half of lane q = 0's group, then lane q = 1's
          const uint32_t e = q ? (o & 0xffffu) | (own << 16) : (own & 0xffffu) | (o << 16);
          const uint32_t f = q ? (o >> 16) | (own & 0xffff0000u) : (own >> 16) | (o & 0xffff0000u);
          if (live) *reinterpret_cast<u32x2*>(p.Yq + (row * N + f0) / 2 + 8 * q) = u32x2{e, f};
        }
        if (live && q == 0) p.Y_scales[row * (N / 32) + f0 / 32] = (uint8_t)s;
      }
    } else {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int f0 = feat0 + wn * NT * 32 + n * 32;
        uint32_t w[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i][0] = pack_bf16x2(acc[n][m][4 * i], acc[n][m][4 * i + 1]);
          w[i][1] = pack_bf16x2(acc[n][m][4 * i + 2], acc[n][m][4 * i + 3]);
        }
        uint32_t o[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) o[i][h] = (uint32_t)__shfl_xor((int)(q ? w[i][h] : w[2 + i][h]), 32, 64);
        if (local < rows && f0 < N) {
          bf16_t* y = p.Y + row * N + f0 + 16 * q;
          if (q) {
            st16(y, u32x4{o[0][0], o[0][1], w[2][0], w[2][1]});
            st16(y + 8, u32x4{o[1][0], o[1][1], w[3][0], w[3][1]});
          } else {
            st16(y, u32x4{w[0][0], w[0][1], o[0][0], o[0][1]});
            st16(y + 8, u32x4{w[1][0], w[1][1], o[1][0], o[1][1]});
          }
        }
      }
    }
  }
}

template <class T, bool SWIGLU, bool WHOLE>
__global__ __launch_bounds__(T::NTH) void k_mx_gemm(MxGemmProblem p) {
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63;
  constexpr int FEAT = SWIGLU ? T::BN / 2 : T::BN;             // output features of a tile
  const int ntiles = (p.N + FEAT - 1) / FEAT;

  // Tiles: groups in order, inside a group m fastest.  Every wave finds its own, a group per lane: the launch cannot
  // know the loads, and what precedes a tile's first copy is time that the compute unit idles.
  struct Block {                                               // of up to 64 groups
    int64_t row0;                                              // this lane's group: rows, clamped to the buffers
    int rows, tiles, upto;                                     // (upto: tiles of the block's groups up to this one)
  };
  auto load = [&](int base) {
    const int g = base + lane;
    Block k = {0, 0, 0, 0};
    if (g < p.groups) {
      if (p.seg_stride > 0) {
        k.row0 = (int64_t)g * p.seg_stride;
        k.rows = min(max(p.offsets[g], 0), p.seg_stride);
      } else {
        const int64_t a = p.offsets[g], b = p.offsets[g + 1];
        k.row0 = min(max(a, (int64_t)0), p.max_rows);
        k.rows = (int)(max(k.row0, min(b, p.max_rows)) - k.row0);
      }
    }
    k.tiles = k.upto = (int)(((int64_t)k.rows + T::BM - 1) / T::BM);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int n = __shfl_up(k.upto, o, 64);
      if (lane >= o) k.upto += n;
    }
    return k;
  };
  Block k = load(0);
  int total = __builtin_amdgcn_readlane(k.upto, 63);
  for (int base = 64; base < p.groups; base += 64) total += __builtin_amdgcn_readlane(load(base).upto, 63);
  // consecutive tiles to one XCD (workgroup b runs on XCD b % 8): they share weights and rows in its L2
  const uint32_t tiles = (uint32_t)total * ntiles, per = (tiles + 7) / 8;   // (the host bounds it by the grid)
  const uint32_t slot = blockIdx.x / 8, tile = blockIdx.x % 8 * per + slot;
  if (slot >= per || tile >= tiles) return;                    // the whole workgroup
  const int at = (int)(tile / ntiles);
  int before = 0, base = 0;
  uint64_t mask;
  while (!(mask = __ballot(at < before + k.upto))) {           // (at < total: some block has it)
    before += __builtin_amdgcn_readlane(k.upto, 63);
    k = load(base += 64);
  }
  const int l = __builtin_ctzll(mask), g = base + l;
  const int mine = __builtin_amdgcn_readlane(k.tiles, l);
  before += __builtin_amdgcn_readlane(k.upto, l) - mine;
  const int local = (int)(tile - (uint32_t)before * ntiles), m0 = local % mine * T::BM;
  const int64_t row0 = (((int64_t)__builtin_amdgcn_readlane((int)(k.row0 >> 32), l) << 32) |
                        (uint32_t)__builtin_amdgcn_readlane((int)k.row0, l)) + m0;
  const int rows = min(T::BM, __builtin_amdgcn_readlane(k.rows, l) - m0);   // >= 1
  const int feat0 = local / mine * FEAT;
  // a group's last rows: as many of a wave's tiles as they need
  if constexpr (T::LOWS > 0)
    if (rows <= 64) return mx_tile<typename T::template Low<1>, SWIGLU, WHOLE>(p, smem, g, row0, rows, feat0);
  if constexpr (T::LOWS > 1)
    if (rows <= 128) return mx_tile<typename T::template Low<2>, SWIGLU, WHOLE>(p, smem, g, row0, rows, feat0);
  mx_tile<T, SWIGLU, WHOLE>(p, smem, g, row0, rows, feat0);
}

// a launch holds the tile and its low ones
template <class T>
constexpr int launch_lds() {
  int most = T::LDS;
  if (T::LOWS > 0 && T::template Low<1>::LDS > most) most = T::template Low<1>::LDS;
  if (T::LOWS > 1 && T::template Low<2>::LDS > most) most = T::template Low<2>::LDS;
  return most;
}

template <class T, bool SWIGLU, bool WHOLE>
hipError_t launch_as(const MxGemmProblem& p, hipStream_t stream) {
  static OccCache cache;
  hipError_t err = hipSuccess;
  const void* fn = reinterpret_cast<const void*>(&k_mx_gemm<T, SWIGLU, WHOLE>);
  const int per_cu = kernel_occupancy(cache, fn, T::NTH, launch_lds<T>(), err);
  if (per_cu <= 0) return err;
  constexpr int FEAT = SWIGLU ? T::BN / 2 : T::BN;
  const int64_t ntiles = (p.N + FEAT - 1) / FEAT;
  // every group adds at most one partial tile
  int64_t mtiles = p.max_rows / T::BM + (p.groups < p.max_rows ? p.groups : p.max_rows);
  if (p.seg_stride > 0) mtiles = (int64_t)p.groups * ((p.seg_stride + T::BM - 1) / T::BM);
  const int64_t blocks = (mtiles * ntiles + 7) / 8 * 8;        // whole rounds of the 8 XCDs
  if (blocks * T::NTH > UINT32_MAX) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_mx_gemm<T, SWIGLU, WHOLE>), dim3((unsigned)blocks), dim3(T::NTH), launch_lds<T>(), stream, p);
  return hipGetLastError();
}

template <int FMT, int WM, int WN, int MT, int NT>
hipError_t launch_tile(const MxGemmProblem& p, hipStream_t stream) {
  const MxSlices slices = mx_slices(FMT == MX_E2M1, WN * NT * 32, p.K);
  if constexpr (FMT == MX_E2M1 && WN * NT == 8) {
    if (slices == MxSlices::kWhole256) {
      using T = MxTile<FMT, WM, WN, MT, NT, 3, 256>;
      return p.swiglu ? launch_as<T, true, true>(p, stream) : launch_as<T, false, true>(p, stream);
    }
  }
  using T = MxTile<FMT, WM, WN, MT, NT, 4, 128>;
  const bool whole = slices == MxSlices::kWhole128;
  if (p.swiglu) return whole ? launch_as<T, true, true>(p, stream) : launch_as<T, true, false>(p, stream);
  return whole ? launch_as<T, false, true>(p, stream) : launch_as<T, false, false>(p, stream);
}

template <int FMT>
hipError_t launch_format(const MxGemmProblem& p, hipStream_t stream) {
  switch (mx_tile_rule(cu_count(), p.max_rows, p.groups, p.N * (p.swiglu ? int64_t(2) : int64_t(1)))) {
    case MxTileId::k128x128: return launch_tile<FMT, 4, 2, 1, 2>(p, stream);
    case MxTileId::k256x256: return launch_tile<FMT, 4, 2, 2, 4>(p, stream);
    default: return launch_tile<FMT, 2, 4, 2, 2>(p, stream);
  }
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmProblem& p, hipStream_t stream) {
  if (p.groups < 1 || p.groups > kMaxGroups || p.K % 32 || p.N % 32 || (int64_t)p.N * p.K >= kMxGroupValues ||
      p.N >= kMxRowValues || p.K >= kMxRowValues)
    return hipErrorInvalidValue;
  return p.format == MX_E4M3 ? launch_format<MX_E4M3>(p, stream) : launch_format<MX_E2M1>(p, stream);
}

}  // namespace moe
