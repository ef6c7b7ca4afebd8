// The whole layer for a few tokens (T <= 64): what it takes is a stream of the active experts' weights,
// each read once, with little else in its way.
//
// Products run on v_mfma_f32_16x16x32_bf16 with 16 weight rows as the first operand and up to 16 token
// rows as the second (columns without a token are zeros), weights straight from memory into registers:
// no row of weights is used twice, so LDS would only add a stop.  A wave works in units of 256 values of
// K, 16 bytes per lane and load; 4-bit weights are turned into bf16 in registers (exactly: an element
// times a power of two).
//
//   logits   16 experts and 16 tokens by a part of K per workgroup, a quarter of it per wave; float32
//            partials that the gate adds
//   gate     one wave per token (gate_device.hpp); the workgroup that ends last makes the plan:
//            the experts that have rows, in blocks of 16 of them, and their slots.  Per expert there is the
//            64-bit mask of its tokens, so a slot's rank is a popcount and the order does not depend on
//            the order of the writes.  (With up to four tokens there is no such launch: up does this for itself)
//   up       a workgroup owns a block of rows of one expert and 16, 32 or 64 features (gate and up rows); its
//            waves take 16 features each, or parts of K of the same ones
//   down     the same on the other weights; float32 rows for each slot
//   combine  the token's rows times their gates, in slot order, and the shared expert's; rounded once
//
// What bounds it is the rate at which the weights arrive, so a wave keeps 4 units of 4-bit weights (3 of bf16) on
// their way and asks the memory for nothing else: the token rows of its expert and the scales of its weights are
// staged in LDS first, in whole lines.  (Fetched lane by lane next to the weights, they took more of the L1's accesses
// than the weights did: 385 us against 210 in the second case below.)  Every load that the compiler sees in
// the loop is unconditional: behind one that may not have been issued, it has to wait for all of them.
//
// Measured: 4 tokens on 8 experts of 4096 x 14336 in 4 bits, top-2, of which 5 to 7 are chosen: 94 - 114 us a call,
// some 5 TB/s of weights; 64 tokens on 48 of 384 experts of 7168 x 2048 in 4 bits, top-8, and a shared expert: 194 - 208 us,
// 4.1 - 4.4 TB/s (up 104 - 114 us, down 78 - 85, gate 14, logits 10, combine 4.7); one token, 128 experts of 2048 x 768 in
// bf16, top-8: 30 us (logits 4.4, up 16.9, down 8.0, combine 3.8), of which the weights' stream is 14 at the rate of a read
// and the four launches that wait for each other the rest.
#include "common.hpp"
#include "decode_geometry.hpp"
#include "gate_device.hpp"
#include "gemm_device.hpp"
#include "kernels.hpp"
#include "mx_device.hpp"

namespace moe {
namespace {

using Geometry = DecodeGeometry;

// an offset past every buffer (they end below it)
constexpr uint32_t kPast = 0x80000000u;

// K values of a unit: the operand fragments of 32 values whose loads a wave issues together.
template <bool MX>
struct Unit {
  static constexpr int K = decode_unit(MX);
  static constexpr int FRAGS = K / 32;
};

// Lane (r = l % 16, q = l / 16) holds 8 values of row r in fragment f of a unit; which 8 is free as long
// as both operands agree.  bf16: every load takes 16 of the 128 bytes that the four q's lanes read of a
// row in two loads; 4 bits: a lane's 16 bytes are one block of 32 values, four fragments.
template <bool MX>
__device__ __forceinline__ int frag_k(int f, int q) {
  return MX ? 128 * (f / 4) + 32 * q + 8 * (f % 4) : 64 * (f / 2) + 16 * q + 8 * (f % 2);
}

// Buffer of `bytes` bytes from a wave-uniform address: loads take a 32-bit offset per lane and give zeros
// past the end, so rows and values that do not exist need no address of their own.  The check subtracts a load's
// uniform offset from the buffer's size, so that offset has to lie inside the buffer.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer(const void* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)min(bytes, (int64_t)kPast), 0x00027000);
}
__device__ __forceinline__ u32x4 load16(Buffer b, uint32_t lane_offset, int uniform_offset) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, (int)lane_offset, uniform_offset, 0));
}

// WHOLE: K is a multiple of the unit, so no load has to ask whether its values exist.
template <bool MX, bool WHOLE>
struct WeightUnit {
  u32x4 v[MX ? 2 : 4];

  // this lane's part of the unit at k0 of 16 rows of K values: zeros from `end` on; not `on`: nothing is read
  __device__ __forceinline__ void load(Buffer w, int r, int q, int k0, int K, int end, bool on = true) {
#pragma unroll
    for (int i = 0; i < (MX ? 2 : 4); ++i) {
      const int k = frag_k<MX>(MX ? 4 * i : i, q);
      v[i] = load16(w, on && (WHOLE || k0 + k < end) ? (MX ? (r * K + k) / 2 : 2 * (r * K + k)) : kPast,
                                  MX ? k0 / 2 : 2 * k0);
    }
  }
  // fragment f; scale: of this lane's block f / 4, as a float (4-bit weights).  The conversion looks at the scale's
  // exponent bits alone: a zero field is 2^-127, 255 NaN.
  __device__ __forceinline__ bf16x8 frag(int f, const float* scale) const {
    if constexpr (MX) {
      const uint32_t w = v[f / 4][f % 4];
      u32x4 r;
      r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale[f / 4], 0));
      r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale[f / 4], 1));
      r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale[f / 4], 2));
      r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale[f / 4], 3));
      return __builtin_bit_cast(bf16x8, r);
    } else {
      return __builtin_bit_cast(bf16x8, v[f]);
    }
  }
};

// FRAGS fragments of one lane's token row, which starts `row` bytes into the buffer (kPast: no token, zeros)
template <bool MX, int FRAGS>
struct RowUnit {
  u32x4 v[FRAGS];
  // fragments first .. first + FRAGS - 1 of the unit at k0
  __device__ __forceinline__ void load(Buffer rows, uint32_t row, int q, int k0, int K, int first = 0) {
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) {
      const int k = frag_k<MX>(first + f, q);
      v[f] = load16(rows, k0 + k < K && row != kPast ? row + 2 * k : kPast, 2 * k0);
    }
  }
};

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// ---------------- logits ----------------
// A workgroup: 16 experts, 16 tokens, one partial's share of K, a quarter of it per wave.
__global__ __launch_bounds__(256) void k_decode_logits(DecodeProblem p, int chunk) {
  __shared__ f32x4 s_sum[3][64];
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int e0 = blockIdx.x * 16, t = blockIdx.y * 16 + r, split = blockIdx.z;
  // the next kernel counts its workgroups here
  if (blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) p.plan->arrived = 0;
  const int begin = (split * 4 + wave) * chunk, end = min(p.d, begin + chunk);
  const Buffer w = buffer(p.w_router + (int64_t)e0 * p.d, (int64_t)min(16, p.E - e0) * p.d * 2);
  const Buffer x = buffer(p.x, (int64_t)p.T * p.d * 2);
  const uint32_t row = t < p.T ? (uint32_t)t * p.d * 2 : kPast;
  constexpr int UK = Unit<false>::K, IN_FLIGHT = 2;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = begin; k0 < end; k0 += IN_FLIGHT * UK) {
    WeightUnit<false, false> u[IN_FLIGHT];
    RowUnit<false, Unit<false>::FRAGS> b[IN_FLIGHT];
#pragma unroll
    for (int i = 0; i < IN_FLIGHT; ++i) {
      const int k = min(k0 + i * UK, p.d - 1) / 8 * 8;             // inside the row, past `end` or not
      const int stop = k0 + i * UK < end ? end : 0;
      u[i].load(w, r, q, k, p.d, stop);                       // (neither side past `end`: an infinity times 0 is NaN)
      b[i].load(x, row, q, k, stop);
    }
#pragma unroll
    for (int i = 0; i < IN_FLIGHT; ++i)
#pragma unroll
      for (int f = 0; f < Unit<false>::FRAGS; ++f) acc = mfma16(u[i].frag(f, nullptr), b[i].v[f], acc);
  }
  if (wave > 0) s_sum[wave - 1][lane] = acc;
  __syncthreads();
  if (wave == 0 && t < p.T) {
    acc += s_sum[0][lane];
    acc += s_sum[1][lane];
    acc += s_sum[2][lane];
    float* out = p.logits + ((int64_t)split * p.T + t) * p.E + e0 + 4 * q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e0 + 4 * q + i < p.E) out[i] = acc[i];
  }
}

// ---------------- gate and plan ----------------
// One wave per token; the workgroup that ends last makes the plan from all tokens' choices.
template <int PL>
__global__ __launch_bounds__(256) void k_decode_gate(DecodeProblem p) {
  __shared__ float s_key[4][64 * PL];
  __shared__ float s_gscore[4][64];
  __shared__ unsigned long long s_mask[kMaxGroups];
  __shared__ int s_begin[kMaxGroups], s_tmp[4], s_last;
  __shared__ uint32_t s_kept[kDecodeTokens];
  const int tid = threadIdx.x, n = p.T * p.top_k, wave = tid >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wave;
  if (tid < kDecodeTokens) s_kept[tid] = 0;
  for (int e = tid; e < p.E_local; e += 256) s_mask[e] = 0ull;
  if (t < p.T) gate_token<PL>(p.gate, t, s_key[wave], s_gscore[wave]);
  // (with other workgroups:) the choices reach the device's memory before the count does, and are read back behind it
  if (gridDim.x > 1) __threadfence();
  __syncthreads();
  if (gridDim.x > 1) {
    if (tid == 0) s_last = atomicAdd(&p.plan->arrived, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
  }
  // this thread's slots and their local experts (-1: none)
  constexpr int SLOTS = kDecodeSlots / 256;
  int mine[SLOTS];
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    const int i = tid + 256 * j, e = i < n ? p.gate.topk_idx[i] - p.e_begin : -1;
    mine[j] = e < p.E_local ? e : -1;
    if (mine[j] >= 0) atomicOr(&s_mask[e], 1ull << (i / p.top_k));
  }
  __syncthreads();
  const int cap = p.expert_capacity > 0 ? p.expert_capacity : kDecodeTokens;
  // four neighbouring experts per thread: rows in the low half, blocks of 16 of them in the high half
  int cnt[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * tid + i;
    cnt[i] = e < p.E_local ? min(__popcll(s_mask[e]), cap) : 0;
    sum += cnt[i] + ((cnt[i] + 15) / 16 << 16);
  }
  int excl;
  const int total = block_exclusive_scan<256>(sum, s_tmp, excl);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (cnt[i] > 0) {
      const int e = 4 * tid + i, a = excl >> 16, b = excl & 0xffff;
      s_begin[e] = b | a << 16;
      for (int k = 0; 16 * k < cnt[i]; ++k) {
        p.plan->entry[a + k].expert = e;
        p.plan->entry[a + k].begin = b + 16 * k;
        p.plan->entry[a + k].count = min(16, cnt[i] - 16 * k);
      }
      excl += cnt[i] + ((cnt[i] + 15) / 16 << 16);
    }
  }
  const int most = decode_entries(p.T, p.top_k, p.E_local);
  for (int a = (total >> 16) + tid; a < most; a += 256) p.plan->entry[a].count = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    const int i = tid + 256 * j, e = mine[j];
    if (e >= 0) {
      const int rank = __popcll(s_mask[e] & ((1ull << (i / p.top_k)) - 1));
      if (rank < cap) {
        p.plan->slot[(s_begin[e] & 0xffff) + rank] = i;
        if (rank % 16 == 0) p.plan->entry[(s_begin[e] >> 16) + rank / 16].first = i;
        atomicOr(&s_kept[i / p.top_k], 1u << (i % p.top_k));
      }
    }
  }
  __syncthreads();
  if (tid < p.T) p.plan->kept[tid] = s_kept[tid];
}

// ---------------- the experts' products ----------------
constexpr int kWaves = kDecodeWaves;
// units of weights a wave has on their way
template <bool MX>
constexpr int kStages = MX ? 4 : 3;

// What a workgroup multiplies: m rows of `rows` (row_at(i) bytes into it) by weight rows [row0, ..) of K values,
// NS streams (gate and up) of them `stream` rows apart.
struct Product {
  const void* w;
  const uint8_t* scales;
  const bf16_t* rows;
  int64_t row0;
  int32_t stream, K, features, f0, m;
  const int32_t* slots;            // of the rows; nullptr: row i is token first + i
  int32_t first;                   // slots[0]
  int32_t per_token;               // slots per row of `rows`: top_k (token rows), or 1 (rows of slots)
  // slot of this lane's row r (a lane without one: the last row's)
  __device__ __forceinline__ int slot_of_lane(int r) const {
    const int i = min(r, m - 1);
    int s = first + (slots ? 0 : i);
    if (slots && m > 1) s = slots[i];
    return s;
  }
};

// acc[s]: features f0w + 4 q + j of row r, for this wave's part of K (of `split` parts)
template <bool MX, bool WHOLE, int NS>
__device__ __forceinline__ void multiply(const Product& p, int slot, int f0w, int part, int split, int room, char* lds,
                                         f32x4 (&acc)[NS]) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int UK = Unit<MX>::K, FRAGS = Unit<MX>::FRAGS, STAGES = kStages<MX>;
  const int K = p.K, units = (K + UK - 1) / UK, KB = K / 32;
  // rows that exist; a wave past them all computes the last one again (its results are not used)
  const int n = max(1, min(16, p.features - f0w));
  const int64_t wbytes = MX ? K / 2 : 2 * (int64_t)K;
  Buffer w[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int64_t row = p.row0 + (int64_t)s * p.stream + min(f0w, p.features - 1);
    w[s] = buffer(static_cast<const char*>(p.w) + row * wbytes, n * wbytes);
    acc[s] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  struct Stage {
    WeightUnit<MX, WHOLE> w[NS];
  };
  const int count = part < units ? (units - part + split - 1) / split : 0;   // this wave's units
  const int rounds = (units + split - 1) / split;                            // the most any wave has
  // the wave's unit i; past the last, loads all the same (they stay unconditional) but of nothing
  auto load = [&](Stage& st, int i) {
    const int u = min(part + split * i, units - 1);
#pragma unroll
    for (int s = 0; s < NS; ++s) st.w[s].load(w[s], r, q, u * UK, K, K, i < count);
  };

  // ---- LDS: the scales of all the workgroup's weight rows, then its token rows, as many rounds of K at a time as
  // there is room for; copied straight from memory ----
  auto copy = [&](const char* src, char* dst, int vectors) {       // of 16 bytes; waves take 64 in turn
    for (int c = 64 * wave; c < vectors; c += 64 * kWaves)
      if (c + lane < vectors) dma16_v(src + 16 * (int64_t)(c + lane), reinterpret_cast<bf16_t*>(dst + 16 * c));
  };
  const int tile = features_of(split);
  char* s_rows = lds + (MX ? NS * tile * KB : 0);
  const int per_round = split * UK;                                // values of K
  const int row = p.per_token > 1 ? slot / p.per_token : slot;
  const int held = max(1, min(rounds, (room / p.m - 16) / (2 * per_round)));   // rounds in LDS
  const int pitch = row_bytes(min(held * per_round, K));
  auto copy_rows = [&](int round) {
    const int k0 = round * per_round, len = min(held * per_round, K - k0);
    for (int i = 0; i < p.m; ++i)                                  // (no load in here: see above)
      copy(reinterpret_cast<const char*>(p.rows) + 2 * ((int64_t)__builtin_amdgcn_readlane(row, i) * K + k0),
           s_rows + i * pitch, len / 8);
  };
  copy_rows(0);
  if constexpr (MX) {
    // 16 rows' scales are K / 2 bytes, whole vectors of 16; features come in 32s
    const int bytes = min(tile, p.features - p.f0) * KB;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      copy(reinterpret_cast<const char*>(p.scales) + (p.row0 + (int64_t)s * p.stream + p.f0) * KB, lds + s * tile * KB,
           bytes / 16);
  }
  Stage st[STAGES];
#pragma unroll
  for (int i = 0; i < STAGES; ++i) load(st[i], i);
  // the copies have landed, and the first unit's loads, when at most the other units' are on their way
  wait_vmcnt<(STAGES - 1) * NS * (MX ? 2 : 4)>();
  raw_barrier();

  const uint8_t* my_scales = reinterpret_cast<const uint8_t*>(lds) + (f0w - p.f0 + r) * KB;
  const char* mine = s_rows + min(r, p.m - 1) * pitch;             // a column without a row reads the last row
  auto step = [&](Stage& now, int i, int first) {                  // round i, rounds from `first` in LDS
    const int k0 = (part + split * i) * UK, base = first * per_round;
    float scale[NS][2];
    if constexpr (MX) {
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int b = k0 / 32 + 4 * j + q;
          scale[s][j] = __uint_as_float((uint32_t)my_scales[s * tile * KB + (WHOLE ? b : min(b, KB - 1))] << 23);
        }
    }
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) {
      const int k = k0 + frag_k<MX>(f, q);
      u32x4 b = ld16(mine + 2 * ((WHOLE ? k : min(k, K - 8)) - base));
      if (!WHOLE && k >= K) b = u32x4{0, 0, 0, 0};                 // values that do not exist: zeros times zeros
#pragma unroll
      for (int s = 0; s < NS; ++s) acc[s] = mfma16(now.w[s].frag(f, scale[s]), b, acc[s]);
    }
  };
  int first = 0;
  for (int i = 0; i < rounds; i += STAGES) {
#pragma unroll
    for (int j = 0; j < STAGES; ++j) {
      if (i + j == first + held && i + j < rounds) {               // the same for every wave
        lds_barrier();                                             // everybody has read the rounds held
        first = i + j;
        copy_rows(first);
        wait_vmcnt<0>();
        raw_barrier();
      }
      if (i + j < count) step(st[j], i + j, first);
      load(st[j], i + j + STAGES);
    }
  }
  __syncthreads();                                                 // the LDS is used again
}

// Multiplies, adds the parts of K in order, and hands each lane of the waves with part 0 its results:
// done(slot, f, sums) for its row's slot and features f .. f + 3.
template <bool MX, bool WHOLE, int NS, class Done>
__device__ __forceinline__ void product(const Product& p, int split, int room, char* lds, Done&& done) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % split;
  const int f0w = p.f0 + 16 * (wave / split);
  f32x4 acc[NS];
  const int slot = p.slot_of_lane(r);
  multiply<MX, WHOLE, NS>(p, slot, f0w, part, split, room, lds, acc);
  if (split > 1) {
    f32x4* red = reinterpret_cast<f32x4*>(lds);
    if (part > 0)
#pragma unroll
      for (int s = 0; s < NS; ++s) red[(wave * NS + s) * 64 + lane] = acc[s];
    __syncthreads();
    if (part == 0)
      for (int w = wave + 1; w < wave + split; ++w)
#pragma unroll
        for (int s = 0; s < NS; ++s) acc[s] += red[(w * NS + s) * 64 + lane];
  }
  if (part == 0 && r < p.m && f0w + 4 * q < p.features) done(slot, f0w + 4 * q, acc);
}

// A few tokens' gates and plan inside the up-projection: every workgroup chooses for itself, which takes less than a
// launch.  All write the same choices; the one that is asked to leaves the plan for the launches behind it.
constexpr int kOwnTokens = kWaves, kOwnSlots = 32;     // a wave per token, a lane per slot
// entry a of the plan, its slots into s_slot; false: there is none.  s_key: kOwnTokens * 64 * PL floats.
template <int PL>
__device__ __forceinline__ bool own_entry(const DecodeProblem& p, int a, bool leave, float* s_key, int* s_slot, DecodePlan::Entry& own) {
  __shared__ float s_gscore[kOwnTokens][64];
  __shared__ int s_idx[kOwnSlots];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = p.T * p.top_k;
  if (wave < p.T) {
    const int e = gate_token<PL>(p.gate, wave, s_key + wave * 64 * PL, s_gscore[wave]);
    if (lane < p.top_k) s_idx[wave * p.top_k + lane] = e;
  }
  __syncthreads();
  // lane = slot; entries in the order of their first slots
  // (a token chooses an expert once, so an expert has a row per token at most: s_slot holds them)
  const int cap = p.expert_capacity > 0 ? min(p.expert_capacity, kOwnTokens) : kOwnTokens;
  int e = lane < n ? s_idx[lane] - p.e_begin : -1;
  if (e >= p.E_local) e = -1;
  int rank = 0, all = 0, head = lane;
  for (int j = n - 1; j >= 0; --j) {
    const bool same = e >= 0 && __builtin_amdgcn_readlane(e, j) == e;
    all += same;
    rank += same && j < lane;
    head = same ? j : head;
  }
  const uint64_t heads = __ballot(e >= 0 && head == lane), kept = __ballot(e >= 0 && rank < cap);
  const int at = __popcll(heads & ((1ull << head) - 1)), count = min(all, cap);
  if (leave && wave == 0) {
    if (e >= 0 && head == lane) p.plan->entry[at] = DecodePlan::Entry{e, at * p.T, count, lane};
    if (e >= 0 && rank < cap) p.plan->slot[at * p.T + rank] = lane;
    if (__popcll(heads) + lane < decode_entries(p.T, p.top_k, p.E_local)) p.plan->entry[__popcll(heads) + lane].count = 0;
    if (lane < p.T) p.plan->kept[lane] = (uint32_t)(kept >> (lane * p.top_k)) & ((1u << p.top_k) - 1);
  }
  const uint64_t mine = __ballot(e >= 0 && head == lane && at == a);
  if (!mine) return false;                             // the whole workgroup
  const int l = __builtin_ctzll(mine);
  own.expert = __builtin_amdgcn_readlane(e, l);
  own.count = __builtin_amdgcn_readlane(count, l);
  own.first = l;
  if (wave == 0 && e == own.expert && rank < cap) s_slot[rank] = lane;
  __syncthreads();                                     // (the caller's LDS is free again, too)
  return true;
}

// The shared expert's workgroups come first (16 tokens and some features each), then those of the plan's entries.
// PL > 0: the plan is own_entry's.
template <bool MX, bool WHOLE, int PL>
__global__ __launch_bounds__(64 * kWaves, MX ? 4 : 3) void k_decode_up(DecodeProblem p, Geometry g) {
  extern __shared__ __align__(16) char lds[];
  __shared__ int s_slot[kOwnTokens];
  const int b = (int)blockIdx.x - g.shared, first = blockIdx.x / g.shared_tiles * 16;
  Product o{p.ws13, p.ws13_scales, p.x, 0, p.F_shared, p.d, p.F_shared,
            (int)(blockIdx.x % g.shared_tiles) * features_of(g.shared_split), min(16, p.T - first), nullptr, first, 1};
  bf16_t* act = p.act_shared;
  int split = g.shared_split;
  if (b >= 0) {
    DecodePlan::Entry e;
    if constexpr (PL > 0) {
      if (!own_entry<PL>(p, b / g.tiles, b == 0, reinterpret_cast<float*>(lds), s_slot, e)) return;
    } else {
      e = p.plan->entry[b / g.tiles];
      if (e.count == 0) return;
    }
    split = g.split;
    o.w = p.w13;
    o.scales = p.w13_scales;
    o.features = o.stream = p.F;
    o.row0 = (int64_t)e.expert * 2 * p.F;
    o.f0 = b % g.tiles * features_of(split);
    o.m = e.count;
    o.slots = PL > 0 ? s_slot : p.plan->slot + e.begin;
    o.first = e.first;
    o.per_token = p.top_k;
    act = p.act;
  }
  product<MX, WHOLE, 2>(o, split, g.room, lds, [&](int slot, int f, const f32x4 (&s)[2]) {
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = s[0][j] * __builtin_amdgcn_rcpf(1.0f + __expf(-s[0][j])) * s[1][j];
    const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    *reinterpret_cast<u32x2*>(act + (int64_t)slot * o.features + f) = w;
  });
}

template <bool MX, bool WHOLE>
__global__ __launch_bounds__(64 * kWaves, 4) void k_decode_down(DecodeProblem p, Geometry g) {
  extern __shared__ __align__(16) char lds[];
  const int b = (int)blockIdx.x - g.shared, first = blockIdx.x / g.shared_tiles * 16;
  Product o{p.ws2, p.ws2_scales, p.act_shared, 0, 0, p.F_shared, p.d,
            (int)(blockIdx.x % g.shared_tiles) * features_of(g.shared_split), min(16, p.T - first), nullptr, first, 1};
  float* y = p.y + (int64_t)p.T * p.top_k * p.d;
  int split = g.shared_split;
  if (b >= 0) {
    const DecodePlan::Entry e = p.plan->entry[b / g.tiles];
    if (e.count == 0) return;
    split = g.split;
    o.w = p.w2;
    o.scales = p.w2_scales;
    o.rows = p.act;
    o.row0 = (int64_t)e.expert * p.d;
    o.K = p.F;
    o.f0 = b % g.tiles * features_of(split);
    o.m = e.count;
    o.slots = p.plan->slot + e.begin;
    o.first = e.first;
    y = p.y;
  }
  product<MX, WHOLE, 1>(o, split, g.room, lds, [&](int slot, int f, const f32x4 (&s)[1]) {
    *reinterpret_cast<f32x4*>(y + (int64_t)slot * p.d + f) = s[0];
  });
}

// ---------------- combine ----------------
// out[t] = bf16(sum over the token's kept slots of gate * row, in slot order, + the shared expert's row); 4 columns
// per thread
__global__ __launch_bounds__(256) void k_decode_combine(DecodeProblem p) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4, t = blockIdx.y;
  if (c >= p.d) return;
  const uint32_t kept = p.plan->kept[t];
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int j = 0; j < p.top_k; ++j)
    if (kept >> j & 1) {
      const int64_t slot = (int64_t)t * p.top_k + j;
      s += *reinterpret_cast<const f32x4*>(p.y + slot * p.d + c) * p.gate.topk_w[slot];
    }
  if (p.F_shared) s += *reinterpret_cast<const f32x4*>(p.y + ((int64_t)p.T * p.top_k + t) * p.d + c);
  *reinterpret_cast<u32x2*>(p.out + (int64_t)t * p.d + c) = u32x2{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
}

// ---------------- launches ----------------
// `features` x K weights of each expert, ns streams of them (`features_s` x K_s of the shared expert)
Geometry geometry(const DecodeProblem& p, int features, int K, int features_s, int K_s, int ns, bool mx) {
  return decode_geometry({p.T, p.E, p.E_local, p.top_k, p.F_shared > 0}, features, K, features_s, K_s, ns, mx);
}

template <class Kernel>
hipError_t launch_product(Kernel kernel, OccCache& cache, const DecodeProblem& p, const Geometry& g, hipStream_t stream) {
  if (g.lds > kDecodeMostLds) return hipErrorInvalidValue;
  // (the limit of 64 KiB of dynamic LDS is raised once per device and kernel)
  hipError_t err = hipSuccess;
  if (kernel_occupancy(cache, reinterpret_cast<const void*>(kernel), 64 * kWaves, kDecodeMostLds, err) <= 0) return err;
  const int64_t blocks = g.shared + (int64_t)decode_entries(p.T, p.top_k, p.E_local) * g.tiles;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kWaves), g.lds, stream, p, g);
  return hipGetLastError();
}

template <int PL>
hipError_t launch_decode_gate(const DecodeProblem& p, hipStream_t stream) {
  hipLaunchKernelGGL(k_decode_gate<PL>, dim3((p.T + 3) / 4), dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <bool MX, bool WHOLE, int PL>
hipError_t launch_up(const DecodeProblem& p, const Geometry& g, hipStream_t stream) {
  static OccCache cache;
  return launch_product(k_decode_up<MX, WHOLE, PL>, cache, p, g, stream);
}
// the gate and the up-projection
template <bool MX, bool WHOLE>
hipError_t launch_gate_and_up(const DecodeProblem& p, hipStream_t stream) {
  const Geometry g = geometry(p, p.F, p.d, p.F_shared, p.d, 2, MX);
  const int64_t blocks = (int64_t)decode_entries(p.T, p.top_k, p.E_local) * g.tiles;
  // The gates in every workgroup, where there is a wave per token and a lane per slot, and all workgroups are on the chip
  // at once and start with them: one token through 128 experts of 2048 x 768 in bf16 29.9 us a captured call against 32.5, in 4
  // bits 22.8 against 25.3, through 48 of 384 of 7168 x 2048 in 4 bits with a shared expert 32.7 against 39.0; four tokens 62.3
  // against 63.6, 34.1 against 35.5, and the same either way.
  if (p.T <= kOwnTokens && p.T * p.top_k <= kOwnSlots && p.E <= 512 && blocks <= 4 * cu_count()) {
    static_assert(kDecodeRedBytes >= kOwnTokens * 64 * 8 * 4, "keys of 512 experts in a launch's LDS");
    return p.E <= 64 ? launch_up<MX, WHOLE, 1>(p, g, stream) : p.E <= 128 ? launch_up<MX, WHOLE, 2>(p, g, stream)
           : p.E <= 256 ? launch_up<MX, WHOLE, 4>(p, g, stream) : launch_up<MX, WHOLE, 8>(p, g, stream);
  }
  const hipError_t e = p.E <= 64 ? launch_decode_gate<1>(p, stream) : p.E <= 128 ? launch_decode_gate<2>(p, stream)
                       : p.E <= 256 ? launch_decode_gate<4>(p, stream) : p.E <= 512 ? launch_decode_gate<8>(p, stream)
                                                                                    : launch_decode_gate<16>(p, stream);
  return e != hipSuccess ? e : launch_up<MX, WHOLE, 0>(p, g, stream);
}
template <bool MX, bool WHOLE>
hipError_t launch_down(const DecodeProblem& p, hipStream_t stream) {
  static OccCache cache;
  const Geometry g = geometry(p, p.d, p.F, p.d, p.F_shared, 1, MX);
  return launch_product(k_decode_down<MX, WHOLE>, cache, p, g, stream);
}

template <bool MX>
hipError_t launch_as(const DecodeProblem& p, hipStream_t stream) {
  const int splits = decode_logits_splits(p.E, p.d);
  const int chunk = ((p.d + 63) / 64 + 4 * splits - 1) / (4 * splits) * 64;
  hipLaunchKernelGGL(k_decode_logits, dim3((p.E + 15) / 16, (p.T + 15) / 16, splits), dim3(256), 0, stream, p, chunk);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int UK = Unit<MX>::K;
  e = p.d % UK == 0 ? launch_gate_and_up<MX, true>(p, stream) : launch_gate_and_up<MX, false>(p, stream);
  if (e != hipSuccess) return e;
  e = p.F % UK == 0 && p.F_shared % UK == 0 ? launch_down<MX, true>(p, stream) : launch_down<MX, false>(p, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_decode_combine, dim3((p.d + 1023) / 1024, p.T), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode(const DecodeProblem& p, hipStream_t stream) {
  if (p.T < 1 || p.T > kDecodeTokens || p.E_local > kMaxGroups) return hipErrorInvalidValue;
  return p.w13_scales ? launch_as<true>(p, stream) : launch_as<false>(p, stream);
}

}  // namespace moe
