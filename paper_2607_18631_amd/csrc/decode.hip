// The whole layer for a few tokens (T <= 64): what it takes is a stream of the active experts' weights,
// each read once, with little else in its way.
//
// Products run on v_mfma_f32_16x16x32_bf16 with 16 weight rows as the first operand and up to 16 token
// rows as the second (columns without a token are zeros), weights straight from memory into registers:
// no row of weights is used twice, so LDS would only add a stop.  A wave works in units of 256 values of
// K, 16 bytes per lane and load; 4-bit weights are turned into bf16 in registers (exactly: an element
// times a power of two).
//
//   logits   16 experts by a chunk of K per wave, float32 partials that the gate adds
//   gate     one wave per token (gate_device.hpp)
//   plan     the experts that have rows and their slots: per expert the 64-bit mask of its tokens, so a
//            slot's rank is a popcount and the order does not depend on the order of the writes
//   up       16 features (gate and up rows) of one expert per workgroup, K dealt to its waves
//   down     16 output columns per workgroup: units of (expert, K chunk) dealt to its waves, each wave
//            adding its gate-weighted rows into token sums of its own in LDS; the waves' sums are added
//            in order and rounded once.  The combine needs no launch and no atomics.
#include "common.hpp"
#include "gate_device.hpp"
#include "gemm_device.hpp"
#include "kernels.hpp"
#include "mx_device.hpp"

namespace moe {
namespace {

constexpr int kUnit = 256;        // K values of a unit: 8 operand fragments of 32
constexpr int kUpWaves = 4;
constexpr int kDownWaves = 8;

// Lane (r = l % 16, q = l / 16) holds 8 values of row r in fragment f of a unit; which 8 is free as long
// as both operands agree.  bf16: every load takes 16 of the 128 bytes that the four q's lanes read of a
// row in two loads; 4 bits: a lane's 16 bytes are one block of 32 values, four fragments.
template <bool MX>
__device__ __forceinline__ int frag_k(int f, int q) {
  return MX ? 128 * (f / 4) + 32 * q + 8 * (f % 4) : 64 * (f / 2) + 16 * q + 8 * (f % 2);
}

// a row of weights, as this lane reads it (nullptr elements: a row that does not exist, zeros)
struct WeightRow {
  const char* elements;
  const uint8_t* scales;
};
template <bool MX>
__device__ __forceinline__ WeightRow weight_row(const void* w, const uint8_t* scales, int64_t row, int K, bool valid) {
  WeightRow r;
  r.elements = valid ? static_cast<const char*>(w) + row * (MX ? K / 2 : 2 * (int64_t)K) : nullptr;
  r.scales = MX && valid ? scales + row * (K / 32) : nullptr;
  return r;
}

__device__ __forceinline__ u32x4 ld16_or_zero(const char* p, bool valid) {
  return ld16(valid ? p : reinterpret_cast<const char*>(g_zero_chunk));
}

template <bool MX>
struct WeightUnit {
  u32x4 v[MX ? 2 : 8];
  uint32_t s[MX ? 2 : 1];

  __device__ __forceinline__ void load(const WeightRow& row, int k0, int K, int q) {
    const bool on = row.elements != nullptr;
    if constexpr (MX) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int b = k0 / 32 + 4 * i + q;
        const bool in = on && b < K / 32;
        v[i] = ld16_or_zero(row.elements + (int64_t)b * 16, in);
        s[i] = *(in ? row.scales + b : reinterpret_cast<const uint8_t*>(g_zero_chunk));
      }
    } else {
#pragma unroll
      for (int f = 0; f < 8; ++f) {
        const int k = k0 + frag_k<false>(f, q);
        v[f] = ld16_or_zero(row.elements + (int64_t)k * 2, on && k < K);
      }
    }
  }
  __device__ __forceinline__ bf16x8 frag(int f) const {
    if constexpr (MX) {
      const uint32_t w = v[f / 4][f % 4];
      const float scale = mx_scale(s[f / 4]);
      u32x4 r;
      r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
      r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
      r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
      r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
      return __builtin_bit_cast(bf16x8, r);
    } else {
      return __builtin_bit_cast(bf16x8, v[f]);
    }
  }
};

template <bool MX>
__device__ __forceinline__ void load_rows(u32x4 (&b)[8], const bf16_t* row, int k0, int K, int q) {
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    const int k = k0 + frag_k<MX>(f, q);
    b[f] = ld16_or_zero(reinterpret_cast<const char*>(row) + (int64_t)k * 2, row != nullptr && k < K);
  }
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// ---------------- logits ----------------
__global__ __launch_bounds__(256) void k_decode_logits(DecodeProblem p, int splits, int chunk) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int e0 = blockIdx.x * 16, split = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (split >= splits) return;
  const int k_end = min(p.d, (split + 1) * chunk);
  const WeightRow w = weight_row<false>(p.w_router, nullptr, e0 + r, p.d, e0 + r < p.E);
  f32x4 acc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = split * chunk; k0 < k_end; k0 += kUnit) {
    WeightUnit<false> u;
    u.load(w, k0, k_end, q);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c * 16 < p.T) {
        const int t = c * 16 + r;
        u32x4 b[8];
        load_rows<false>(b, t < p.T ? p.x + (int64_t)t * p.d : nullptr, k0, k_end, q);
#pragma unroll
        for (int f = 0; f < 8; ++f) acc[c] = mfma16(u.frag(f), b[f], acc[c]);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int t = c * 16 + r;
    if (t < p.T) {
      float* out = p.logits + ((int64_t)split * p.T + t) * p.E + e0 + 4 * q;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e0 + 4 * q + i < p.E) out[i] = acc[c][i];
    }
  }
}

// ---------------- plan ----------------
__global__ __launch_bounds__(256) void k_decode_plan(DecodeProblem p) {
  __shared__ unsigned long long s_mask[kMaxGroups];
  __shared__ int s_begin[kMaxGroups];
  __shared__ int s_tmp[4];
  const int tid = threadIdx.x, n = p.T * p.top_k;
  for (int e = tid; e < p.E_local; e += 256) s_mask[e] = 0ull;
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const int e = p.gate.topk_idx[i] - p.e_begin;
    if (e >= 0 && e < p.E_local) atomicOr(&s_mask[e], 1ull << (i / p.top_k));
  }
  __syncthreads();
  const int cap = p.expert_capacity > 0 ? p.expert_capacity : kDecodeTokens;
  // four neighbouring experts per thread: rows in the low half, experts with rows in the high half
  int cnt[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * tid + i;
    cnt[i] = e < p.E_local ? min(__popcll(s_mask[e]), cap) : 0;
    sum += cnt[i] + (cnt[i] > 0 ? 1 << 16 : 0);
  }
  int excl;
  const int total = block_exclusive_scan<256>(sum, s_tmp, excl);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (cnt[i] > 0) {
      const int e = 4 * tid + i, a = excl >> 16, b = excl & 0xffff;
      s_begin[e] = b;
      p.plan->expert[a] = e;
      p.plan->begin[a] = b;
      excl += cnt[i] + (1 << 16);
    }
  }
  if (tid == 0) {
    p.plan->n_active = total >> 16;
    p.plan->begin[total >> 16] = total & 0xffff;
  }
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const int e = p.gate.topk_idx[i] - p.e_begin;
    if (e >= 0 && e < p.E_local) {
      const int rank = __popcll(s_mask[e] & ((1ull << (i / p.top_k)) - 1));
      if (rank < cap) p.plan->slot[s_begin[e] + rank] = i;
    }
  }
}

// ---------------- up ----------------
// act[row_of(c)][f0 .. f0 + 15] = bf16(silu(gate) * up) for the m rows x[token_of(c)], c < m
template <bool MX, int CB>
__device__ __forceinline__ void up_tile(const DecodeProblem& p, const void* w13, const uint8_t* scales, int64_t wrow0,
                                        int F, int f0, int m, const int32_t* slots, bf16_t* act, float* s_red) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int K = p.d, units = (K + kUnit - 1) / kUnit;
  const bool in = f0 + r < F;
  const WeightRow gate = weight_row<MX>(w13, scales, wrow0 + f0 + r, K, in);
  const WeightRow up = weight_row<MX>(w13, scales, wrow0 + F + f0 + r, K, in);
  const bf16_t* x[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const int i = c * 16 + r;
    x[c] = nullptr;
    if (i < m) x[c] = p.x + (int64_t)(slots ? slots[i] / p.top_k : i) * K;
  }
  f32x4 acc[2][CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[0][c] = acc[1][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int u = wave; u < units; u += kUpWaves) {
    WeightUnit<MX> wg, wu;
    wg.load(gate, u * kUnit, K, q);
    wu.load(up, u * kUnit, K, q);
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      u32x4 b[8];
      load_rows<MX>(b, x[c], u * kUnit, K, q);
#pragma unroll
      for (int f = 0; f < 8; ++f) {
        acc[0][c] = mfma16(wg.frag(f), b[f], acc[0][c]);
        acc[1][c] = mfma16(wu.frag(f), b[f], acc[1][c]);
      }
    }
  }
  // the waves' sums, added in wave order
  f32x4* red = reinterpret_cast<f32x4*>(s_red);
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    red[((wave * 2 + 0) * CB + c) * 64 + lane] = acc[0][c];
    red[((wave * 2 + 1) * CB + c) * 64 + lane] = acc[1][c];
  }
  __syncthreads();
  for (int c = wave; c < CB; c += kUpWaves) {
    f32x4 h = red[c * 64 + lane], u = red[(CB + c) * 64 + lane];
#pragma unroll
    for (int w = 1; w < kUpWaves; ++w) {
      h += red[((w * 2 + 0) * CB + c) * 64 + lane];
      u += red[((w * 2 + 1) * CB + c) * 64 + lane];
    }
    const int i = c * 16 + r;
    if (i < m && f0 + 4 * q < F) {
      float a[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) a[j] = h[j] / (1.0f + expf(-h[j])) * u[j];
      const u32x2 v = {pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3])};
      *reinterpret_cast<u32x2*>(act + (int64_t)(slots ? slots[i] : i) * F + f0 + 4 * q) = v;
    }
  }
}

template <bool MX>
__global__ __launch_bounds__(64 * kUpWaves, 4) void k_decode_up(DecodeProblem p, int shared_tiles, int tiles) {
  __shared__ __align__(16) float s_red[kUpWaves * 2 * 4 * 64 * 4];
  const void* w13 = p.ws13;
  const uint8_t* scales = p.ws13_scales;
  int64_t wrow0 = 0;
  int F = p.F_shared, m = p.T, tile = blockIdx.x;
  const int32_t* slots = nullptr;
  bf16_t* act = p.act_shared;
  if (tile >= shared_tiles) {
    const int a = (tile - shared_tiles) / tiles;
    if (a >= p.plan->n_active) return;
    tile = (tile - shared_tiles) % tiles;
    const int b = p.plan->begin[a];
    w13 = p.w13;
    scales = p.w13_scales;
    F = p.F;
    wrow0 = (int64_t)p.plan->expert[a] * 2 * F;
    m = p.plan->begin[a + 1] - b;
    slots = p.plan->slot + b;
    act = p.act;
  }
  if (m <= 16) up_tile<MX, 1>(p, w13, scales, wrow0, F, tile * 16, m, slots, act, s_red);
  else if (m <= 32) up_tile<MX, 2>(p, w13, scales, wrow0, F, tile * 16, m, slots, act, s_red);
  else up_tile<MX, 4>(p, w13, scales, wrow0, F, tile * 16, m, slots, act, s_red);
}

// ---------------- down and combine ----------------
template <bool MX>
__global__ __launch_bounds__(64 * kDownWaves, 2) void k_decode_down(DecodeProblem p) {
  // every wave's sums of the tokens' 16 columns
  extern __shared__ __align__(16) float s_sum[];
  __shared__ int s_begin[kDecodeSlots + 1], s_expert[kDecodeSlots], s_slot[kDecodeSlots];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, q = lane >> 4, wave = tid >> 6;
  const int T = p.T, d0 = blockIdx.x * 16;
  const int n_active = p.plan->n_active;
  for (int i = tid; i <= n_active; i += 64 * kDownWaves) {
    s_begin[i] = p.plan->begin[i];
    if (i < n_active) s_expert[i] = p.plan->expert[i];
  }
  const int rows = p.plan->begin[n_active];
  for (int i = tid; i < rows; i += 64 * kDownWaves) s_slot[i] = p.plan->slot[i];
  for (int i = tid; i < kDownWaves * T * 16; i += 64 * kDownWaves) s_sum[i] = 0.f;
  __syncthreads();
  float* mine = s_sum + (int64_t)wave * T * 16;
  const int per = (p.F + kUnit - 1) / kUnit, per_s = (p.F_shared + kUnit - 1) / kUnit;
  const int routed = n_active * per, units = routed + per_s;
  for (int u = wave; u < units; u += kDownWaves) {
    const bool shared = u >= routed;
    const int a = shared ? 0 : u / per, k0 = (shared ? u - routed : u % per) * kUnit;
    const int F = shared ? p.F_shared : p.F, begin = shared ? 0 : s_begin[a];
    const int m = shared ? T : s_begin[a + 1] - begin;
    const int64_t wrow = (shared ? 0 : (int64_t)s_expert[a] * p.d) + d0 + r;
    const WeightRow row = weight_row<MX>(shared ? p.ws2 : p.w2, shared ? p.ws2_scales : p.w2_scales, wrow, F, d0 + r < p.d);
    WeightUnit<MX> w;
    w.load(row, k0, F, q);
    for (int c = 0; c < m; c += 16) {
      const bool on = c + r < m;
      int t = c + r;
      float g = 1.0f;
      const bf16_t* act = nullptr;
      if (on && shared) act = p.act_shared + (int64_t)t * F;
      if (on && !shared) {
        const int slot = s_slot[begin + c + r];
        t = slot / p.top_k;
        g = p.gate.topk_w[slot];
        act = p.act + (int64_t)slot * F;
      }
      u32x4 b[8];
      load_rows<MX>(b, act, k0, F, q);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < 8; ++f) acc = mfma16(w.frag(f), b[f], acc);
      if (on) {
        f32x4* s = reinterpret_cast<f32x4*>(mine + t * 16 + 4 * q);
        *s = *s + acc * g;
      }
    }
  }
  __syncthreads();
  // 8 columns per thread
  for (int i = tid; i < 2 * T; i += 64 * kDownWaves) {
    const int t = i >> 1, c = 8 * (i & 1);
    if (d0 + c < p.d) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
      for (int w = 0; w < kDownWaves; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += s_sum[(w * T + t) * 16 + c + j];
      st16(p.out + (int64_t)t * p.d + d0 + c, pack8(v));
    }
  }
}

template <bool MX>
hipError_t launch_as(const DecodeProblem& p, hipStream_t stream) {
  const int splits = decode_logits_splits(p.E, p.d);
  const int chunk = ((p.d + kUnit - 1) / kUnit + splits - 1) / splits * kUnit;
  hipLaunchKernelGGL(k_decode_logits, dim3((p.E + 15) / 16, (splits + 3) / 4), dim3(256), 0, stream, p, splits, chunk);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if ((e = launch_gate(p.gate, stream)) != hipSuccess) return e;
  hipLaunchKernelGGL(k_decode_plan, dim3(1), dim3(256), 0, stream, p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int tiles = (p.F + 15) / 16, shared_tiles = (p.F_shared + 15) / 16;
  const int active = p.E_local < p.T * p.top_k ? p.E_local : p.T * p.top_k;
  hipLaunchKernelGGL(k_decode_up<MX>, dim3(shared_tiles + active * tiles), dim3(64 * kUpWaves), 0, stream, p,
                     shared_tiles, tiles);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(k_decode_down<MX>, dim3((p.d + 15) / 16), dim3(64 * kDownWaves),
                     sizeof(float) * kDownWaves * p.T * 16, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode(const DecodeProblem& p, hipStream_t stream) {
  if (p.T < 1 || p.T > kDecodeTokens || p.E_local > kMaxGroups) return hipErrorInvalidValue;
  return p.w13_scales ? launch_as<true>(p, stream) : launch_as<false>(p, stream);
}

}  // namespace moe
