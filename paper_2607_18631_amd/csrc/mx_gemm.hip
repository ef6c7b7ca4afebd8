// Grouped products on block-scaled operands: Y[r, n] = sum_k X[r, k] W_g[n, k], X in e4m3 or e2m1, W in
// e2m1, on v_mfma_scale_f32_32x32x64_f8f6f4 (elements multiplied as they are, each block of 32 products
// times both blocks' powers of two, float32 accumulation).
//
// A workgroup owns BM rows of one group and BN weight rows; its K loop runs over slices of 128 values
// held in a ring of LDS stages, filled by direct-to-LDS copies that are issued STAGES - 1 slices ahead.
// Each wave multiplies MT x 2 tiles of 32 x 32: the weights are the first operand, so that a lane holds
// 16 of the 32 output features of one row, its partner lane (l ^ 32) the others.
//
// SwiGLU: a wave's two weight tiles are the gate and the up rows of the same 32 features, so the
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

namespace moe {
namespace {

constexpr int kSlice = 128;            // K values per stage

// 4-byte direct-to-LDS copy, as dma16_v
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma4_v(const void* src, void* dst) {
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(char*)dst;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

template <int FMT, int WM, int WN, int MT, int STAGES_>
struct MxTile {
  static constexpr int F = FMT, M_WAVES = WM, N_WAVES = WN, M_TILES = MT, STAGES = STAGES_;
  static constexpr int WAVES = WM * WN;
  static constexpr int NTH = WAVES * 64;
  static constexpr int BM = WM * MT * 32;
  static constexpr int BN = WN * 64;                          // weight rows
  static constexpr int XROW = FMT == MX_E4M3 ? 128 : 64;      // bytes of a slice's row
  static constexpr int X_BYTES = BM * XROW;
  static constexpr int W_BYTES = BN * 64;
  static constexpr int S_BYTES = (BM + BN + 63) / 64 * 256;   // scales: 4 blocks per row
  static constexpr int STAGE = X_BYTES + W_BYTES + S_BYTES;
  static constexpr int LDS = STAGE * STAGES;
  static constexpr int NX = X_BYTES / 1024, NW = W_BYTES / 1024, NS = S_BYTES / 256;   // wave copies
  static_assert(X_BYTES % 1024 == 0 && W_BYTES % 1024 == 0, "whole wave copies");
  static constexpr int COPIES = NX + NW + NS;
};

// 16-byte chunk of a row where the stage holds the row's chunk c: rows that share a bank cycle take
// different chunks, so the 16 lanes of a read pass touch every bank once
template <int ROW>
__device__ __forceinline__ int mx_chunk(int row, int c) {
  constexpr int CPR = ROW / 16, RPG = 16 / CPR;
  return c ^ ((row / RPG) % CPR);
}

template <class T, bool SWIGLU, bool WHOLE>
__global__ __launch_bounds__(T::NTH) void k_mx_gemm(MxGemmProblem p) {
  extern __shared__ __align__(16) char smem[];
  __shared__ int s_tmp[T::WAVES];
  __shared__ int s_own[4];
  constexpr int FMT = T::F, MT = T::M_TILES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = p.K, N = p.N;
  constexpr int FEAT = SWIGLU ? T::BN / 2 : T::BN;             // output features of a tile
  const int ntiles = (N + FEAT - 1) / FEAT;

  // ---- this workgroup's tile: groups in order, inside a group m fastest ----
  // rows of group g, clamped to the buffers
  auto segment = [&](int g, int64_t& a, int64_t& b) {
    if (p.seg_stride > 0) {
      a = (int64_t)g * p.seg_stride;
      b = a + min(max(p.offsets[g], 0), p.seg_stride);
    } else {
      a = min(max((int64_t)p.offsets[g], (int64_t)0), p.max_rows);
      b = max(a, min((int64_t)p.offsets[g + 1], p.max_rows));
    }
  };
  constexpr int GPT = (kMaxGroups + T::NTH - 1) / T::NTH;
  int mt[GPT], sum = 0;
#pragma unroll
  for (int i = 0; i < GPT; ++i) {
    const int g = tid * GPT + i;
    mt[i] = 0;
    if (g < p.groups) {
      int64_t a, b;
      segment(g, a, b);
      mt[i] = (int)((b - a + T::BM - 1) / T::BM);
    }
    sum += mt[i];
  }
  int excl;
  const int total = block_exclusive_scan<T::NTH>(sum, s_tmp, excl);
  // consecutive tiles to one XCD (workgroup b runs on XCD b % 8): they share weights and rows in its L2
  const int64_t tiles = (int64_t)total * ntiles;
  const int64_t per = (tiles + 7) / 8;
  const int64_t slot = blockIdx.x / 8;
  const int64_t tile = (int64_t)(blockIdx.x % 8) * per + slot;
  if (slot >= per || tile >= tiles) return;                    // the whole workgroup
#pragma unroll
  for (int i = 0; i < GPT; ++i) {
    const int64_t first = (int64_t)excl * ntiles, last = (int64_t)(excl + mt[i]) * ntiles;
    if (tile >= first && tile < last) {
      s_own[0] = tid * GPT + i;
      s_own[1] = (int)((tile - first) % mt[i]);
      s_own[2] = (int)((tile - first) / mt[i]);
    }
    excl += mt[i];
  }
  __syncthreads();
  const int g = __builtin_amdgcn_readfirstlane(s_own[0]);
  const int tm = __builtin_amdgcn_readfirstlane(s_own[1]);
  const int tn = __builtin_amdgcn_readfirstlane(s_own[2]);
  int64_t seg_a, seg_b;
  segment(g, seg_a, seg_b);
  const int64_t row0 = seg_a + (int64_t)tm * T::BM;
  const int rows = (int)min((int64_t)T::BM, seg_b - row0);     // live rows, >= 1
  const int feat0 = tn * FEAT;

  // ---- slice copies ----
  const int KB = K / 32;                                       // blocks of a row
  const int nk = (K + kSlice - 1) / kSlice;
  const int64_t wrow0 = (int64_t)g * (SWIGLU ? 2 * (int64_t)N : N);
  const int64_t xbytes = FMT == MX_E4M3 ? K : K / 2, wbytes = K / 2;
  // weight row (of the group) of the stage's row i: plain, or per wave 32 gate and 32 up rows
  auto weight_row = [&](int i) -> int64_t {
    if constexpr (SWIGLU) {
      const int f = min(feat0 + (i / 64) * 32 + (i & 31), N - 1);
      return wrow0 + ((i & 32) ? N + f : f);
    } else {
      return wrow0 + min(feat0 + i, N - 1);
    }
  };
  // each wave's share of a stage: copies wave, wave + WAVES, ... of the token rows, the weights and the
  // scales; the sources of slice 0, which move by the same step each slice
  constexpr int MINE = (T::COPIES + T::WAVES - 1) / T::WAVES;
  const char* src[MINE];
  int kofs[MINE];                                              // first K value (copies of 16 bytes) or block
#pragma unroll
  for (int c = 0; c < MINE; ++c) {
    const int id = wave + c * T::WAVES;
    src[c] = nullptr;
    kofs[c] = 0;
    if (id < T::NX) {
      const int byte = id * 1024 + lane * 16, r = byte / T::XROW, ch = mx_chunk<T::XROW>(r, (byte % T::XROW) / 16);
      src[c] = (const char*)p.X + (row0 + min(r, rows - 1)) * xbytes + ch * 16;
      kofs[c] = ch * (FMT == MX_E4M3 ? 16 : 32);
    } else if (id < T::NX + T::NW) {
      const int byte = (id - T::NX) * 1024 + lane * 16, r = byte / 64, ch = mx_chunk<64>(r, (byte % 64) / 16);
      src[c] = (const char*)p.W + weight_row(r) * wbytes + ch * 16;
      kofs[c] = ch * 32;
    } else if (id < T::COPIES) {
      const int r = (id - T::NX - T::NW) * 64 + lane;          // rows of X, then of W (and a few more)
      src[c] = r < T::BM ? (const char*)p.X_scales + (row0 + min(r, rows - 1)) * KB
                         : (const char*)p.W_scales + weight_row(r - T::BM) * KB;
    }
  }
  auto stage = [&](int s, int ring) {
    char* base = smem + ring * T::STAGE;
#pragma unroll
    for (int c = 0; c < MINE; ++c) {
      const int id = wave + c * T::WAVES;                      // wave-uniform
      if (id < T::NX + T::NW) {
        const bool x = id < T::NX;
        const int64_t step = x ? (FMT == MX_E4M3 ? 128 : 64) : 64;
        const char* q = src[c] + s * step;
        if constexpr (!WHOLE) {
          if (s * kSlice + kofs[c] >= K) q = (const char*)g_zero_chunk;
        }
        dma16_v(q, (bf16_t*)(base + id * 1024));
      } else if (id < T::COPIES) {
        char* dst = base + T::X_BYTES + T::W_BYTES + (id - T::NX - T::NW) * 256;
        if constexpr (WHOLE) {
          dma4_v(src[c] + s * 4, dst);
        } else {
          // scales past the row's end are zeros, never the next row's bytes (255 would make NaN of zeros)
          uint32_t v = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (s * 4 + j < KB) v |= (uint32_t)(uint8_t)src[c][s * 4 + j] << (8 * j);
          *reinterpret_cast<uint32_t*>(dst + lane * 4) = v;
        }
      }
    }
  };

  // ---- K loop ----
  // copies that every wave issues per stage at least: the wait counts by these
  constexpr int PER_WAVE = (WHOLE ? T::COPIES : T::NX + T::NW) / T::WAVES;
  const int wm = wave / T::N_WAVES, wn = wave % T::N_WAVES;
  const int r = lane & 31, q = lane >> 5;
  f32x16 acc[2][MT];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.f;

#pragma unroll
  for (int s = 0; s < T::STAGES - 1; ++s)
    if (s < nk) stage(s, s);
  int ring = 0;
  for (int s = 0; s < nk; ++s) {
    // slice s has landed once at most the copies of the slices behind it are in flight
    if (s + T::STAGES - 1 <= nk) wait_vmcnt<(T::STAGES - 2) * PER_WAVE>();
    else wait_vmcnt<0>();
    lds_barrier();                     // every wave's copies, and its reads of the stage filled next
    if (s + T::STAGES - 1 < nk) stage(s + T::STAGES - 1, ring == 0 ? T::STAGES - 1 : ring - 1);
    const char* X = smem + ring * T::STAGE;
    const char* W = X + T::X_BYTES;
    const uint32_t* S = reinterpret_cast<const uint32_t*>(W + T::W_BYTES);
    int sx[MT], sw[2];
#pragma unroll
    for (int m = 0; m < MT; ++m) sx[m] = (int)(S[(wm * MT + m) * 32 + r] >> (8 * q));
#pragma unroll
    for (int n = 0; n < 2; ++n) sw[n] = (int)(S[T::BM + wn * 64 + n * 32 + r] >> (8 * q));
    static_for<2>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
      i32x8 w[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int row = wn * 64 + n * 32 + r;
        const u32x4 v = ld16(W + row * 64 + mx_chunk<64>(row, 2 * j + q) * 16);
        w[n] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int row = (wm * MT + m) * 32 + r;
        i32x8 x;
        if constexpr (FMT == MX_E4M3) {
          const u32x4 lo = ld16(X + row * 128 + mx_chunk<128>(row, 4 * j + q) * 16);
          const u32x4 hi = ld16(X + row * 128 + mx_chunk<128>(row, 4 * j + 2 + q) * 16);
          x = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
        } else {
          const u32x4 v = ld16(X + row * 64 + mx_chunk<64>(row, 2 * j + q) * 16);
          x = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
          acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[n], x, acc[n][m], 4, FMT == MX_E4M3 ? 0 : 4,
                                                                      2 * j, sw[n], 2 * j, sx[m]);
      }
    });
    ring = ring == T::STAGES - 1 ? 0 : ring + 1;
  }

  // ---- results: lane (r, q) holds features 8 g + 4 q + i (g, i < 4) of row r of each tile ----
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int local = (wm * MT + m) * 32 + r;
    const int64_t row = row0 + local;
    if constexpr (SWIGLU) {
      const int f0 = feat0 + wn * 32;
      float a[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float h = acc[0][m][i], u = acc[1][m][i];
        a[i] = h / (1.0f + expf(-h)) * u;
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
    } else {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int f0 = feat0 + wn * 64 + n * 32;
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
hipError_t launch_as(const MxGemmProblem& p, hipStream_t stream) {
  static OccCache cache;
  hipError_t err = hipSuccess;
  const void* fn = reinterpret_cast<const void*>(&k_mx_gemm<T, SWIGLU, WHOLE>);
  if (kernel_occupancy(cache, fn, T::NTH, T::LDS, err) <= 0) return err;
  constexpr int FEAT = SWIGLU ? T::BN / 2 : T::BN;
  const int64_t ntiles = (p.N + FEAT - 1) / FEAT;
  // every group adds at most one partial tile
  int64_t mtiles = p.max_rows / T::BM + (p.groups < p.max_rows ? p.groups : p.max_rows);
  if (p.seg_stride > 0) mtiles = (int64_t)p.groups * ((p.seg_stride + T::BM - 1) / T::BM);
  const int64_t blocks = (mtiles * ntiles + 7) / 8 * 8;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_mx_gemm<T, SWIGLU, WHOLE>), dim3((unsigned)blocks), dim3(T::NTH), T::LDS, stream, p);
  return hipGetLastError();
}

template <class T>
hipError_t launch_tile(const MxGemmProblem& p, hipStream_t stream) {
  const bool whole = p.K % kSlice == 0;    // no slice has a row's end inside
  if (p.swiglu) return whole ? launch_as<T, true, true>(p, stream) : launch_as<T, true, false>(p, stream);
  return whole ? launch_as<T, false, true>(p, stream) : launch_as<T, false, false>(p, stream);
}

template <int FMT>
hipError_t launch_format(const MxGemmProblem& p, hipStream_t stream) {
  const int64_t per_group = p.max_rows / p.groups;             // the rows themselves stay on the device
  if (per_group > 128) return launch_tile<MxTile<FMT, 2, 4, 4, 3>>(p, stream);
  if (per_group > 32) return launch_tile<MxTile<FMT, 2, 4, 2, 3>>(p, stream);
  return launch_tile<MxTile<FMT, 1, 4, 1, 4>>(p, stream);
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmProblem& p, hipStream_t stream) {
  if (p.groups < 1 || p.groups > kMaxGroups || p.K % 32 || p.N % 32) return hipErrorInvalidValue;
  return p.format == MX_E4M3 ? launch_format<MX_E4M3>(p, stream) : launch_format<MX_E2M1>(p, stream);
}

}  // namespace moe
