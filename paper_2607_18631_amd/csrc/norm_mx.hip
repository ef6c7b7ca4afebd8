// Block-scaled conversion, and the residual addition + RMS norm in front of a layer.
//
// Conversion.  A thread owns 8 neighbouring values (one 16-byte vector of bf16), a quad of lanes one
// block of 32: the block's largest magnitude is two DPP exchanges away.  One pass over the data.
//
// Norm.  h = bf16(x + r), rstd = 1 / sqrt(mean(h^2) + eps), y = bf16(h rstd gamma): a row stays in
// registers between its sum of squares and its scaling, so x and r are read once and h, y and the
// 8-bit form of y are written once.  Rows of up to 2048 values belong to one wave (no barrier), longer
// ones to a workgroup of 256 (one barrier); a row past 16384 values is read again from h.
//
// Norm backward.  With u = h rstd, g = dy gamma: dx = rstd (g - u mean(g u)) + dh, and dgamma = sum over
// rows of dy u.  A wave or workgroup walks rows and keeps the dgamma sums of its columns in registers;
// each workgroup leaves one row of partial sums, which a second kernel adds in a fixed order (a single workgroup writes
// dgamma itself).
//
// All of them are bound by memory.  Measured (bytes read and written over the time; a large copy runs at 5.1 - 5.5 TB/s):
// conversion of 131072 x 7168 to e2m1 and back 841 us, 5.1 TB/s; norm of 8192 x 7168 with both results 98 us, 5.4 TB/s;
// norm and backward of 16384 x 2048 106 us, 4.4 TB/s, of 3001 x 2040 26.5 us (three launches), 3.2 TB/s; one row 4.5 us,
// a launch.
#include "common.hpp"
#include "kernels.hpp"
#include "mx_device.hpp"

namespace moe {
namespace {

constexpr int kThreads = 256;

// ---------------- conversion ----------------
constexpr int kUnroll = 4;    // vectors in flight per thread

template <int FMT>
__global__ __launch_bounds__(kThreads) void k_mx_quantize(MxConvertProblem p) {
  const int64_t nv = p.n / 8;                                 // vectors; a multiple of 4
  const int64_t base = (int64_t)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
  u32x4 v[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = base + u * kThreads;
    v[u] = i < nv ? ld16(p.x + i * 8) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = base + u * kThreads;
    float f[8];
    unpack8(v[u], f);
    // a quad's four vectors are one block, and in range or not together
    const uint32_t s = mx_scale_byte<FMT>(quad_max(abs_max_bits(f)));
    if (i < nv) {
      if constexpr (FMT == MX_E2M1) {
        reinterpret_cast<uint32_t*>(p.elements)[i] = mx_pack8_e2m1(f, s);
      } else {
        u32x2 w = {mx_pack4_e4m3(f[0], f[1], f[2], f[3], s), mx_pack4_e4m3(f[4], f[5], f[6], f[7], s)};
        reinterpret_cast<u32x2*>(p.elements)[i] = w;
      }
      if ((threadIdx.x & 3) == 0) p.scales[i / 4] = (uint8_t)s;
    }
  }
}

// bf16 of 8 elements; the products with the scale are exact in float32, one rounding to bf16
template <int FMT>
__device__ __forceinline__ u32x4 mx_values8(const uint32_t* w, uint32_t s) {
  const float scale = mx_scale(s);
  u32x4 r;
  if constexpr (FMT == MX_E2M1) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 3));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      r[2 * i] = pack_bf16x2(lo[0] * scale, lo[1] * scale);
      r[2 * i + 1] = pack_bf16x2(hi[0] * scale, hi[1] * scale);
    }
  }
  if (s == 255u) r = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
  return r;
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize(MxConvertProblem p) {
  constexpr int W = FMT == MX_E2M1 ? 1 : 2;                   // dwords per 8 elements
  const int64_t nv = p.n / 8;
  const int64_t base = (int64_t)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
  uint32_t w[kUnroll][W], s[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = min(base + u * kThreads, nv - 1);
    if constexpr (W == 1) {
      w[u][0] = reinterpret_cast<const uint32_t*>(p.elements)[i];
    } else {
      const u32x2 q = reinterpret_cast<const u32x2*>(p.elements)[i];
      w[u][0] = q[0];
      w[u][1] = q[1];
    }
    s[u] = p.scales[i / 4];
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = base + u * kThreads;
    if (i < nv) st16(p.out + i * 8, mx_values8<FMT>(w[u], s[u]));
  }
}

// ---------------- norm ----------------
using moe::wave_sum;                                          // (float32: a sum of another type would hide it)
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Sum over the threads of a row: a wave (TPR = 64), or the workgroup through LDS (one slot per wave,
// two sets used in turn so that consecutive calls need one barrier each).
template <int TPR, class F>
__device__ __forceinline__ F row_sum(F v, F* s_part, int set) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    F* q = s_part + set * NW;
    if ((threadIdx.x & 63) == 0) q[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += q[w];
  }
  return v;
}

// Forward: the sum of squares, rstd and the product in float64, so that y is the bf16 of the float64 result's float32 for
// rows of any finite size (float32 has no room for h * gamma of large rows, or for rstd of subnormal ones).  A block's 8-bit
// form turns on y's last bit: its scale doubles where its largest value rounds up to a power of two, and all 32 elements
// change with it.  (Hidden behind the memory, and as fast as float32 products with a second, float64 look at those next to a
// border between two bf16 values: 8192 rows of 7168 99 us either way, one row 4.2 against 4.4, 3001 of 2040 10.6 against 10.7.)
__device__ __forceinline__ double row_rstd(double sum, const AddNormProblem& p) {
  return 1.0 / sqrt(sum / p.d + (double)p.eps);
}
// scaled values of one vector: y and its 8-bit form
__device__ __forceinline__ void norm_store(const AddNormProblem& p, int64_t at, const float (&f)[8], double rstd,
                                           u32x4 gamma, bool live) {
  float g[8], y[8];
  unpack8(gamma, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = (float)((double)f[j] * (double)g[j] * rstd);   // (f g is exact)
  const u32x4 yb = pack8(y);
  if (live && p.y) st16(p.y + at, yb);
  if (p.y_q) {
    unpack8(yb, y);                                           // the 8-bit form is of the bf16 values
    const uint32_t s = mx_scale_byte<MX_E4M3>(quad_max(abs_max_bits(y)));
    if (live) {
      u32x2 w = {mx_pack4_e4m3(y[0], y[1], y[2], y[3], s), mx_pack4_e4m3(y[4], y[5], y[6], y[7], s)};
      *reinterpret_cast<u32x2*>(p.y_q + at) = w;
      if ((threadIdx.x & 3) == 0) p.y_scales[at / 32] = (uint8_t)s;
    }
  }
}

// TPR threads per row, up to VPT vectors of 8 values per thread
template <int TPR, int VPT>
__global__ __launch_bounds__(kThreads) void k_add_norm(AddNormProblem p) {
  constexpr int RPB = kThreads / TPR;
  __shared__ double s_part[2 * (kThreads / 64)];
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (row >= p.rows) return;                                  // whole waves (TPR = 64), or the whole workgroup
  const int nv = p.d / 8;
  const int64_t at = row * p.d;
  u32x4 a[VPT], b[VPT], gm[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = min(t + i * TPR, nv - 1);
    a[i] = ld16(p.x + at + v * 8);
    if (p.residual) b[i] = ld16(p.residual + at + v * 8);
    gm[i] = ld16(p.gamma + v * 8);
  }
  double sq = 0;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = t + i * TPR;
    if (p.residual) {
      float f[8], r[8];
      unpack8(a[i], f);
      unpack8(b[i], r);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] += r[j];
      a[i] = pack8(f);
      if (v < nv) st16(p.h + at + v * 8, a[i]);
    }
    if (v < nv) {
      float f[8];
      unpack8(a[i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) sq = fma((double)f[j], (double)f[j], sq);
    }
  }
  const double rstd = row_rstd(row_sum<TPR>(sq, s_part, 0), p);
  if (p.rstd && t == 0) p.rstd[row] = (float)rstd;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = t + i * TPR;
    float f[8];
    unpack8(a[i], f);
    norm_store(p, at + (int64_t)v * 8, f, rstd, gm[i], v < nv);
  }
}

// rows too long for the registers of a workgroup: h (or x) is read a second time, each vector by the
// thread that wrote it
__global__ __launch_bounds__(kThreads) void k_add_norm_long(AddNormProblem p) {
  __shared__ double s_part[2 * (kThreads / 64)];
  const int64_t row = blockIdx.x;
  const int nv = p.d / 8;
  const int64_t at = row * p.d;
  double sq = 0;
  for (int v = threadIdx.x; v < nv; v += kThreads) {
    float f[8];
    u32x4 a = ld16(p.x + at + (int64_t)v * 8);
    unpack8(a, f);
    if (p.residual) {
      float r[8];
      unpack8(ld16(p.residual + at + (int64_t)v * 8), r);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] += r[j];
      a = pack8(f);
      st16(p.h + at + (int64_t)v * 8, a);
      unpack8(a, f);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fma((double)f[j], (double)f[j], sq);
  }
  const double rstd = row_rstd(row_sum<kThreads>(sq, s_part, 0), p);
  if (p.rstd && threadIdx.x == 0) p.rstd[row] = (float)rstd;
  const bf16_t* src = p.residual ? p.h : p.x;
  // whole quads per round: the lanes past the row take part in the block maxima
  for (int v0 = 0; v0 < nv; v0 += kThreads) {
    const int v = v0 + threadIdx.x, c = min(v, nv - 1);
    float f[8];
    unpack8(ld16(src + at + (int64_t)c * 8), f);
    norm_store(p, at + (int64_t)v * 8, f, rstd, ld16(p.gamma + (int64_t)c * 8), v < nv);
  }
}

// ---------------- norm backward ----------------
template <int TPR, int VPT, bool DH>
__global__ __launch_bounds__(kThreads) void k_add_norm_bwd(AddNormBwdProblem p) {
  constexpr int RPB = kThreads / TPR;
  __shared__ float s_part[2 * (kThreads / 64)];
  const int t = threadIdx.x % TPR;
  const int nv = p.d / 8;
  const float inv_d = 1.0f / (float)p.d;
  u32x4 gm[VPT];
  float dg[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    gm[i] = ld16(p.gamma + min(t + i * TPR, nv - 1) * 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = 0.f;
  }
  int set = 0;
  for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * RPB) {
    const int64_t at = row * p.d;
    u32x4 vy[VPT], vh[VPT], vr[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = min(t + i * TPR, nv - 1);
      vy[i] = ld16(p.dy + at + v * 8);
      vh[i] = ld16(p.h + at + v * 8);
      if constexpr (DH) vr[i] = ld16(p.dh + at + v * 8);
    }
    const float rstd = p.rstd[row];
    float c = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (t + i * TPR < nv) {
        float y[8], h[8], g[8];
        unpack8(vy[i], y);
        unpack8(vh[i], h);
        unpack8(gm[i], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float u = h[j] * rstd;
          dg[i][j] = fmaf(y[j], u, dg[i][j]);
          c = fmaf(y[j] * g[j], u, c);
        }
      }
    }
    c = row_sum<TPR>(c, s_part, set) * inv_d;
    set ^= 1;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = t + i * TPR;
      if (v < nv) {
        float y[8], h[8], g[8], r[8], o[8];
        unpack8(vy[i], y);
        unpack8(vh[i], h);
        unpack8(gm[i], g);
        if constexpr (DH) unpack8(vr[i], r);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o[j] = rstd * (y[j] * g[j] - h[j] * rstd * c);
          if constexpr (DH) o[j] += r[j];
        }
        st16(p.dx + at + v * 8, pack8(o));
      }
    }
  }
  // the workgroup's partial sums; of the only workgroup, the result
  const bool only = gridDim.x == 1;
  float* part = p.parts + (int64_t)blockIdx.x * p.d;
  if constexpr (RPB > 1) {
    // the waves' sums of the same columns, added in wave order
    __shared__ float s_dg[RPB][TPR * 8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) s_dg[threadIdx.x / TPR][j * TPR + t] = dg[i][j];
      __syncthreads();
      for (int c = threadIdx.x; c < TPR * 8; c += kThreads) {
        const int col = (i * TPR + c / 8) * 8 + c % 8;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < RPB; ++w) s += s_dg[w][(c % 8) * TPR + c / 8];
        if (col < p.d) {
          if (only) p.dgamma[col] = (bf16_t)f32_to_bf16(s);
          else part[col] = s;
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = t + i * TPR;
      if (v < nv && only) {
        st16(p.dgamma + v * 8, pack8(dg[i]));
      } else if (v < nv) {
        *reinterpret_cast<f32x4*>(part + v * 8) = f32x4{dg[i][0], dg[i][1], dg[i][2], dg[i][3]};
        *reinterpret_cast<f32x4*>(part + v * 8 + 4) = f32x4{dg[i][4], dg[i][5], dg[i][6], dg[i][7]};
      }
    }
  }
}

// rows past the registers: the partial sums live in the workgroup's row of the workspace
template <bool DH>
__global__ __launch_bounds__(kThreads) void k_add_norm_bwd_long(AddNormBwdProblem p) {
  __shared__ float s_part[2 * (kThreads / 64)];
  const int nv = p.d / 8;
  const float inv_d = 1.0f / (float)p.d;
  float* part = p.parts + (int64_t)blockIdx.x * p.d;
  for (int v = threadIdx.x; v < nv; v += kThreads)
    for (int j = 0; j < 8; ++j) part[v * 8 + j] = 0.f;
  int set = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const int64_t at = row * p.d;
    const float rstd = p.rstd[row];
    float c = 0.f;
    for (int v = threadIdx.x; v < nv; v += kThreads) {
      float y[8], h[8], g[8];
      unpack8(ld16(p.dy + at + (int64_t)v * 8), y);
      unpack8(ld16(p.h + at + (int64_t)v * 8), h);
      unpack8(ld16(p.gamma + (int64_t)v * 8), g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = h[j] * rstd;
        part[v * 8 + j] = fmaf(y[j], u, part[v * 8 + j]);
        c = fmaf(y[j] * g[j], u, c);
      }
    }
    c = row_sum<kThreads>(c, s_part, set) * inv_d;
    set ^= 1;
    for (int v = threadIdx.x; v < nv; v += kThreads) {
      float y[8], h[8], g[8], r[8], o[8];
      unpack8(ld16(p.dy + at + (int64_t)v * 8), y);
      unpack8(ld16(p.h + at + (int64_t)v * 8), h);
      unpack8(ld16(p.gamma + (int64_t)v * 8), g);
      if constexpr (DH) unpack8(ld16(p.dh + at + (int64_t)v * 8), r);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = rstd * (y[j] * g[j] - h[j] * rstd * c);
        if constexpr (DH) o[j] += r[j];
      }
      st16(p.dx + at + (int64_t)v * 8, pack8(o));
    }
  }
}

// dgamma: 32 columns per workgroup, the partial rows dealt to 8 groups of threads and the groups' sums
// added in order
__global__ __launch_bounds__(kThreads) void k_dgamma(const float* parts, int n, int d, bf16_t* dgamma) {
  __shared__ float s[8][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c;
  float a = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int r = g; r < n; r += 8) a += parts[(int64_t)r * d + col];
  }
  s[g][c] = a;
  __syncthreads();
  if (g == 0 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += s[i][c];
    dgamma[col] = (bf16_t)f32_to_bf16(t);
  }
}

constexpr int kWaveRow = 2048;      // longest row of one wave (4 vectors per lane)
constexpr int kBlockRow = 16384;    // longest row of a workgroup's registers (8 vectors per thread)

}  // namespace

// A launch has less than 2^32 threads; what needs more goes in parts of this many workgroups.
constexpr int64_t kMostBlocks = int64_t(1) << 23;

namespace {
template <class T>
T* rows_on(T* p, int64_t values) {
  return p ? p + values : p;
}
template <class Launch>
hipError_t convert_parts(MxConvertProblem p, Launch&& launch) {
  const int64_t per = (int64_t)kThreads * kUnroll * 8, most = kMostBlocks * per;
  for (int64_t left = p.n; left > 0; left -= most) {
    p.n = left < most ? left : most;
    launch(p, dim3((unsigned)((p.n + per - 1) / per)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.x = rows_on(p.x, most);
    p.out = rows_on(p.out, most);
    p.elements += p.format == MX_E2M1 ? most / 2 : most;
    p.scales += most / 32;
  }
  return hipSuccess;
}
}  // namespace

hipError_t launch_mx_quantize(const MxConvertProblem& p, hipStream_t stream) {
  return convert_parts(p, [&](const MxConvertProblem& q, dim3 blocks) {
    if (q.format == MX_E2M1)
      hipLaunchKernelGGL(k_mx_quantize<MX_E2M1>, blocks, dim3(kThreads), 0, stream, q);
    else
      hipLaunchKernelGGL(k_mx_quantize<MX_E4M3>, blocks, dim3(kThreads), 0, stream, q);
  });
}

hipError_t launch_mx_dequantize(const MxConvertProblem& p, hipStream_t stream) {
  return convert_parts(p, [&](const MxConvertProblem& q, dim3 blocks) {
    if (q.format == MX_E2M1)
      hipLaunchKernelGGL(k_mx_dequantize<MX_E2M1>, blocks, dim3(kThreads), 0, stream, q);
    else
      hipLaunchKernelGGL(k_mx_dequantize<MX_E4M3>, blocks, dim3(kThreads), 0, stream, q);
  });
}

namespace {
// rows_per_block rows per workgroup
template <class Kernel>
hipError_t norm_parts(Kernel kernel, int rows_per_block, AddNormProblem p, hipStream_t stream) {
  const int64_t most = kMostBlocks * rows_per_block;
  for (int64_t left = p.rows; left > 0; left -= most) {
    p.rows = left < most ? left : most;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.rows + rows_per_block - 1) / rows_per_block)), dim3(kThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.x += most * p.d;
    p.residual = rows_on(p.residual, most * p.d);
    p.h = rows_on(p.h, most * p.d);
    p.y = rows_on(p.y, most * p.d);
    p.y_q = rows_on(p.y_q, most * p.d);
    p.y_scales = rows_on(p.y_scales, most * (p.d / 32));
    p.rstd = rows_on(p.rstd, most);
  }
  return hipSuccess;
}
template <int TPR, int VPT>
hipError_t norm_as(const AddNormProblem& p, hipStream_t stream) {
  return norm_parts(k_add_norm<TPR, VPT>, kThreads / TPR, p, stream);
}
template <int TPR, int VPT>
hipError_t norm_bwd_as(const AddNormBwdProblem& p, int parts, hipStream_t stream) {
  if (p.dh)
    hipLaunchKernelGGL((k_add_norm_bwd<TPR, VPT, true>), dim3(parts), dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL((k_add_norm_bwd<TPR, VPT, false>), dim3(parts), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_add_norm(const AddNormProblem& p, hipStream_t stream) {
  if (p.d <= 512) return norm_as<64, 1>(p, stream);
  if (p.d <= 1024) return norm_as<64, 2>(p, stream);
  if (p.d <= kWaveRow) return norm_as<64, 4>(p, stream);
  if (p.d <= 4096) return norm_as<256, 2>(p, stream);
  if (p.d <= 8192) return norm_as<256, 4>(p, stream);
  if (p.d <= kBlockRow) return norm_as<256, 8>(p, stream);
  return norm_parts(k_add_norm_long, 1, p, stream);
}

hipError_t launch_add_norm_bwd(const AddNormBwdProblem& p, hipStream_t stream) {
  const int parts = add_norm_bwd_parts(p.rows, p.d);
  hipError_t e;
  if (p.d <= 512) e = norm_bwd_as<64, 1>(p, parts, stream);
  else if (p.d <= 1024) e = norm_bwd_as<64, 2>(p, parts, stream);
  else if (p.d <= kWaveRow) e = norm_bwd_as<64, 4>(p, parts, stream);
  else if (p.d <= 4096) e = norm_bwd_as<256, 2>(p, parts, stream);
  else if (p.d <= 8192) e = norm_bwd_as<256, 4>(p, parts, stream);
  else if (p.d <= kBlockRow) e = norm_bwd_as<256, 8>(p, parts, stream);
  else {
    if (p.dh) hipLaunchKernelGGL(k_add_norm_bwd_long<true>, dim3(parts), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL(k_add_norm_bwd_long<false>, dim3(parts), dim3(kThreads), 0, stream, p);
    e = hipGetLastError();
  }
  // (one workgroup's sums are the result: a launch less for up to 16 rows)
  if (e != hipSuccess || (parts == 1 && p.d <= kBlockRow)) return e;
  hipLaunchKernelGGL(k_dgamma, dim3((p.d + 31) / 32), dim3(kThreads), 0, stream, p.parts, parts, p.d, p.dgamma);
  return hipGetLastError();
}

}  // namespace moe
