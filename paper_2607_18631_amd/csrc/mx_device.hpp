// Device helpers of the block-scaled formats: 32 values share 2^e, held as the byte e + 127; elements
// are e2m1 (4 bits) or e4m3 (8 bits).
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace moe {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));

// Scale byte of a block whose largest magnitude has the float32 bits `m`: floor(log2) is the exponent
// field less 127; LEAD is that of the format's largest value.  Subnormal and zero maxima have field 0
// and land on the lowest scale; Inf and NaN give 255.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t m) {
  constexpr int LEAD = FMT == MX_E2M1 ? 2 : 8;
  const int e = (int)(m >> 23);
  if (e == 255) return 255u;
  return (uint32_t)max(e - LEAD, 0);
}
// 2^(s - 127) as float32 (s = 0 is subnormal, 255 NaN)
__device__ __forceinline__ float mx_scale(uint32_t s) {
  return __uint_as_float(s == 0 ? 0x00400000u : s == 255u ? 0x7fc00000u : s << 23);
}

// largest magnitude (float32 bits) of values in registers; integer order of |v| is float order, with
// Inf and NaN on top
template <int N>
__device__ __forceinline__ uint32_t abs_max_bits(const float (&v)[N]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
// maximum over the 4 lanes of a quad
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));   // [1,0,3,2]
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));   // [2,3,0,1]
}

// Four values over their block's scale, as 4 bytes (e4m3): round to nearest even.  The conversion
// gives NaN past the largest value, so values are cut first (448 * 2^(s - 127) is a normal float).
// A block of scale 255 gets zeros.
__device__ __forceinline__ uint32_t mx_pack4_e4m3(float a, float b, float c, float d, uint32_t s) {
  if (s == 255u) return 0u;
  const float scale = mx_scale(s);
  const float top = __uint_as_float(((s + 8u) << 23) | 0x600000u);
  a = fminf(fmaxf(a, -top), top);
  b = fminf(fmaxf(b, -top), top);
  c = fminf(fmaxf(c, -top), top);
  d = fminf(fmaxf(d, -top), top);
  s16x2_t r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// Eight values as 8 half-bytes (e2m1); this conversion cuts at the largest value by itself.
__device__ __forceinline__ uint32_t mx_pack8_e2m1(const float (&v)[8], uint32_t s) {
  if (s == 255u) return 0u;
  const float scale = mx_scale(s);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
  return r;
}

// the 8 bf16 values of a 16-byte vector as float32
__device__ __forceinline__ void unpack8(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(v[i] << 16);
    f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  return v;
}

}  // namespace moe
