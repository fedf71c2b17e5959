// 8-bit tensors with a power-of-two scale per 32 channels: the device side of packing and unpacking.
//
// A block of 32 consecutive channels of a row is packed as q = round_e4m3(x * 2^-e), with 2^e the smallest power of two
// (e >= -127) for which the largest finite |x| of the block is at most 448 * 2^e, so that no element saturates and the
// largest keeps at least three of its four significant bits' range.  The scale code is e + 127.  A value that is not finite takes
// no part in the maximum and becomes NaN in e4m3 (the conversion instruction's own overflow result).
#pragma once
#include "toma_common.h"

namespace toma {

// Scale code of a block from its largest finite magnitude: 448 = 1.75 * 2^8, so the code is the magnitude's biased
// exponent minus 8, one more where its significand exceeds 1.75 (the addition carries into the exponent exactly then).
__device__ __forceinline__ uint32_t mx_code(float amax) {
  const uint32_t e = (__builtin_bit_cast(uint32_t, amax) + 0x1fffffu) >> 23;
  return e > 8u ? e - 8u : 0u;
}
// 2^(127 - code): what the elements of the block are multiplied by (code <= 247, so a normal number)
__device__ __forceinline__ float mx_inverse(uint32_t code) { return __builtin_bit_cast(float, (254u - code) << 23); }
// 2^(code - 127)
__device__ __forceinline__ float mx_scale(uint32_t code) {
  return __builtin_bit_cast(float, code == 0 ? 0x00400000u : code << 23);
}
__device__ __forceinline__ float mx_magnitude(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
  return b < 0x7f800000u ? __builtin_bit_cast(float, b) : 0.0f;
}
__device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d, float inv) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, v, true);
  return (uint32_t)v;
}
// largest of the four lanes of a quad
__device__ __forceinline__ float quad_max_f32(float v) {
  v = fmaxf(v, dpp_f32<0xB1>(v));
  return fmaxf(v, dpp_f32<0x4E>(v));
}

// Eight consecutive channels <-> registers.
struct F8 { float v[8]; };
__device__ __forceinline__ F8 load8(const bf16_t *p) {
  const u32x4 r = *reinterpret_cast<const u32x4 *>(p);
  F8 o;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    o.v[2 * i] = __builtin_bit_cast(float, r[i] << 16);
    o.v[2 * i + 1] = __builtin_bit_cast(float, r[i] & 0xffff0000u);
  }
  return o;
}
__device__ __forceinline__ F8 load8(const float *p) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
  F8 o;
#pragma unroll
  for (int i = 0; i < 4; i++) { o.v[i] = a[i]; o.v[4 + i] = b[i]; }
  return o;
}
__device__ __forceinline__ void add8(F8 &x, const Pkt &r) {  // eight bf16
#pragma unroll
  for (int i = 0; i < 4; i++) {
    x.v[2 * i] += __builtin_bit_cast(float, r.v[i] << 16);
    x.v[2 * i + 1] += __builtin_bit_cast(float, r.v[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(bf16_t *p, const F8 &x) {
  bf16x8 o;
#pragma unroll
  for (int i = 0; i < 8; i++) o[i] = (bf16_t)x.v[i];
  *reinterpret_cast<bf16x8 *>(p) = o;
}
__device__ __forceinline__ void store8(float *p, const F8 &x) {
  f32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; i++) { a[i] = x.v[i]; b[i] = x.v[4 + i]; }
  *reinterpret_cast<f32x4 *>(p) = a;
  *reinterpret_cast<f32x4 *>(p + 4) = b;
}
// Largest finite magnitude of eight values.  The maximum drops NaN by itself; infinities are looked for only where the result is one.
__device__ __forceinline__ float mx_largest(const F8 &x) {
  float m = fmaxf(__builtin_fabsf(x.v[0]), __builtin_fabsf(x.v[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2) m = fmaxf(fmaxf(m, __builtin_fabsf(x.v[i])), __builtin_fabsf(x.v[i + 1]));  // (one max3 each)
  if (__builtin_expect(!(m < __builtin_inff()), 0)) {
    m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) m = fmaxf(m, mx_magnitude(x.v[i]));
  }
  return m;
}
// Packs a block whose 32 channels four consecutive lanes of a quad hold, eight each.  Returns the code; q: the lane's eight bytes.
__device__ __forceinline__ uint32_t mx_pack_quad(const F8 &x, u32x2 &q) {
  const uint32_t code = mx_code(quad_max_f32(mx_largest(x)));
  const float inv = mx_inverse(code);
  q[0] = mx_pack4(x.v[0], x.v[1], x.v[2], x.v[3], inv);
  q[1] = mx_pack4(x.v[4], x.v[5], x.v[6], x.v[7], inv);
  return code;
}

}  // namespace toma
