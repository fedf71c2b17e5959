// Pieces that the linear layer's kernels share: arguments, the epilogue's arithmetic, and the tile order.
#pragma once
#include "toma_gemm.h"
#include "toma_internal.h"
#include "toma_mx.h"

namespace toma {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// X [rows, K], W [K, N] (8-bit: [N, K]); Xs, Ws, Ys: scale codes; R, R2: residuals (R2: a second one, of the feed-forward block)
struct LinArgs {
  const void *X, *W;
  const uint8_t *Xs, *Ws;
  const void *bias, *R, *R2;
  void *Y;
  uint8_t *Ys;
  int rows, K, N, act, xs_stride, ys_stride;
};

// Activations.  fp32 outputs: to fp32 accuracy.  bf16 and 8-bit outputs (half a step is 2^-9 of the value at best): gelu with the
// normal tail Q(a) = 1 - Phi(a) = exp(-a^2 / 2) P(1 / (1 + 0.38 a)), P of degree 5 fitted to a relative error of 2^-14.8 over all
// a >= 0 (so small results of large negative inputs keep their relative accuracy), 13 instructions and two transcendental ones
// instead of the error function's about 60: a 256 x 256 tile's epilogue was as long as ten K steps with that.
template <bool F32> __device__ __forceinline__ float gelu_f32(float v) {
  if constexpr (F32) return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
  const float a = __builtin_fabsf(v), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.38f, a, 1.0f));
  float p = __builtin_fmaf(-0.08992693573f, t, 0.18887339532f);
  p = __builtin_fmaf(p, t, 0.09198205173f);
  p = __builtin_fmaf(p, t, 0.15782876313f);
  p = __builtin_fmaf(p, t, 0.15122520924f);
  const float q = p * t * __builtin_amdgcn_exp2f(v * v * -0.72134752044448f);  // -log2(e) / 2
  return v * (v > 0.0f ? 1.0f - q : q);
}
// v / (1 + exp(-u))
__device__ __forceinline__ float gate_f32(float v, float u) {
  return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -1.4426950408889634f));
}
template <bool F32, int N> __device__ __forceinline__ void activate(float (&v)[N], int act) {  // act: the same for all lanes
  if (act == TOMA_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = gelu_f32<F32>(v[i]);
  } else if (act == TOMA_ACT_GELU_TANH) {
    // x/2 (1 + tanh(u)) = x / (1 + exp(-2u)), u = sqrt(2/pi) (x + 0.044715 x^3)
#pragma unroll
    for (int i = 0; i < N; i++)
      v[i] = gate_f32(v[i], v[i] * __builtin_fmaf(0.0713548162726f * v[i], v[i], 1.5957691216057308f));
  } else if (act == TOMA_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = gate_f32(v[i], v[i]);
  }
}
__device__ __forceinline__ f32x4 load4(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ __forceinline__ f32x4 load4(const bf16_t *p) {
  const u32x2 r = *reinterpret_cast<const u32x2 *>(p);
  return (f32x4){__builtin_bit_cast(float, r[0] << 16), __builtin_bit_cast(float, r[0] & 0xffff0000u),
                 __builtin_bit_cast(float, r[1] << 16), __builtin_bit_cast(float, r[1] & 0xffff0000u)};
}

// Tile of a workgroup.  Ids go round the eight XCDs, so each XCD gets a contiguous run of tiles (xcd_remap); inside a run
// the tiles go down eight rows of tiles before they go right: the 32 tiles an XCD works on at a time then share 8 + 4
// operand panels in its L2 instead of 1 + 32.
__device__ __forceinline__ void tile_of(int id, int total, int tiles_m, int tiles_n, int &tm, int &tn) {
  const int t = xcd_remap(id, total), per = 8 * tiles_n, grp = t / per, in = t - grp * per;
  const int high = min(8, tiles_m - 8 * grp);
  tn = in / high;
  tm = 8 * grp + in - tn * high;
}

int launch_linear_tile(int kind, const LinArgs &a, bool mx_out, hipStream_t st);

}  // namespace toma
