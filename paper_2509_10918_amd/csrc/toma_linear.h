// Pieces that the linear layer's kernels share: arguments, the epilogue's arithmetic, and the tile order.
#pragma once
#include "toma_gemm.h"
#include "toma_internal.h"
#include "toma_mx.h"

namespace toma {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// X [rows, K], W [K, N] (8-bit: [N, K]); Xs, Ws, Ys: scale codes; R, R2: residuals (R2: a second one, of the feed-forward block)
struct LinArgs {
  const void *X, *W;
  const uint8_t *Xs, *Ws;
  const void *bias, *R, *R2;
  void *Y;
  uint8_t *Ys;
  int rows, K, N, act, xs_stride, ys_stride;
};

// Activations.  fp32 outputs: gelu by the complementary error function.  bf16 and 8-bit outputs (half a step is 2^-9 of the value at
// best): v Phi(v) with Phi(v) = |s - Q(|v|)|, s = 1 for v > 0 and else 0, and the normal tail Q(a) = exp(-a^2 / 2) P(1 / (1 + 0.38 a)),
// the form of Hastings' approximations, P of degree 5 fitted to a relative error of 2^-14.8 over all a >= 0; nothing cancels, and the
// result is off by 2^-14.3 of itself at most down to v = -12.  (As v / 2 + |v| (1/2 - Q) it was off by 4 % at -5 and zero from -5.75
// on.)  11 instructions and two transcendental ones instead of the error function's about 60, with which a 256 x 256 tile's
// epilogue was as long as ten K steps.
template <bool F32> __device__ __forceinline__ float gelu_f32(float v) {
  if constexpr (F32) return 0.5f * v * erfcf(v * -0.70710678118654752f);
  const float k = v * 0.84932180028802f;  // sqrt(log2(e) / 2)
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.44741580910612f, __builtin_fabsf(k), 1.0f));  // 0.38 |v|
  float p = __builtin_fmaf(-0.08992693573f, t, 0.18887339532f);
  p = __builtin_fmaf(p, t, 0.09198205173f);
  p = __builtin_fmaf(p, t, 0.15782876313f);
  p = __builtin_fmaf(p, t, 0.15122520924f);
  const float e = __builtin_amdgcn_exp2f(-(k * k)), s = __builtin_amdgcn_fmed3f(v * 0x1p126f, 0.0f, 1.0f);
  return v * __builtin_fabsf(__builtin_fmaf(-(p * t), e, s));
}
// v / (1 + exp(-u)).  fp32 outputs: by the library's exponential and quotient.  The exponential instruction's argument, u log2(e) rounded,
// is off by a few |u| 2^-24 (silu 16 times fp32's accuracy at -20), and a reciprocal below 2^-126 comes as zero (silu from -87.3 on);
// both are far below half a step of bf16.
template <bool F32> __device__ __forceinline__ float gate_f32(float v, float u) {
  if constexpr (F32) return v / (1.0f + expf(-u));
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
      v[i] = gate_f32<F32>(v[i], v[i] * __builtin_fmaf(0.0713548162726f * v[i], v[i], 1.5957691216057308f));
  } else if (act == TOMA_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = gate_f32<F32>(v[i], v[i]);
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

enum { LIN_BF16 = 0, LIN_MX = 1 };

constexpr uint32_t kNoPacket = 0x80000000u;  // lane offset of a packet that is not there: zeros (tiles span less than 2^30 bytes)
constexpr uint32_t kAllPackets = 0x40000000u;
typedef __attribute__((address_space(3))) const uint8_t *lds_ptr;
typedef __attribute__((address_space(3))) const u32x4 *lds_u32x4_ptr;
typedef __attribute__((address_space(3))) const u32x2 *lds_u32x2_ptr;
typedef __attribute__((address_space(3))) const uint32_t *lds_u32_ptr;
typedef s16x4 __attribute__((address_space(3))) *lds_s16x4_ptr;

// One load-to-LDS instruction through a buffer descriptor: lane l's 16 bytes at base + off land at lds_addr + 16 l, zeros for a lane
// whose offset is kNoPacket or beyond `bytes` (base, bytes, lds_addr: uniform).
__device__ __forceinline__ u32x4 buffer_of(const uint8_t *base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return (u32x4){(uint32_t)b, (uint32_t)(b >> 32), bytes, 0x00020000u};
}
__device__ __forceinline__ void buffer_to_lds16(const uint8_t *base, uint32_t bytes, uint32_t off, uint32_t lds_addr) {
  const u32x4 rsrc = buffer_of(base, bytes);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(off), "s"(rsrc) : "memory", "m0");
}
// workgroup barrier that the compiler may not move memory accesses across
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ i32x8 join_halves(u32x4 a, u32x4 b) {
  return __builtin_bit_cast(i32x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// half e of a bf16 fragment pair
__device__ __forceinline__ bf16x8 bf16_half(const i32x8 &v, int e) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 h = e ? __builtin_shufflevector(v, v, 4, 5, 6, 7) : __builtin_shufflevector(v, v, 0, 1, 2, 3);
  return __builtin_bit_cast(bf16x8, h);
}
// byte g of d[0] and of d[1] (masked) as the low bytes of a word
__device__ __forceinline__ uint32_t gather_bytes(const uint32_t (&d)[2], uint32_t mask, int g) {
  const uint32_t sel = (uint32_t)g | (uint32_t)(4 + g) << 8;  // byte g of the second, then of the first operand
  return __builtin_amdgcn_perm(d[1] & mask, d[0] & mask, sel) & 0xffffu;
}
// Turns a 4 x 4 matrix of bytes over between a word's bytes and the four lane groups: byte b of the result is byte g of the word
// of lane group b (same lane of the group).  Halves of the wave first: a word's two bytes for either group of the half, from
// both halves' words; then the groups of a half.
__device__ __forceinline__ uint32_t turn_selector(int k) {  // bytes k, k + 1 of the second and of the first operand, alternating
  return (uint32_t)k * 0x01010101u + 0x05010400u;
}
__device__ __forceinline__ uint32_t turn_bytes(uint32_t d, uint32_t pairs, uint32_t own) {
  const auto h = __builtin_amdgcn_permlane32_swap(d, d, false, false);
  const uint32_t p = __builtin_amdgcn_perm(h[1], h[0], pairs);
  const auto r = __builtin_amdgcn_permlane16_swap(p, p, false, false);
  return __builtin_amdgcn_perm(r[1], r[0], own);
}
// place of packet pi of k-row k in a k-major stage of PPR packets a row: four rows of 32 bytes that a transpose read takes together
// fall on the four quarters of 256 bytes, the rows eight further on (the upper half of the wave) on what they leave
template <int PPR> __device__ __forceinline__ int km_place(int k, int pi) {
  if constexpr (PPR >= 16) return pi ^ ((k & 3) << 2) ^ (((k >> 3) & 1) << 1);
  return pi ^ (((k >> 1) & 1) << 2) ^ (((k >> 3) & 1) << 1);
}

// Epilogue of a wave's tile of TM x TN accumulators (lane: row 16 i + lane % 16, columns 16 j + 4 (lane / 16) + r) at (m_w, n_w).
// Through LDS (tl: kEpilogueFloats of the wave's own), 32 rows at a time, so that a row's columns are stored as whole 16-byte
// packets side by side.
template <int TN> constexpr int kEpilogueFloats = 32 * (16 * TN + 4);
template <int TM, int TN, bool MX_OUT>
__device__ __forceinline__ void linear_epilogue(const LinArgs &a, const f32x4 (&acc)[TM][TN], float *tl, int m_w, int n_w, int lane) {
  constexpr int LD = 16 * TN + 4;               // floats
  constexpr int LPR = 2 * TN, RPP = 64 / LPR;   // lanes per row, rows per pass
  const int g = lane >> 4, c = lane & 15, er = lane / LPR, ec = (lane % LPR) * 8, n = n_w + ec;
  F8 bias;
#pragma unroll
  for (int i = 0; i < 8; i++) bias.v[i] = 0.0f;
  if (a.bias && n < a.N) bias = load8(static_cast<const bf16_t *>(a.bias) + n);
#pragma unroll
  for (int i = 0; i < TM; i += 2) {
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int j = 0; j < TN; j++) *reinterpret_cast<f32x4 *>(tl + (16 * h + c) * LD + 16 * j + 4 * g) = acc[i + h][j];
    // (a wave's own rows: its LDS operations complete in order)
    asm volatile("" ::: "memory");
    // a lane's rows of the pass: residuals first, all on their way together
    constexpr int NP = 32 / RPP;
    const int mi = m_w + 16 * i + er;
    Pkt res[NP], res2[NP];
#pragma unroll
    for (int p = 0; p < NP; p++) {
      const size_t at = (size_t)min(mi + p * RPP, a.rows - 1) * a.N + min(n, a.N - 8);
      if (a.R) res[p] = pkt_load(static_cast<const bf16_t *>(a.R) + at);
      if (a.R2) res2[p] = pkt_load(static_cast<const bf16_t *>(a.R2) + at);
    }
#pragma unroll
    for (int p = 0; p < NP; p++) {
      const int m = mi + p * RPP;
      F8 v = load8(tl + (p * RPP + er) * LD + ec);
#pragma unroll
      for (int e = 0; e < 8; e++) v.v[e] += bias.v[e];
      activate<false>(v.v, a.act);
      if (a.R) add8(v, res[p]);
      if (a.R2) add8(v, res2[p]);
      const bool in = m < a.rows && n < a.N;
      const size_t at = (size_t)m * a.N + n;
      if constexpr (MX_OUT) {  // N % 32 == 0: a quad's 32 columns are in or out together
        u32x2 o;
        const uint32_t code = mx_pack_quad(v, o);
        if (in) *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.Y) + at) = o;
        if (in && (lane & 3) == 0) {
          uint8_t *s = a.Ys + (size_t)m * a.ys_stride + (n >> 5);
          *s = (uint8_t)code;
          if (n + 32 == a.N)  // the last block writes the padding's codes
            for (int e = 1; (n >> 5) + e < a.ys_stride; e++) s[e] = 0;
        }
      } else if (in) {
        store8(static_cast<bf16_t *>(a.Y) + at, v);
      }
    }
    asm volatile("" ::: "memory");
  }
}

// 128 x 128 tiles, at most one for every CU: four stages instead of two
inline bool medium_alone(int rows, int N) { return (long long)((rows + 127) / 128) * ((N + 127) / 128) <= 256; }

// part: fp32 scratch [nsplit][rows][N] when nsplit > 1
void launch_linear_small(const LinArgs &a, bool mx_out, int nsplit, float *part, hipStream_t st);
void launch_linear_tile(int kind, bool large, const LinArgs &a, bool mx_out, hipStream_t st);

}  // namespace toma
