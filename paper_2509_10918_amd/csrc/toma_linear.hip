// Linear layer with its epilogue: Y = act(X W + bias) + R.
#include <stdlib.h>

#include "toma_linear.h"

namespace toma {

template <typename T> struct EpiPol {
  static constexpr bool A_KS = false, B_KS = true, SPLIT_K = false, ACC_T = true;
  static constexpr int EPI = 1;
  static constexpr bool EPI_LDS = false;
  const T *In, *Wt, *bias, *R;
  T *Out;
  int rows, K, N, act;
  __device__ __forceinline__ GemmCtx setup(int) const { return GemmCtx{rows, N, K, 0, 0, 0}; }
  __device__ __forceinline__ bool a_linear(int) const { return true; }
  __device__ __forceinline__ bool b_linear(int) const { return true; }
  __device__ __forceinline__ const T *a_ptr(const GemmCtx &, int m, int k) const { return In + (size_t)m * K + k; }
  __device__ __forceinline__ const T *b_ptr(const GemmCtx &, int n, int k) const { return Wt + (size_t)k * N + n; }
  template <int TM, int TN>
  __device__ __forceinline__ void epilogue(const GemmCtx &x, const WaveAccT<TM, TN> &acc, int m_w, int n_w,
                                           int lane, void *) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int j = 0; j < TN; j++) {
      const int n = n_w + 16 * j + 4 * g;
      if (n >= x.N) continue;
      f32x4 b = (f32x4){0.f, 0.f, 0.f, 0.f};
      if (bias) b = load4(bias + n);
#pragma unroll
      for (int i = 0; i < TM; i++) {
        const int m = m_w + 16 * i + c;
        if (m >= x.M) continue;
        f32x4 v = acc.t[i][j] + b;
        float e[4] = {v[0], v[1], v[2], v[3]};
        activate<sizeof(T) == 4>(e, act);
        v = (f32x4){e[0], e[1], e[2], e[3]};
        const size_t at = (size_t)m * x.N + n;
        if (R) v += load4(R + at);
        store4<T>(Out + at, v);
      }
    }
  }
};

template <typename T>
static int linear_typed(const toma_linear_desc &d, const void *X, const void *W, const void *bias, const void *R, void *Y,
                        hipStream_t st) {
  if (sizeof(T) == 2 && !getenv("LIN_OLD")) {
    LinArgs a{X, W, nullptr, nullptr, bias, R, nullptr, Y, nullptr, d.rows, d.K, d.N, d.act, 0, 0};
    return launch_linear_tile(0, a, false, st);
  }
  EpiPol<T> p{};
  p.In = static_cast<const T *>(X); p.Wt = static_cast<const T *>(W); p.bias = static_cast<const T *>(bias);
  p.R = static_cast<const T *>(R); p.Out = static_cast<T *>(Y);
  p.rows = d.rows; p.K = d.K; p.N = d.N; p.act = d.act;
  launch_gemm<T>(K_LINEAR, p, d.rows, d.N, d.K, 1, st);
  return launch_status();
}

// ---- 8-bit products ---------------------------------------------------------------------------------------------------
// v_mfma_scale_f32_16x16x128_f8f6f4: lane l holds row / column l % 16; its first 16 bytes are k = 16 g .. 16 g + 15 and its second
// 64 + 16 g .. (g = l / 16), and the scale code it supplies is that of the block k = 32 g .. 32 g + 31.
__device__ __forceinline__ f32x4 mma_mx(const i32x8 &a, const i32x8 &b, const f32x4 &c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}

// 32 x 32 outputs per wave, fragments straight from memory.
template <bool MX_OUT>
__global__ __launch_bounds__(256) void k_linear_mx(const LinArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
  const int tiles_n = (a.N + 63) / 64;
  const int m0 = (int)(blockIdx.x / tiles_n) * 64 + (w >> 1) * 32, n0 = (int)(blockIdx.x % tiles_n) * 64 + (w & 1) * 32;
  f32x4 acc[2][2];
  const uint8_t *px[2], *pw[2], *sx[2], *sw[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int m = min(m0 + 16 * i + c, a.rows - 1), n = min(n0 + 16 * i + c, a.N - 1);
    px[i] = static_cast<const uint8_t *>(a.X) + (size_t)m * a.K; sx[i] = a.Xs + (size_t)m * a.xs_stride;
    pw[i] = static_cast<const uint8_t *>(a.W) + (size_t)n * a.K; sw[i] = a.Ws + (size_t)n * a.xs_stride;
    acc[i][0] = acc[i][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  auto half = [&](const uint8_t *p, int k) { return k < a.K ? *reinterpret_cast<const u32x4 *>(p + k) : (u32x4){0u, 0u, 0u, 0u}; };
  auto frag = [&](const uint8_t *p, int k0) {
    const u32x4 lo = half(p, k0 + 16 * g), hi = half(p, k0 + 64 + 16 * g);
    return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  for (int k0 = 0; k0 < a.K; k0 += 128) {
    i32x8 fx[2], fw[2];
    uint32_t cx[2], cw[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      fx[i] = frag(px[i], k0); fw[i] = frag(pw[i], k0);
      cx[i] = sx[i][(k0 >> 5) + g]; cw[i] = sw[i][(k0 >> 5) + g];
    }
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int j = 0; j < 2; j++) acc[i][j] = mma_mx(fw[j], fx[i], acc[i][j], cw[j], cx[i]);
  }
  // lane: row m0 + 16 i + c, columns n0 + 16 j + 4 g + r
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int m = m0 + 16 * i + c;
    f32x4 v[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int n = n0 + 16 * j + 4 * g;
      const bool in = m < a.rows && n < a.N;
      v[j] = acc[i][j];
      if (a.bias && in) v[j] += load4(static_cast<const bf16_t *>(a.bias) + n);
      float e[4] = {v[j][0], v[j][1], v[j][2], v[j][3]};
      activate<false>(e, a.act);
      v[j] = (f32x4){e[0], e[1], e[2], e[3]};
      if (a.R && in) v[j] += load4(static_cast<const bf16_t *>(a.R) + (size_t)m * a.N + n);
      if (!MX_OUT && in) store4<bf16_t>(static_cast<bf16_t *>(a.Y) + (size_t)m * a.N + n, v[j]);
    }
    if constexpr (MX_OUT) {  // N % 32 == 0: the 32 columns of this wave are in or out together
      float mx = 0.0f;
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int r = 0; r < 4; r++) mx = fmaxf(mx, mx_magnitude(v[j][r]));
      mx = fmaxf(mx, wave_xor_f32(mx, 16));
      mx = fmaxf(mx, wave_xor_f32(mx, 32));
      const uint32_t code = mx_code(mx);
      const float inv = mx_inverse(code);
      if (m < a.rows && n0 < a.N) {
#pragma unroll
        for (int j = 0; j < 2; j++)
          *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(a.Y) + (size_t)m * a.N + n0 + 16 * j + 4 * g) =
              mx_pack4(v[j][0], v[j][1], v[j][2], v[j][3], inv);
        if (g == 0) a.Ys[(size_t)m * a.ys_stride + (n0 >> 5)] = (uint8_t)code;
        // the padding's codes behind the last block
        if (n0 + 32 == a.N && g > 0 && (n0 >> 5) + g < a.ys_stride) a.Ys[(size_t)m * a.ys_stride + (n0 >> 5) + g] = 0;
      }
    }
  }
}

static int linear_mx(const toma_linear_desc &d, const void *X, const void *Xs, const void *W, const void *Ws, const void *bias,
                     const void *R, void *Y, void *Ys, hipStream_t st) {
  LinArgs a{X, W, static_cast<const uint8_t *>(Xs), static_cast<const uint8_t *>(Ws), bias, R, nullptr, Y, static_cast<uint8_t *>(Ys),
            d.rows, d.K, d.N, d.act, mx_scale_stride(d.K), mx_scale_stride(d.N)};
  if (!getenv("LIN_OLD")) return launch_linear_tile(1, a, Ys != nullptr, st);
  const dim3 grid((unsigned)(((d.rows + 63) / 64) * (long long)((d.N + 63) / 64)));
  KernelTimer kt(K_LINEAR, st);
  if (Ys) hipLaunchKernelGGL(k_linear_mx<true>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_linear_mx<false>, grid, dim3(256), 0, st, a);
  return launch_status();
}

size_t linear_workspace_bytes(const toma_linear_desc &) { return 0; }

int launch_linear(const toma_linear_desc &d, const void *X, const void *Xs, const void *W, const void *Ws, const void *bias,
                  const void *R, void *Y, void *Ys, void *, hipStream_t st) {
  if (d.x_type == TOMA_MX8) return linear_mx(d, X, Xs, W, Ws, bias, R, Y, Ys, st);
  return d.x_type == TOMA_BF16 ? linear_typed<bf16_t>(d, X, W, bias, R, Y, st) : linear_typed<float>(d, X, W, bias, R, Y, st);
}

}  // namespace toma
