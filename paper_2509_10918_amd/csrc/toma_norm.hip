// Root-mean-square norm with the residual's addition, and the packing of 8-bit tensors.
//
//   h = x + r,  y = h rsqrt(mean h^2 + eps) gamma     (per row; r, gamma and the store of h are optional)
//
// Bound by memory: every element of x and r is read once, of h and y written once; a row lives in the registers of the
// lanes that share it between its sum of squares and its output, so nothing is read twice.
#include <type_traits>

#include "toma_internal.h"
#include "toma_mx.h"

namespace toma {

struct NormArgs {
  const void *X, *R, *gamma;
  void *H, *Y;
  uint8_t *Ys;
  int rows, C, stride;  // stride: scale codes per row
  float eps;
  double inv_C;     // 1 / C
};

// What a row shares is kept to more than fp32's accuracy: its squares are summed in fp32 eight at a time and in fp64 from there
// on, and the inverse root takes a Newton step in fp64.  Of 42 million packed outputs 20 instead of 25 then lie on the other side of
// a rounding border from the exact ones, at the same time within 1 %.
__device__ __forceinline__ float inverse_root(double v) {
  const float f = 1.0f / sqrtf((float)v);
  const double d = (double)f, n = d * (1.5 - 0.5 * v * d * d);
  return v < 3.0e38 ? (float)n : f;  // (past fp32's range: 0)
}

// L lanes share a row, each holding NP packets of eight channels (packet p of lane l: channels 8 (L p + l) ..): a wave's loads
// then cover 16 L consecutive bytes per row and packet, and all of a lane's loads are on their way together (up to eight of x and
// eight of r; packets behind the row's end repeat its last, so no load waits for a branch).  L = 256 is a whole workgroup per
// row, with one exchange of the waves' sums through LDS.
// 32768 x 1280 with residual and 8-bit output, 295 MB: 58 us; with 64 lanes a row and each load under its own branch 79 us.
template <typename T, bool MX, int L, int NP>
__global__ __launch_bounds__(256) void k_rmsnorm(const NormArgs a) {
  constexpr int kRows = 256 / L;  // rows per workgroup
  const int tid = threadIdx.x, l = tid & (L - 1);
  const long long row = (long long)blockIdx.x * kRows + tid / L;
  const bool live = row < a.rows;
  const T *X = static_cast<const T *>(a.X), *R = static_cast<const T *>(a.R), *G = static_cast<const T *>(a.gamma);
  T *H = static_cast<T *>(a.H);
  const int packets = a.C >> 3;
  const size_t base = (size_t)(live ? row : a.rows - 1) * a.C;
  F8 h[NP], r[NP];
#pragma unroll
  for (int p = 0; p < NP; p++) h[p] = load8(X + base + 8 * min(L * p + l, packets - 1));
  if (R) {
#pragma unroll
    for (int p = 0; p < NP; p++) r[p] = load8(R + base + 8 * min(L * p + l, packets - 1));
#pragma unroll
    for (int p = 0; p < NP; p++)
#pragma unroll
      for (int i = 0; i < 8; i++) h[p].v[i] += r[p].v[i];
  }
  double sum = 0.0;
#pragma unroll
  for (int p = 0; p < NP; p++) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) s = __builtin_fmaf(h[p].v[i], h[p].v[i], s);
    if (L * p + l < packets) sum += (double)s;
  }
#pragma unroll
  for (int m = 1; m < (L < 64 ? L : 64); m *= 2) sum += wave_xor_f64(sum, m);
  if constexpr (L > 64) {
    __shared__ double part[L / 64];
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < L / 64; i++) sum += part[i];
  }
  if (!live) return;  // (the quads of a row go on together)
  const float f = inverse_root(sum * a.inv_C + (double)a.eps);
#pragma unroll
  for (int p = 0; p < NP; p++) {
    const int q = L * p + l;
    const bool in = q < packets;
    if (H && in) store8(H + base + 8 * q, h[p]);
    F8 y = h[p];
    if (G) {  // (bf16: h gamma is exact unless x and r are more than eight powers of two apart)
      const F8 g = load8(G + 8 * min(q, packets - 1));
#pragma unroll
      for (int i = 0; i < 8; i++) y.v[i] *= g.v[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i++) y.v[i] *= f;
    if constexpr (MX) {
      u32x2 o;
      const uint32_t code = mx_pack_quad(y, o);  // (C % 32 == 0: a quad is in or out as a whole)
      if (in) *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.Y) + base + 8 * q) = o;
      if ((l & 3) == 0 && (q >> 2) < a.stride) a.Ys[(size_t)row * a.stride + (q >> 2)] = in ? (uint8_t)code : 0;
    } else if (in) {
      store8(static_cast<T *>(a.Y) + base + 8 * q, y);
    }
  }
}

// The fewest lanes a row that hold it in eight packets each.
template <typename T, bool MX>
static void launch_norm_typed(const NormArgs &a, hipStream_t st) {
  using std::integral_constant;
  // 8-bit outputs: the lanes also cover the padded scale codes
  const int packets = MX ? a.stride * 4 : a.C >> 3;
  auto go = [&](auto lanes, auto np) {
    constexpr int L = decltype(lanes)::value, NP = decltype(np)::value;
    const int per = 256 / L;
    hipLaunchKernelGGL((k_rmsnorm<T, MX, L, NP>), dim3((unsigned)((a.rows + (long long)per - 1) / per)), dim3(256), 0, st, a);
  };
  auto most = [&](auto lanes) {  // more than four packets a lane
    const int np = (packets + decltype(lanes)::value - 1) / decltype(lanes)::value;
    if (np <= 5) go(lanes, integral_constant<int, 5>());
    else if (np == 6) go(lanes, integral_constant<int, 6>());
    else go(lanes, integral_constant<int, 8>());
  };
  if (packets <= 8) go(integral_constant<int, 8>(), integral_constant<int, 1>());
  else if (packets <= 16) go(integral_constant<int, 8>(), integral_constant<int, 2>());
  else if (packets <= 32) go(integral_constant<int, 8>(), integral_constant<int, 4>());
  else if (packets <= 64) most(integral_constant<int, 8>());
  else if (packets <= 128) most(integral_constant<int, 16>());
  else if (packets <= 256) most(integral_constant<int, 32>());
  else if (packets <= 512) most(integral_constant<int, 64>());
  else if (packets <= 1024) go(integral_constant<int, 256>(), integral_constant<int, 4>());
  else most(integral_constant<int, 256>());
}

int launch_rmsnorm(const toma_norm_desc &d, const void *X, const void *R, const void *gamma, void *H, void *Y, void *Ys,
                   hipStream_t st) {
  NormArgs a{X, R, gamma, H, Y, static_cast<uint8_t *>(Ys), d.rows, d.C, mx_scale_stride(d.C), d.eps, 1.0 / d.C};
  KernelTimer kt(K_NORM, st);
  const bool mx = d.y_type == TOMA_MX8;
  if (d.x_type == TOMA_BF16) mx ? launch_norm_typed<bf16_t, true>(a, st) : launch_norm_typed<bf16_t, false>(a, st);
  else mx ? launch_norm_typed<float, true>(a, st) : launch_norm_typed<float, false>(a, st);
  return launch_status();
}

// ---- packing --------------------------------------------------------------------------------------------------------

// One thread per eight channels, a row padded to whole groups of 128 channels (16 threads), so that a quad of lanes is
// one block and the padding's codes have their writer.
template <typename T>
__global__ __launch_bounds__(256) void k_mx_quantize(const T *__restrict__ X, uint8_t *__restrict__ Q, uint8_t *__restrict__ S,
                                                     int rows, int K, int stride) {
  const size_t t = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int per_row = stride * 4;
  const long long row = (long long)(t / per_row);
  const int q = (int)(t - (size_t)row * per_row);
  const bool in = row < rows && 8 * q < K;
  F8 x;
#pragma unroll
  for (int i = 0; i < 8; i++) x.v[i] = 0.0f;
  if (in) x = load8(X + (size_t)row * K + 8 * q);
  u32x2 o;
  const uint32_t code = mx_pack_quad(x, o);
  if (in) *reinterpret_cast<u32x2 *>(Q + (size_t)row * K + 8 * q) = o;
  if (row < rows && (q & 3) == 0) S[(size_t)row * stride + (q >> 2)] = in ? (uint8_t)code : 0;
}

// One thread per block of 32 input channels of one output channel: the lanes of a wave read 64 consecutive output
// channels of a row of W at a time.  (Once per weight: the scattered 32-byte stores do not matter.)
template <typename T>
__global__ __launch_bounds__(256) void k_mx_quantize_weight(const T *__restrict__ W, uint8_t *__restrict__ Q,
                                                            uint8_t *__restrict__ S, int K, int N, int stride) {
  const int n = blockIdx.x * 256 + threadIdx.x, kb = blockIdx.y;
  if (n >= N) return;
  if (32 * kb >= K) {
    S[(size_t)n * stride + kb] = 0;
    return;
  }
  float x[32], m = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; i++) {
    x[i] = to_f32(W[(size_t)(32 * kb + i) * N + n]);
    m = fmaxf(m, mx_magnitude(x[i]));
  }
  const uint32_t code = mx_code(m);
  const float inv = mx_inverse(code);
  u32x4 o[2];
#pragma unroll
  for (int i = 0; i < 8; i++) o[i >> 2][i & 3] = mx_pack4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], inv);
  u32x4 *dst = reinterpret_cast<u32x4 *>(Q + (size_t)n * K + 32 * kb);
  dst[0] = o[0];
  dst[1] = o[1];
  S[(size_t)n * stride + kb] = (uint8_t)code;
}

template <typename T>
__global__ __launch_bounds__(256) void k_mx_dequantize(const uint8_t *__restrict__ Q, const uint8_t *__restrict__ S,
                                                       T *__restrict__ Y, long long packets, int K, int stride) {
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  if (t >= packets) return;
  const int per_row = K >> 3;
  const long long row = t / per_row;
  const int q = (int)(t - row * per_row);
  const u32x2 e = *reinterpret_cast<const u32x2 *>(Q + 8 * t);
  const float sc = mx_scale(S[(size_t)row * stride + (q >> 2)]);
  F8 y;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    y.v[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)e[i], 0) * sc;
    y.v[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)e[i], 1) * sc;
    y.v[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)e[i], 2) * sc;
    y.v[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)e[i], 3) * sc;
  }
  store8(Y + 8 * t, y);
}

int launch_mx_quantize(int x_type, int rows, int K, const void *X, void *Q, void *S, hipStream_t st) {
  const int stride = mx_scale_stride(K);
  const long long threads = (long long)rows * stride * 4;
  const dim3 grid((unsigned)((threads + 255) / 256));
  KernelTimer kt(K_MX_QUANTIZE, st);
  if (x_type == TOMA_BF16)
    hipLaunchKernelGGL(k_mx_quantize<bf16_t>, grid, dim3(256), 0, st, static_cast<const bf16_t *>(X), static_cast<uint8_t *>(Q), static_cast<uint8_t *>(S), rows, K, stride);
  else
    hipLaunchKernelGGL(k_mx_quantize<float>, grid, dim3(256), 0, st, static_cast<const float *>(X), static_cast<uint8_t *>(Q), static_cast<uint8_t *>(S), rows, K, stride);
  return launch_status();
}

int launch_mx_quantize_weight(int w_type, int K, int N, const void *W, void *Q, void *S, hipStream_t st) {
  const int stride = mx_scale_stride(K);
  const dim3 grid((unsigned)((N + 255) / 256), (unsigned)stride);
  KernelTimer kt(K_MX_QUANTIZE, st);
  if (w_type == TOMA_BF16)
    hipLaunchKernelGGL(k_mx_quantize_weight<bf16_t>, grid, dim3(256), 0, st, static_cast<const bf16_t *>(W), static_cast<uint8_t *>(Q), static_cast<uint8_t *>(S), K, N, stride);
  else
    hipLaunchKernelGGL(k_mx_quantize_weight<float>, grid, dim3(256), 0, st, static_cast<const float *>(W), static_cast<uint8_t *>(Q), static_cast<uint8_t *>(S), K, N, stride);
  return launch_status();
}

int launch_mx_dequantize(int y_type, int rows, int K, const void *Q, const void *S, void *Y, hipStream_t st) {
  const int stride = mx_scale_stride(K);
  const long long packets = (long long)rows * (K >> 3);
  const dim3 grid((unsigned)((packets + 255) / 256));
  KernelTimer kt(K_MX_DEQUANTIZE, st);
  if (y_type == TOMA_BF16)
    hipLaunchKernelGGL(k_mx_dequantize<bf16_t>, grid, dim3(256), 0, st, static_cast<const uint8_t *>(Q), static_cast<const uint8_t *>(S), static_cast<bf16_t *>(Y), packets, K, stride);
  else
    hipLaunchKernelGGL(k_mx_dequantize<float>, grid, dim3(256), 0, st, static_cast<const uint8_t *>(Q), static_cast<const uint8_t *>(S), static_cast<float *>(Y), packets, K, stride);
  return launch_status();
}

}  // namespace toma
