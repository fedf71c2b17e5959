// Linear layer with its epilogue, Y = act(X W + bias) + R: which kernel a shape takes, and the fp32 and small bf16 products.
#include <stdlib.h>
#include <algorithm>

#include "toma_linear.h"

namespace toma {

// fp32, and bf16 with few tiles: the tiled product of the other stages with this epilogue.
template <typename T> struct EpiPol {
  static constexpr bool A_KS = false, B_KS = true, SPLIT_K = true, ACC_T = true;
  static constexpr int EPI = 1;
  static constexpr bool EPI_LDS = false;
  const T *In, *Wt, *bias, *R, *R2;
  T *Out;
  float *part;
  int rows, K, N, act;
  __device__ __forceinline__ GemmCtx setup(int) const { return GemmCtx{rows, N, K, 0, 0, 0}; }
  __device__ __forceinline__ bool a_linear(int) const { return true; }
  __device__ __forceinline__ bool b_linear(int) const { return true; }
  __device__ __forceinline__ const T *a_ptr(const GemmCtx &, int m, int k) const { return In + (size_t)m * K + k; }
  __device__ __forceinline__ const T *b_ptr(const GemmCtx &, int n, int k) const { return Wt + (size_t)k * N + n; }
  __device__ __forceinline__ float *split_buffer() const { return part; }
  // four columns n .. n + 3 of row m; b: their bias
  __device__ __forceinline__ void put(int m, int n, f32x4 v, const f32x4 &b) const {
    float e[4] = {v[0] + b[0], v[1] + b[1], v[2] + b[2], v[3] + b[3]};
    activate<sizeof(T) == 4>(e, act);
    v = (f32x4){e[0], e[1], e[2], e[3]};
    const size_t at = (size_t)m * N + n;
    if (R) v += load4(R + at);
    if (R2) v += load4(R2 + at);
    store4<T>(Out + at, v);
  }
  __device__ __forceinline__ f32x4 bias4(int n) const { return bias ? load4(bias + n) : (f32x4){0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void finish(const GemmCtx &, int m, int n, const f32x4 &v) const { put(m, n, v, bias4(n)); }
  template <int TM, int TN>
  __device__ __forceinline__ void epilogue(const GemmCtx &x, const WaveAccT<TM, TN> &acc, int m_w, int n_w,
                                           int lane, void *) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int j = 0; j < TN; j++) {
      const int n = n_w + 16 * j + 4 * g;
      if (n >= x.N) continue;
      const f32x4 b = bias4(n);
#pragma unroll
      for (int i = 0; i < TM; i++) {
        const int m = m_w + 16 * i + c;
        if (m < x.M) put(m, n, acc.t[i][j], b);
      }
    }
  }
};

// the planner's and the load-to-LDS path's smallest row count (rows past the end are clamped, so fewer do as well)
static int gemm_rows(int rows) { return std::max(rows, 8); }

enum Path { PATH_LARGE, PATH_MEDIUM, PATH_SMALL };
struct LinPlan { Path path; int nsplit; };

static LinPlan plan_linear(const toma_linear_desc &d) {
  const char *e = getenv("LIN_TILE");
  const int es = d.x_type == TOMA_F32 ? 4 : 2;
  if (e && d.x_type != TOMA_F32) {
    const int t = atoi(e);
    if (t == 0) return {PATH_LARGE, 1};
    if (t == 1) return {PATH_MEDIUM, 1};
    if (d.x_type == TOMA_MX8) return {PATH_SMALL, std::max(1, std::min(t - 1, (d.K + 511) / 512))};
    return {PATH_SMALL, gemm_async_fits(gemm_rows(d.rows), d.N, d.K, es) ? plan_gemm_async(gemm_rows(d.rows), d.N, d.K, 1, es, true, false, true, 1).nsplit : 1};
  }
  int nsplit = 1;
  if (d.x_type != TOMA_MX8 && gemm_async_fits(gemm_rows(d.rows), d.N, d.K, es)) nsplit = plan_gemm_async(gemm_rows(d.rows), d.N, d.K, 1, es, true, false, true, 1).nsplit;
  return {PATH_SMALL, nsplit};
}

template <typename T>
static void linear_typed(const LinArgs &a, const LinPlan &plan, float *part, hipStream_t st) {
  EpiPol<T> p{};
  p.In = static_cast<const T *>(a.X); p.Wt = static_cast<const T *>(a.W); p.bias = static_cast<const T *>(a.bias);
  p.R = static_cast<const T *>(a.R); p.R2 = static_cast<const T *>(a.R2); p.Out = static_cast<T *>(a.Y);
  p.part = part;
  p.rows = a.rows; p.K = a.K; p.N = a.N; p.act = a.act;
  launch_gemm<T>(K_LINEAR, p, gemm_rows(a.rows), a.N, a.K, 1, st);
}

size_t linear_workspace_bytes(const toma_linear_desc &d) {
  const LinPlan p = plan_linear(d);
  return p.nsplit > 1 ? (size_t)p.nsplit * gemm_rows(d.rows) * d.N * sizeof(float) : 0;
}

int launch_linear(const toma_linear_desc &d, const void *X, const void *Xs, const void *W, const void *Ws, const void *bias,
                  const void *R, const void *R2, void *Y, void *Ys, void *ws, hipStream_t st) {
  const LinArgs a{X, W, static_cast<const uint8_t *>(Xs), static_cast<const uint8_t *>(Ws), bias, R, R2, Y, static_cast<uint8_t *>(Ys),
                  d.rows, d.K, d.N, d.act, mx_scale_stride(d.K), mx_scale_stride(d.N)};
  const LinPlan plan = plan_linear(d);
  float *part = static_cast<float *>(ws);
  const bool mx_out = Ys != nullptr;
  if (plan.path != PATH_SMALL) {
    KernelTimer kt(K_LINEAR, st);
    launch_linear_tile(d.x_type == TOMA_MX8 ? LIN_MX : LIN_BF16, plan.path == PATH_LARGE, a, mx_out, st);
  } else if (d.x_type == TOMA_MX8) {
    KernelTimer kt(K_LINEAR, st);
    launch_linear_small(a, mx_out, plan.nsplit, part, st);
  } else if (d.x_type == TOMA_BF16) {
    linear_typed<bf16_t>(a, plan, part, st);
  } else {
    linear_typed<float>(a, plan, part, st);
  }
  return launch_status();
}

}  // namespace toma
