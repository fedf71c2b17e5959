// Linear layer with its epilogue, Y = act(X W + bias) + R: which kernel a shape takes, the fp32 and small bf16 products, and those
// of few rows.
#include <algorithm>
#include <cmath>

#include "toma_linear.h"

namespace toma {

// fp32, and bf16 with few tiles: the tiled product of the other stages with this epilogue.  That product takes whole K steps (128
// bytes a row): the channels behind the last whole step are added from memory when the sum is at hand, before the epilogue.
// (The register-staged kernel, which takes any K, has no K split: fp32 900 x 1000 x 1504 took it 78 us, this way 41.)
template <typename T> struct EpiPol {
  static constexpr bool A_KS = false, B_KS = true, SPLIT_K = true, ACC_T = true;
  static constexpr int EPI = 1;
  static constexpr bool EPI_LDS = false;
  const T *In, *Wt, *bias, *R, *R2;
  T *Out;
  float *part;
  int rows, K, N, act, K_steps;  // K_steps: channels in whole steps
  __device__ __forceinline__ GemmCtx setup(int) const { return GemmCtx{rows, N, K_steps, 0, 0, 0}; }
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
  __device__ __forceinline__ void finish(const GemmCtx &, int m, int n, f32x4 v) const {
    for (int k = K_steps; k < K; k++) v += to_f32(In[(size_t)m * K + k]) * load4(Wt + (size_t)k * N + n);
    put(m, n, v, bias4(n));
  }
  // the channels behind the last whole step: a fragment's eight slots (k-group g: channels k + 8 g ..) straight from memory
  template <int TM, int TN> __device__ __forceinline__ void add_tail(WaveAccT<TM, TN> &acc, int m_w, int n_w, int lane) const {
    const int g = lane >> 4, c = lane & 15;
    for (int k0 = K_steps; k0 < K; k0 += 32) {
      const int k = k0 + 8 * g;
      Frag<T> fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; i++) {
        const T *src = In + (size_t)min(m_w + 16 * i + c, rows - 1) * K;
#pragma unroll
        for (int e = 0; e < 8; e++) fa[i].v[e] = k + e < K ? src[k + e] : from_f32<T>(0.0f);
      }
#pragma unroll
      for (int j = 0; j < TN; j++) {
        const T *src = Wt + min(n_w + 16 * j + c, N - 1);
#pragma unroll
        for (int e = 0; e < 8; e++) fb[j].v[e] = k + e < K ? src[(size_t)(k + e) * N] : from_f32<T>(0.0f);
      }
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) mma16(acc.t[i][j], fb[j], fa[i]);
    }
  }
  template <int TM, int TN>
  __device__ __forceinline__ void epilogue(const GemmCtx &x, WaveAccT<TM, TN> &acc, int m_w, int n_w,
                                           int lane, void *) const {
    const int g = lane >> 4, c = lane & 15;
    if (K_steps < K) add_tail<TM, TN>(acc, m_w, n_w, lane);
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

// Few rows: bound by reading W once.  W goes from memory straight into the matrix instruction's registers: a lane takes a 16-byte
// packet of columns of KS / 4 rows of W, so tile j of the products is made of the j-th column of every packet (bf16: the rows'
// pairs of columns are regrouped by byte permutes), and its results are packets of neighbouring columns again.  The eight waves of
// a workgroup take the K steps in turn, each with DEPTH steps on their way, and add their sums up through LDS; K is split between
// workgroups as well where the columns alone are too few.  RT: tiles of 16 rows.
// Taken for every call of up to 16 rows (fp32: 32), by the row count alone.  One row, us, this kernel and the 64 x 64 tiles (K split
// planned): bf16 1280 x 5120 5.8 and 7.3, 640 x 640 4.3 and 5.4, 5120 x 1280 8.3 and 8.8; fp32 1280 x 5120 8.5 and 13.9, 640 x 640 6.1
// and 14.7, 4096 x 4096 17.0 and 26.5, 8192 x 8192 46 and 82.  32 rows: fp32 1280 x 5120 11.7 and 14.4, 8192 x 8192 56 and 82; bf16
// 1280 x 5120 8.5 and 7.8.  In bf16 the rule is not the faster one for large weights: 1 x 4096 x 4096 9.8 and 9.5, 16 rows 11.2
// and 9.6; 1 x 8192 x 8192 (134 MB) 25.5 and 23.4; 16 x 20480 x 5120 49 and 37, but 4 x 5120 x 20480 34 and 37.  The planner's estimate
// of the tiles is not fitted to so few rows, so the two are not weighed against each other.
template <typename T, int RT>
__global__ __launch_bounds__(512, 2) void k_linear_few(const EpiPol<T> p, int nsplit) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int EPL = 16 / sizeof(T), CG = 16 * EPL, KS = F32 ? 16 : 32, WR = KS / 4, NW = 8, DEPTH = F32 ? 6 : 4;
  constexpr int LD = CG + 4;  // floats
  __shared__ __align__(16) float red[NW][16 * RT][LD];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const int n0 = blockIdx.x * CG, split = blockIdx.y, steps = (p.K + KS - 1) / KS;
  const int s0 = (int)((long long)steps * split / nsplit), s1 = (int)((long long)steps * (split + 1) / nsplit);
  // (columns and rows behind the end repeat the last: their results are not stored)
  const T *wp = p.Wt + min(n0 + c * EPL, p.N - EPL) + (size_t)(WR * g) * p.N;
  const T *xp[RT];
#pragma unroll
  for (int t = 0; t < RT; t++) xp[t] = p.In + (size_t)min(16 * t + c, p.rows - 1) * p.K + WR * g;
  struct Step { u32x4 w[WR], x[RT]; };
  auto load = [&](Step &b, int s) {
    const int k0 = s * KS;
    if (k0 + KS <= p.K) {
#pragma unroll
      for (int i = 0; i < WR; i++) b.w[i] = *reinterpret_cast<const u32x4 *>(wp + (size_t)(k0 + i) * p.N);
#pragma unroll
      for (int t = 0; t < RT; t++) b.x[t] = *reinterpret_cast<const u32x4 *>(xp[t] + k0);
    } else {  // a lane's channels are in or out together (K % WR == 0); those that are not there are zeros on both sides
      const bool in = k0 + WR * g < p.K;
#pragma unroll
      for (int i = 0; i < WR; i++) b.w[i] = in ? *reinterpret_cast<const u32x4 *>(wp + (size_t)(k0 + i) * p.N) : (u32x4){0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < RT; t++) b.x[t] = in ? *reinterpret_cast<const u32x4 *>(xp[t] + k0) : (u32x4){0, 0, 0, 0};
    }
  };
  f32x4 acc[RT][EPL];
#pragma unroll
  for (int t = 0; t < RT; t++)
#pragma unroll
    for (int j = 0; j < EPL; j++) acc[t][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
  auto products = [&](const Step &b) {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < WR; i++) {
        const f32x4 wf = __builtin_bit_cast(f32x4, b.w[i]);
#pragma unroll
        for (int t = 0; t < RT; t++) {
          const f32x4 xf = __builtin_bit_cast(f32x4, b.x[t]);
#pragma unroll
          for (int j = 0; j < EPL; j++) acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[j], xf[i], acc[t][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < EPL; j++) {
        u32x4 f;
#pragma unroll
        for (int q = 0; q < 4; q++) f[q] = __builtin_amdgcn_perm(b.w[2 * q + 1][j / 2], b.w[2 * q][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int t = 0; t < RT; t++)
          acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, b.x[t]), acc[t][j], 0, 0, 0);
      }
    }
  };
  Step buf[DEPTH];
  int s = s0 + w;
#pragma unroll
  for (int d = 0; d < DEPTH; d++)
    if (s + NW * d < s1) load(buf[d], s + NW * d);
  for (; s < s1; s += NW * DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; d++)
      if (s + NW * d < s1) {
        products(buf[d]);
        if (s + NW * (d + DEPTH) < s1) load(buf[d], s + NW * (d + DEPTH));
      }
  }
  // a lane: row 16 t + c, columns EPL (4 g + r) + j
#pragma unroll
  for (int t = 0; t < RT; t++)
    if (16 * t + c < p.rows) {
#pragma unroll
      for (int r = 0; r < 4; r++)
#pragma unroll
        for (int j = 0; j < EPL; j += 4)
          *reinterpret_cast<f32x4 *>(&red[w][16 * t + c][EPL * (4 * g + r) + j]) = (f32x4){acc[t][j][r], acc[t][j + 1][r], acc[t][j + 2][r], acc[t][j + 3][r]};
    }
  __syncthreads();
  for (int e = tid; e < p.rows * (CG / 4); e += 64 * NW) {
    const int m = e / (CG / 4), col = e % (CG / 4) * 4, n = n0 + col;
    if (n >= p.N) continue;
    f32x4 v = *reinterpret_cast<const f32x4 *>(&red[0][m][col]);
#pragma unroll
    for (int i = 1; i < NW; i++) v += *reinterpret_cast<const f32x4 *>(&red[i][m][col]);
    if (nsplit > 1) *reinterpret_cast<f32x4 *>(p.part + ((size_t)split * p.rows + m) * p.N + n) = v;
    else p.put(m, n, v, p.bias4(n));
  }
}

// the load-to-LDS path's channels: whole steps, where there is one (else all of them, on the register-staged kernel)
static int gemm_steps(int K, int elem_size) {
  const int step = 128 / elem_size;
  return K >= step ? K / step * step : K;
}
// its tile and K split.  256 x 256 is not on offer: with this epilogue its sums do not fit the registers (bf16 4096 x 320 x 2560:
// 39.6 us, 16.2 on the tiled kernel; fp32 8192 x 1024 x 4096: 612 us, 540 with 256 x 128)
static GemmPlan plan_tiles(int rows, int N, int K_steps, int elem_size) {
  return plan_gemm_async(rows, N, K_steps, 1, elem_size, true, false, true, 1, 1);
}

// ---- which kernel --------------------------------------------------------------------------------------------------------
// Estimated times in microseconds, fitted to measurements of every kernel on the same shapes (replayed graphs, so without host
// time).  A kernel's workgroups run in rounds of what the chip holds; a round costs a fixed part (first loads, epilogue) and a part
// per K step of 128 bytes a row, which is smaller where CUs are left over or hold one workgroup instead of two.
// The estimates are off by up to a quarter, so between kernels closer than that the choice may miss the faster one.
// Measured and estimated, us (bf16, rows x K x N):            large        medium       planned tiles
//   16384 x 4096 x 8192                                       795 / 775    984 / 899    1003 / 965
//   4096 x 640 x 2560                                         21.1 / 23.0  20.4 / 22.2  28.9 / 32.7
//   1024 x 1280 x 5120                                        29.0 / 30.0  20.4 / 22.5  23.3 / 24.5
//   4096 x 2560 x 640                                         47.3 / 51.0  23.2 / 23.8  23.7 / 29.6
//   1024 x 5120 x 1280                                        83.9 / 93.0  37.3 / 40.6  24.6 / 29.2 (K split in 3)
// and in 8 bits:                                              large        medium       small
//   16384 x 4096 x 8192                                       484 / 493    616 / 535    1000 / 1002
//   4096 x 640 x 2560                                         17.6 / 17.5  16.3 / 16.2  27.9 / 24.8
//   1024 x 1280 x 5120                                        22.4 / 21.5  15.9 / 15.5  20.1 / 20.4
//   1024 x 5120 x 1280                                        56.5 / 59.0  27.7 / 28.6  21.3 / 20.9 (K split in 2)
//   77 x 8192 x 1280                                          82.4 / 89.0  36.1 / 41.6  20.6 / 21.8, K split in 5: 11.3 / 11.2
// rest: the fixed part of a last, started round (two workgroups on a CU: it starts while the others end); few: per step where at
// most half of the slots are taken; act: per round for each activation (two workgroups on a CU run one's epilogue beside the other's
// products: 16384 x 640 x 2560 in 8 bits 48 and 47 us without activation, 65 and 60 with gelu)
struct RoundCost { int tile, slots; double fixed, rest, full, few, act[4]; };
constexpr RoundCost kLarge[2] = {{256, 256, 7.0, 7.0, 1.4, 1.05, {0.0, 5.3, 3.0, 1.0}},     // bf16
                                 {256, 256, 7.0, 7.0, 1.7, 1.25, {0.0, 5.3, 3.0, 1.0}}};    // 8 bits
constexpr RoundCost kMedium[2] = {{128, 512, 4.5, 2.2, 0.8, 0.5, {0.0, 1.9, 1.2, 0.4}}, {128, 512, 4.5, 2.2, 0.9, 0.6, {0.0, 1.9, 1.2, 0.4}}};
constexpr RoundCost kAlone[2] = {{128, 256, 5.0, 5.0, 0.42, 0.42, {0.0, 1.9, 1.2, 0.4}}, {128, 256, 5.0, 5.0, 0.54, 0.54, {0.0, 1.9, 1.2, 0.4}}};
constexpr RoundCost kSmall = {64, 512, 2.5, 2.5, 0.41, 0.27, {0.0, 0.6, 0.4, 0.2}};         // 8 bits

static double rounds_cost(const RoundCost &c, const toma_linear_desc &d, int steps, int nsplit = 1) {
  const long long wgs = (long long)((d.rows + c.tile - 1) / c.tile) * ((d.N + c.tile - 1) / c.tile) * nsplit;
  const long long rest = wgs % c.slots;
  const double act = nsplit == 1 ? c.act[d.act] : 0.0;
  double t = 2.0 + (double)(wgs / c.slots) * (c.fixed + act + c.full * steps);
  if (rest) t += (wgs > c.slots ? c.rest : c.fixed) + act + (2 * rest > c.slots ? c.full : c.few) * steps;
  return t;
}

// What the planner's estimate, whose steps are about a tenth too long here, leaves out of an unsplit product in bf16, per round: this
// epilogue, and the channels behind the last whole step (strided loads, two bytes each of W).  4096 x 648 x 1280, us: 128 x 128
// tiles of the tiled kernel 15.5, planned tiles of 256 x 128 18.4; 4096 x 64 x 1280: 7.8 and 9.3; 4096 x 72 x 1280: 8.4 and 11.8.
static double epilogue_cost(const GemmPlan &p, const toma_linear_desc &d, int rows, bool tail) {
  const long long wgs = (long long)((rows + p.bm - 1) / p.bm) * ((d.N + p.bn - 1) / p.bn);
  const double area = p.bm * p.bn / 16384.0, part = std::min(area, 1.0);
  return (double)((wgs + 255) / 256) * (4.75 * std::sqrt(part) + (tail ? 3.0 * part : 0.0) + kMedium[0].act[d.act] * area);
}

// 128 x 128 tiles, with four stages where every CU gets at most one
static double medium_cost(int kind, const toma_linear_desc &d, int steps) {
  return rounds_cost(medium_alone(d.rows, d.N) ? kAlone[kind] : kMedium[kind], d, steps);
}

// The fp32 partial sums of a K split are written and read once, by a kernel more.
static double split_cost(int rows, int N, int nsplit) { return 3.0 + (8.0 * nsplit + 4.0) * rows * N / 4.0e6; }

enum Path { PATH_LARGE, PATH_MEDIUM, PATH_SMALL, PATH_FEW };
struct LinPlan { Path path; int bm, bn, nsplit; };

// Few rows: the K split by the estimated time, fitted to splits in 1, 2, 4 and 8 of the shapes above: a wave's steps one after the
// other, or W at 7 TB/s, and the second kernel of a split.
constexpr int few_rows(int type) { return type == TOMA_F32 ? 32 : 16; }
static LinPlan plan_few(const toma_linear_desc &d) {
  const bool f32 = d.x_type == TOMA_F32;
  LinPlan best{PATH_FEW, d.rows <= 16 ? 16 : 32, f32 ? 64 : 128, 1};
  const int steps = f32 ? (d.K + 15) / 16 : (d.K + 31) / 32, groups = (d.N + best.bn - 1) / best.bn;
  const double step = best.bm == 32 ? 1.4 : 0.75, bytes = (f32 ? 4.0 : 2.0) * d.K * d.N;
  double least = 1e30;
  for (int ns = 1; ns <= 16 && (ns == 1 || 8 * ns <= steps); ns++) {
    const int turns = ((steps + ns - 1) / ns + 7) / 8;
    const long long rounds = ((long long)groups * ns + 255) / 256;
    const double t = std::max(step * turns * (double)rounds, bytes / 7.0e6) + (ns > 1 ? 2.6 + 0.2 * ns + 8.0 * ns * d.rows * d.N / 4.0e6 : 0.0);
    if (t < least) { least = t; best.nsplit = ns; }
  }
  return best;
}

static LinPlan plan_linear(const toma_linear_desc &d) {
  if (d.x_type == TOMA_MX8) {
    const int steps = (d.K + 127) / 128, groups = (steps + 3) / 4;
    LinPlan best{PATH_LARGE, 256, 256, 1};
    double least = rounds_cost(kLarge[1], d, steps);
    auto offer = [&](double t, const LinPlan &p) {
      if (t < least) { least = t; best = p; }
    };
    offer(medium_cost(1, d, steps), {PATH_MEDIUM, 128, 128, 1});
    offer(rounds_cost(kSmall, d, steps), {PATH_SMALL, 64, 64, 1});
    for (int ns = 2; ns <= 8 && ns <= groups; ns++)
      offer(rounds_cost(kSmall, d, (groups + ns - 1) / ns * 4, ns) + split_cost(d.rows, d.N, ns), {PATH_SMALL, 64, 64, ns});
    return best;
  }
  if (d.rows <= few_rows(d.x_type)) return plan_few(d);
  const int es = d.x_type == TOMA_F32 ? 4 : 2, rows = d.rows, K = gemm_steps(d.K, es);
  LinPlan best{PATH_SMALL, 64, 64, 1};
  double least;
  if (gemm_async_fits(rows, d.N, K, es)) {
    const GemmPlan p = plan_tiles(rows, d.N, K, es);
    best = {PATH_SMALL, p.bm, p.bn, p.nsplit};
    least = p.cost / 2100.0;
    if (d.x_type == TOMA_BF16 && p.nsplit == 1) least = 0.9 * least + epilogue_cost(p, d, rows, K < d.K);
  } else {  // less than one step: the register-staged kernel
    least = 2.5 + (double)(((long long)((rows + 63) / 64) * ((d.N + 63) / 64) + 511) / 512) * 2.0;
  }
  if (d.x_type == TOMA_BF16) {
    const int steps = (d.K + 63) / 64;
    const double large = rounds_cost(kLarge[0], d, steps), medium = medium_cost(0, d, steps);
    if (std::min(large, medium) < least) best = large < medium ? LinPlan{PATH_LARGE, 256, 256, 1} : LinPlan{PATH_MEDIUM, 128, 128, 1};
  }
  return best;
}

void plan_linear_tile(const toma_linear_desc &d, int32_t *out3) {
  const LinPlan p = plan_linear(d);
  out3[0] = p.bm; out3[1] = p.bn; out3[2] = p.nsplit;
}

const char *linear_kernel_name(const toma_linear_desc &d) {
  const LinPlan p = plan_linear(d);
  if (p.path == PATH_LARGE) return "large";
  if (p.path == PATH_MEDIUM) return medium_alone(d.rows, d.N) ? "medium_four_stages" : "medium";
  if (p.path == PATH_FEW) return "few_rows";
  if (d.x_type == TOMA_MX8) return "small";
  const int es = d.x_type == TOMA_F32 ? 4 : 2;
  return gemm_async_fits(d.rows, d.N, gemm_steps(d.K, es), es) ? "planned" : "short";
}

template <typename T>
static void linear_typed(const LinArgs &a, const LinPlan &plan, float *part, hipStream_t st) {
  EpiPol<T> p{};
  p.In = static_cast<const T *>(a.X); p.Wt = static_cast<const T *>(a.W); p.bias = static_cast<const T *>(a.bias);
  p.R = static_cast<const T *>(a.R); p.R2 = static_cast<const T *>(a.R2); p.Out = static_cast<T *>(a.Y);
  p.part = part;
  p.rows = a.rows; p.K = a.K; p.N = a.N; p.act = a.act; p.K_steps = gemm_steps(a.K, (int)sizeof(T));
  const int M = a.rows, N = a.N;
  if (plan.path == PATH_FEW) {
    KernelTimer kt(K_LINEAR, st);
    p.K_steps = a.K;
    const dim3 grid((unsigned)((N + plan.bn - 1) / plan.bn), (unsigned)plan.nsplit);
    if (plan.bm == 16) hipLaunchKernelGGL((k_linear_few<T, 1>), grid, dim3(512), 0, st, p, plan.nsplit);
    else if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((k_linear_few<T, 2>), grid, dim3(512), 0, st, p, plan.nsplit);
  } else {
    KernelTimer kt(K_LINEAR, st);
    const int tm = (M + plan.bm - 1) / plan.bm, tn = (N + plan.bn - 1) / plan.bn;
    const dim3 grid(tm * tn * plan.nsplit);
    if (!gemm_async_fits(M, N, p.K_steps, (int)sizeof(T)))
      hipLaunchKernelGGL((k_gemm<T, EpiPol<T>, 64, 64>), grid, dim3(256), 0, st, p, tm, tn);
    else if (plan.bm == 256)
      hipLaunchKernelGGL((k_gemm_async<T, EpiPol<T>, 256, 128, 3>), grid, dim3(512), 0, st, p, tm, tn, 1, plan.nsplit);
    else if (plan.bn == 128)
      hipLaunchKernelGGL((k_gemm_async<T, EpiPol<T>, 128, 128, 4>), grid, dim3(512), 0, st, p, tm, tn, 1, plan.nsplit);
    else if (plan.bm == 128)
      hipLaunchKernelGGL((k_gemm_async<T, EpiPol<T>, 128, 64, 4>), grid, dim3(512), 0, st, p, tm, tn, 1, plan.nsplit);
    else
      hipLaunchKernelGGL((k_gemm_async<T, EpiPol<T>, 64, 64, 4>), grid, dim3(512), 0, st, p, tm, tn, 1, plan.nsplit);
  }
  if (plan.nsplit > 1) {
    KernelTimer kt(K_SPLIT, st);
    const size_t quads = (size_t)M * (N / 4);
    hipLaunchKernelGGL((k_split_finish<T, EpiPol<T>>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, p, 1, plan.nsplit);
  }
}

size_t linear_workspace_bytes(const toma_linear_desc &d) {
  const LinPlan p = plan_linear(d);
  return p.nsplit > 1 ? (size_t)p.nsplit * d.rows * d.N * sizeof(float) : 0;
}

int launch_linear(const toma_linear_desc &d, const void *X, const void *Xs, const void *W, const void *Ws, const void *bias,
                  const void *R, const void *R2, void *Y, void *Ys, void *ws, hipStream_t st) {
  const LinArgs a{X, W, static_cast<const uint8_t *>(Xs), static_cast<const uint8_t *>(Ws), bias, R, R2, Y, static_cast<uint8_t *>(Ys),
                  d.rows, d.K, d.N, d.act, mx_scale_stride(d.K), mx_scale_stride(d.N)};
  const LinPlan plan = plan_linear(d);
  float *part = static_cast<float *>(ws);
  const bool mx_out = Ys != nullptr;
  if (plan.path == PATH_LARGE || plan.path == PATH_MEDIUM) {
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
