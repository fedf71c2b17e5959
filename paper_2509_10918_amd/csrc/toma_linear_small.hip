// 8-bit products of the linear layer with few output tiles.
//
// With fewer tiles than the chip has places, a call takes as long as one workgroup's walk through K, and that walk as long as
// its instructions and waits: 64 x 64 outputs by four waves, K in units of two steps of 128 bytes a row, one barrier per unit.
// The fragments of a unit are read from LDS while the products of the unit before run, and a unit's loads go out UNITS units
// ahead.  Row layout, fragments and scale codes as in the large tiles' kernel.
// K may be split between workgroups; the fp32 partial sums are then added up by a second kernel.
#include <type_traits>

#include "toma_linear.h"

namespace toma {

// Two loads of 1 KiB each to consecutive KiB of LDS behind lds_addr, from one buffer; off[t] carries 4096 - 1024 t on top (the
// instruction's immediate adds 1024 t to both addresses; the buffer's base lies 4096 below).
__device__ __forceinline__ void buffer_to_lds_pair(const uint8_t *base, uint32_t bytes, const uint32_t (&off)[2], uint32_t lds_addr) {
  const u32x4 rsrc = buffer_of(base - 4096, bytes);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\tbuffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds" ::"s"(lds_addr),
               "v"(off[0]), "v"(off[1]), "s"(rsrc) : "memory", "m0");
}

constexpr int kSmall = 64, kSmallWaves = 4;  // rows and columns of a tile; two by two waves

// RAGGED: K is no multiple of a step
template <bool MX_OUT, bool RAGGED>
__global__ __launch_bounds__(64 * kSmallWaves) void k_linear_small(const LinArgs a, int tiles_m, int tiles_n, int nsplit, float *part) {
  constexpr int BM = kSmall, BN = kSmall, NW = kSmallWaves, WN = 2, WTM = BM / 2, WTN = BN / 2, TM = 2, TN = 2;
  constexpr int BK = 128, UNITS = 2;
  constexpr int NIA = BM / 8 / NW, NIB = BN / 8 / NW;  // load instructions (1 KiB) per wave and step
  constexpr int L = 2 * (NIA + NIB) + 1;               // loads per wave and unit: with half of four steps' scale codes
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_BYTES = (BM + BN) * 16;
  constexpr int SLOTS = 2;                             // of four steps' codes
  constexpr int B_AT = UNITS * 2 * A_BYTES, S_AT = B_AT + UNITS * 2 * B_BYTES, LDS_BYTES = S_AT + SLOTS * S_BYTES;
  static_assert(NIA == 2 && NIB == 2 && (BM + BN) / 16 == 2 * NW, "loads in pairs; one load of scale codes per wave and unit");
  static_assert(NW * kEpilogueFloats<TN> * 4 <= LDS_BYTES, "the epilogue's rows fit the stages");
  __shared__ __align__(1024) uint8_t lds[LDS_BYTES];

  int tile_m, tile_n;
  tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tile_m, tile_n);
  const int split = blockIdx.y;
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w / WN, wn = w % WN;
  const int g = lane >> 4, c = lane & 15;
  const int K = a.K, nk_all = (K + BK - 1) / BK;
  // this workgroup's share of the steps: whole groups of four, whose codes come together
  const int groups = (nk_all + 3) >> 2;
  const int u0 = (int)((long long)groups * split / nsplit) * 2, nk = min((int)((long long)groups * (split + 1) / nsplit) * 4, nk_all), nu = (nk + 1) >> 1;

  // ---- loads ----------------------------------------------------------------------------------------------------------
  const uint8_t *xb = static_cast<const uint8_t *>(a.X) + (size_t)m0 * K;
  const uint8_t *wb = static_cast<const uint8_t *>(a.W) + (size_t)n0 * K;
  // (rows and columns behind the end repeat the last: their results are not stored)
  uint32_t xo[NIA], wo[NIB];
  int xk[NIA], wk[NIB];  // first channel of the lane's packet
#pragma unroll
  for (int t = 0; t < NIA; t++) {
    const int row = (w * NIA + t) * 8 + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
    xk[t] = p * 16;
    xo[t] = (uint32_t)min(row, a.rows - 1 - m0) * (uint32_t)K + p * 16 + 4096 - 1024 * t;
  }
#pragma unroll
  for (int t = 0; t < NIB; t++) {
    const int row = (w * NIB + t) * 8 + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
    wk[t] = p * 16;
    wo[t] = (uint32_t)min(row, a.N - 1 - n0) * (uint32_t)K + p * 16 + 4096 - 1024 * t;
  }
  const uint32_t l0 = lds_addr_of(lds);
  const uint32_t lx = l0 + (uint32_t)(w * NIA * 1024), lw = l0 + B_AT + (uint32_t)(w * NIB * 1024);
  auto issue_codes = [&](int chunk, int part) {  // half of the rows' codes of four steps; behind the end of a row its last repeat
    const int sr = (part * NW + w) * 16;
    const bool of_x = sr < BM;
    const uint8_t *base = of_x ? a.Xs + (size_t)m0 * a.xs_stride : a.Ws + (size_t)n0 * a.xs_stride;
    const int row = min(sr + (lane >> 2) - (of_x ? 0 : BM), of_x ? a.rows - 1 - m0 : a.N - 1 - n0);
    const uint32_t off = (uint32_t)row * (uint32_t)a.xs_stride + (uint32_t)min(16 * chunk + 4 * (lane & 3), a.xs_stride - 4);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(l0 + S_AT + (uint32_t)(__builtin_amdgcn_readfirstlane(chunk % SLOTS) * S_BYTES + sr * 16)),
                 "v"(off), "s"(base)
                 : "memory", "m0");
  };
  auto issue = [&](int slot, int u) {
    issue_codes(((u - 1) >> 1) + 1, (u - 1) & 1);  // (a chunk is complete with its first unit's loads)
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int j = 2 * u + h;
      const uint32_t bytes = j < nk ? kAllPackets : 0u;
      uint32_t ox[NIA], ow[NIB];
#pragma unroll
      for (int t = 0; t < NIA; t++) ox[t] = !RAGGED || xk[t] < K - j * BK ? xo[t] : kNoPacket;
#pragma unroll
      for (int t = 0; t < NIB; t++) ow[t] = !RAGGED || wk[t] < K - j * BK ? wo[t] : kNoPacket;
      buffer_to_lds_pair(xb + (size_t)j * 128, bytes, ox, lx + (uint32_t)((2 * slot + h) * A_BYTES));
      buffer_to_lds_pair(wb + (size_t)j * 128, bytes, ow, lw + (uint32_t)((2 * slot + h) * B_BYTES));
    }
  };

  // ---- fragments ------------------------------------------------------------------------------------------------------
  const uint32_t p0 = (uint32_t)(g ^ ((c >> 1) & 7)) << 4;
  lds_ptr rx[2], rw[2];
#pragma unroll
  for (int e = 0; e < 2; e++) {
    rx[e] = (lds_ptr)(lds + (wm * WTM + c) * 128 + (p0 ^ (64u * e)));
    rw[e] = (lds_ptr)(lds + B_AT + (wn * WTN + c) * 128 + (p0 ^ (64u * e)));
  }
  const lds_ptr rs = (lds_ptr)(lds + S_AT + c * 16);
  i32x8 fx[2][2][TM], fw[2][2][TN];  // [set][half of the unit]
  u32x2 raw_x[TM], raw_w[TN];
  uint32_t cx[2], cw[2];             // codes of the two halves
  auto read = [&](auto set_, int slot, int u) {
    constexpr int set = decltype(set_)::value;
    const int ax = slot * (2 * A_BYTES), aw = slot * (2 * B_BYTES);
#pragma unroll
    for (int h = 0; h < 2; h++) {
#pragma unroll
      for (int i = 0; i < TM; i++)
        fx[set][h][i] = join_halves(*(lds_u32x4_ptr)(rx[0] + ax + h * A_BYTES + i * 2048), *(lds_u32x4_ptr)(rx[1] + ax + h * A_BYTES + i * 2048));
#pragma unroll
      for (int j = 0; j < TN; j++)
        fw[set][h][j] = join_halves(*(lds_u32x4_ptr)(rw[0] + aw + h * B_BYTES + j * 2048), *(lds_u32x4_ptr)(rw[1] + aw + h * B_BYTES + j * 2048));
    }
    // a row's codes of the unit's two steps: eight bytes
    const lds_ptr at = rs + ((u >> 1) % SLOTS * S_BYTES + (u & 1) * 8);
#pragma unroll
    for (int i = 0; i < TM; i++) raw_x[i] = *(lds_u32x2_ptr)(at + (wm * WTM + 16 * i) * 16);
#pragma unroll
    for (int j = 0; j < TN; j++) raw_w[j] = *(lds_u32x2_ptr)(at + (BM + wn * WTN + 16 * j) * 16);
  };
  const uint32_t tail_mask = K % 128 ? 0xffffffffu >> (32 - (K >> 5) % 4 * 8) : 0u;  // codes of the last group that stand for channels
  auto gather_codes = [&](int u) {
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int j = 2 * u + h;
      const uint32_t mask = j < (K >> 7) ? 0xffffffffu : j == (K >> 7) ? tail_mask : 0u;
      uint32_t dx[TM], dw[TN];
#pragma unroll
      for (int i = 0; i < TM; i++) dx[i] = raw_x[i][h];
#pragma unroll
      for (int i = 0; i < TN; i++) dw[i] = raw_w[i][h];
      cx[h] = gather_bytes(dx, mask, g);
      cw[h] = gather_bytes(dw, mask, g);
    }
  };

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  // ---- K loop -----------------------------------------------------------------------------------------------------------
  using std::integral_constant;
  constexpr integral_constant<int, 0> even{};
  constexpr integral_constant<int, 1> odd{};
  issue_codes(u0 >> 1, 0);
#pragma unroll
  for (int u = 0; u < UNITS; u++) issue(u, u0 + u);
  wait_vmcnt<(UNITS - 1) * L>();
  meet();
  read(even, 0, u0);
  gather_codes(u0);
  __builtin_amdgcn_s_waitcnt(0xc07f);
  wait_vmcnt<(UNITS - 2) * L>();
  meet();
  int slot = 0;
  // behind the barrier in front of unit u every wave has read its fragments of u (so u's slot is free), and u + 1 has landed
  auto unit = [&](auto set_, int u) {
    constexpr int set = decltype(set_)::value;
    const int next = slot + 1 == UNITS ? 0 : slot + 1;
    read(integral_constant<int, set ^ 1>(), next, u + 1);
    issue(slot, u + UNITS);
    __builtin_amdgcn_sched_barrier(0);
    auto one = [&](auto h_, auto i_, auto j_) {
      constexpr int h = decltype(h_)::value, i = decltype(i_)::value, j = decltype(j_)::value;
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[set][h][j], fx[set][h][i], acc[i][j], 0, 0, j, (int)cw[h], i, (int)cx[h]);
    };
    auto half = [&](auto h_) { one(h_, even, even); one(h_, even, odd); one(h_, odd, even); one(h_, odd, odd); };
    half(even);
    half(odd);
    __builtin_amdgcn_sched_barrier(0);
    gather_codes(u + 1);
    __builtin_amdgcn_s_waitcnt(0xc07f);
    wait_vmcnt<(UNITS - 2) * L>();
    meet();
    slot = next;
  };
  for (int u = u0;;) {
    unit(even, u);
    if (++u >= nu) break;
    unit(odd, u);
    if (++u >= nu) break;
  }
  wait_vmcnt<0>();  // (the zeros of the units behind the last)
  meet();
  if (part) {  // fp32 partial sums [split][rows][N]; k_linear_finish adds them up
#pragma unroll
    for (int i = 0; i < TM; i++) {
      const int m = m0 + wm * WTM + 16 * i + c;
#pragma unroll
      for (int j = 0; j < TN; j++) {
        const int n = n0 + wn * WTN + 16 * j + 4 * g;
        if (m < a.rows && n < a.N) *reinterpret_cast<f32x4 *>(part + ((size_t)split * a.rows + m) * a.N + n) = acc[i][j];
      }
    }
    return;
  }
  linear_epilogue<TM, TN, MX_OUT>(a, acc, reinterpret_cast<float *>(lds) + w * kEpilogueFloats<TN>, m0 + wm * WTM, n0 + wn * WTN, lane);
}

// Sum of the partial products in the order of K, then the epilogue.  One thread per eight columns; a row's threads cover whole
// groups of 128 columns, so that a quad is one packed block and the padding's codes have their writer.
template <bool MX_OUT>
__global__ __launch_bounds__(256) void k_linear_finish(const LinArgs a, int nsplit, const float *__restrict__ part, int per_row) {
  const size_t t = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(t / per_row), n = (int)(t - (size_t)m * per_row) * 8;
  const bool in = m < a.rows && n < a.N;
  const size_t at = (size_t)m * a.N + n;
  F8 v;
#pragma unroll
  for (int i = 0; i < 8; i++) v.v[i] = 0.0f;
  if (in) {
    for (int s = 0; s < nsplit; s++) {
      const F8 p = load8(part + (size_t)s * a.rows * a.N + at);
#pragma unroll
      for (int i = 0; i < 8; i++) v.v[i] += p.v[i];
    }
    if (a.bias) add8(v, pkt_load(static_cast<const bf16_t *>(a.bias) + n));
    activate<false>(v.v, a.act);
    if (a.R) add8(v, pkt_load(static_cast<const bf16_t *>(a.R) + at));
    if (a.R2) add8(v, pkt_load(static_cast<const bf16_t *>(a.R2) + at));
  }
  if constexpr (MX_OUT) {
    u32x2 o;
    const uint32_t code = mx_pack_quad(v, o);
    if (in) *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.Y) + at) = o;
    if (m < a.rows && (n & 31) == 0 && (n >> 5) < a.ys_stride) a.Ys[(size_t)m * a.ys_stride + (n >> 5)] = in ? (uint8_t)code : 0;
  } else if (in) {
    store8(static_cast<bf16_t *>(a.Y) + at, v);
  }
}

void launch_linear_small(const LinArgs &a, bool mx_out, int nsplit, float *part, hipStream_t st) {
  const int tm = (a.rows + kSmall - 1) / kSmall, tn = (a.N + kSmall - 1) / kSmall;
  const dim3 grid((unsigned)(tm * (long long)tn), (unsigned)nsplit), block(64 * kSmallWaves);
  auto run = [&](auto out, auto ragged) {
    hipLaunchKernelGGL((k_linear_small<decltype(out)::value, decltype(ragged)::value>), grid, block, 0, st, a, tm, tn, nsplit,
                       nsplit > 1 ? part : nullptr);
  };
  const bool ragged = a.K % 128 != 0;
  if (mx_out && nsplit == 1) ragged ? run(std::true_type(), std::true_type()) : run(std::true_type(), std::false_type());
  else ragged ? run(std::false_type(), std::true_type()) : run(std::false_type(), std::false_type());
  if (nsplit > 1) {
    const int per_row = mx_out ? a.ys_stride * 4 : a.N / 8;
    const dim3 blocks((unsigned)(((size_t)a.rows * per_row + 255) / 256));
    if (mx_out) hipLaunchKernelGGL(k_linear_finish<true>, blocks, dim3(256), 0, st, a, nsplit, part, per_row);
    else hipLaunchKernelGGL(k_linear_finish<false>, blocks, dim3(256), 0, st, a, nsplit, part, per_row);
  }
}

}  // namespace toma
