// Products of the linear layer with few output tiles: bf16, and 8 bits with a power-of-two scale per 32 channels.
//
// With fewer tiles than the chip has places, a call takes as long as one workgroup's walk through K, and that walk as long as
// its instructions and waits: 64 x 64 outputs by four waves, K in units of two steps of 128 bytes a row, one barrier per unit.
// The fragments of a unit are read from LDS while the products of the unit before run, and a unit's loads go out UNITS units
// ahead.  Row layout, fragments and scale codes as in the large tiles' kernel.
#include <type_traits>

#include "toma_linear.h"

namespace toma {

// N loads of 1 KiB each to consecutive KiB of LDS behind lds_addr, from one buffer; off[t] carries 4096 - 1024 t on top (the
// instruction's immediate adds 1024 t to both addresses; the buffer's base lies 4096 below).
template <int N>
__device__ __forceinline__ void buffer_to_lds_run(const uint8_t *base, uint32_t bytes, const uint32_t (&off)[N], uint32_t lds_addr) {
  static_assert(N == 1 || N == 2 || N == 4, "spelled out");
  const u32x4 rsrc = buffer_of(base - 4096, bytes);
  if constexpr (N == 1)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(off[0]), "s"(rsrc) : "memory", "m0");
  else if constexpr (N == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\tbuffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds" ::"s"(lds_addr),
                 "v"(off[0]), "v"(off[1]), "s"(rsrc) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\tbuffer_load_dwordx4 %2, %5, 0 offen offset:1024 lds\n\t"
                 "buffer_load_dwordx4 %3, %5, 0 offen offset:2048 lds\n\tbuffer_load_dwordx4 %4, %5, 0 offen offset:3072 lds" ::"s"(lds_addr),
                 "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(rsrc) : "memory", "m0");
}

// RAGGED: K is no multiple of a step
template <int KIND, int BM, int BN, int WM, int WN, int UNITS, bool MX_OUT, bool RAGGED>
__global__ __launch_bounds__(64 * WM * WN) void k_linear_small(const LinArgs a, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  constexpr int ES = KIND == LIN_MX ? 1 : 2, BK = 128 / ES;
  constexpr int NIA = BM / 8 / NW, NIB = BN / 8 / NW;  // load instructions (1 KiB) per wave and step
  constexpr int NS = (BM + BN) / 16, NIS = KIND == LIN_MX ? (NS + 2 * NW - 1) / (2 * NW) : 0;  // per unit: half of four steps' scale codes
  constexpr int L = 2 * (NIA + NIB) + NIS;             // loads per wave and unit
  constexpr int PPR = BN / 8;                          // packets per k-row of a k-major stage
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_BYTES = KIND == LIN_MX ? (BM + BN) * 16 : 0;
  constexpr int SLOTS = (UNITS + 3) / 2;               // of four steps' codes
  constexpr int B_AT = UNITS * 2 * A_BYTES, S_AT = B_AT + UNITS * 2 * B_BYTES, LDS_BYTES = S_AT + SLOTS * S_BYTES;
  static_assert(TM % 2 == 0 && TM <= 4 && TN <= 4 && (UNITS - 1) * L < 64, "blocks spelled out below; the wait count's range");
  static_assert(NW * kEpilogueFloats<TN> * 4 <= LDS_BYTES, "the epilogue's rows fit the stages");
  __shared__ __align__(1024) uint8_t lds[LDS_BYTES];

  int tile_m, tile_n;
  tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w / WN, wn = w % WN;
  const int g = lane >> 4, c = lane & 15;
  const int K = a.K, nk = (K + BK - 1) / BK, nu = (nk + 1) >> 1;

  // ---- loads ----------------------------------------------------------------------------------------------------------
  const uint8_t *xb = static_cast<const uint8_t *>(a.X) + (size_t)m0 * K * ES;
  const uint8_t *wb = static_cast<const uint8_t *>(a.W) + (KIND == LIN_MX ? (size_t)n0 * K : (size_t)n0 * 2);
  const size_t w_step = KIND == LIN_MX ? 128 : (size_t)BK * a.N * 2;
  // (rows and columns behind the end repeat the last: their results are not stored)
  uint32_t xo[NIA], wo[NIB];
  int xk[NIA], wk[NIB];  // first channel (k-row) of the lane's packet
#pragma unroll
  for (int t = 0; t < NIA; t++) {
    const int row = (w * NIA + t) * 8 + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
    xk[t] = p * (16 / ES);
    xo[t] = (uint32_t)min(row, a.rows - 1 - m0) * (uint32_t)(K * ES) + p * 16 + 4096 - 1024 * t;
  }
#pragma unroll
  for (int t = 0; t < NIB; t++) {
    if constexpr (KIND == LIN_MX) {
      const int row = (w * NIB + t) * 8 + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
      wk[t] = p * 16;
      wo[t] = (uint32_t)min(row, a.N - 1 - n0) * (uint32_t)K + p * 16 + 4096 - 1024 * t;
    } else {
      const int k = (w * NIB + t) * (64 / PPR) + lane / PPR, p = km_place<PPR>(k, lane % PPR);
      wk[t] = k;
      wo[t] = (uint32_t)k * (uint32_t)(a.N * 2) + (uint32_t)min(p * 16, (a.N - n0 - 8) * 2) + 4096 - 1024 * t;
    }
  }
  const uint32_t l0 = lds_addr_of(lds);
  const uint32_t lx = l0 + (uint32_t)(w * NIA * 1024), lw = l0 + B_AT + (uint32_t)(w * NIB * 1024);
  auto issue_codes = [&](int chunk, int part) {  // half of the rows' codes of four steps; behind the end of a row its last repeat
#pragma unroll
    for (int t = 0; t < NIS; t++) {
      const int sr = ((part * NW + w) * NIS + t) % NS * 16;
      const bool of_x = sr < BM;
      const uint8_t *base = of_x ? a.Xs + (size_t)m0 * a.xs_stride : a.Ws + (size_t)n0 * a.xs_stride;
      const int row = min(sr + (lane >> 2) - (of_x ? 0 : BM), of_x ? a.rows - 1 - m0 : a.N - 1 - n0);
      const uint32_t off = (uint32_t)row * (uint32_t)a.xs_stride + (uint32_t)min(16 * chunk + 4 * (lane & 3), a.xs_stride - 4);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(l0 + S_AT + (uint32_t)(__builtin_amdgcn_readfirstlane(chunk % SLOTS) * S_BYTES + sr * 16)),
                   "v"(off), "s"(base)
                   : "memory", "m0");
    }
  };
  auto issue = [&](int slot, int u) {
    if constexpr (KIND == LIN_MX) issue_codes(((u - 1) >> 1) + 1, (u - 1) & 1);  // (a chunk is complete with its first unit's loads)
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int j = 2 * u + h;
      const uint32_t bytes = j < nk ? kAllPackets : 0u;
      uint32_t ox[NIA], ow[NIB];
#pragma unroll
      for (int t = 0; t < NIA; t++) ox[t] = !RAGGED || xk[t] < K - j * BK ? xo[t] : kNoPacket;
#pragma unroll
      for (int t = 0; t < NIB; t++) ow[t] = !RAGGED || wk[t] < K - j * BK ? wo[t] : kNoPacket;
      buffer_to_lds_run<NIA>(xb + (size_t)j * 128, bytes, ox, lx + (uint32_t)((2 * slot + h) * A_BYTES));
      buffer_to_lds_run<NIB>(wb + (size_t)j * w_step, bytes, ow, lw + (uint32_t)((2 * slot + h) * B_BYTES));
    }
  };

  // ---- fragments ------------------------------------------------------------------------------------------------------
  const uint32_t p0 = (uint32_t)(g ^ ((c >> 1) & 7)) << 4;
  const int kq = 8 * g + (c >> 2), kcol = wn * WTN + 4 * (c & 3);  // (k-major weights: transpose reads)
  constexpr int NRW = KIND == LIN_MX ? 2 : TN;
  lds_ptr rx[2], rw[NRW];
#pragma unroll
  for (int e = 0; e < 2; e++) rx[e] = (lds_ptr)(lds + (wm * WTM + c) * 128 + (p0 ^ (64u * e)));
#pragma unroll
  for (int e = 0; e < NRW; e++) {
    if constexpr (KIND == LIN_MX) rw[e] = (lds_ptr)(lds + B_AT + (wn * WTN + c) * 128 + (p0 ^ (64u * e)));
    else rw[e] = (lds_ptr)(lds + B_AT + (kq * PPR + km_place<PPR>(kq, (kcol + 16 * e) >> 3)) * 16 + (kcol & 7) * 2);
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
      for (int j = 0; j < TN; j++) {
        if constexpr (KIND == LIN_MX) {
          fw[set][h][j] = join_halves(*(lds_u32x4_ptr)(rw[0] + aw + h * B_BYTES + j * 2048), *(lds_u32x4_ptr)(rw[1] + aw + h * B_BYTES + j * 2048));
        } else {
          u32x4 f[2];
#pragma unroll
          for (int e = 0; e < 2; e++) {
            const lds_ptr at = rw[j] + aw + h * B_BYTES + 32 * e * PPR * 16;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)at));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + 4 * PPR * 16)));
            f[e] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
          }
          fw[set][h][j] = join_halves(f[0], f[1]);
        }
      }
    }
    if constexpr (KIND == LIN_MX) {  // a row's codes of the unit's two steps: eight bytes
      const lds_ptr at = rs + ((u >> 1) % SLOTS * S_BYTES + (u & 1) * 8);
#pragma unroll
      for (int i = 0; i < TM; i++) raw_x[i] = *(lds_u32x2_ptr)(at + (wm * WTM + 16 * i) * 16);
#pragma unroll
      for (int j = 0; j < TN; j++) raw_w[j] = *(lds_u32x2_ptr)(at + (BM + wn * WTN + 16 * j) * 16);
    }
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
      cx[h] = gather_bytes(dx, TM, mask, g);
      cw[h] = gather_bytes(dw, TN, mask, g);
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
  if constexpr (KIND == LIN_MX) issue_codes(0, 0);
#pragma unroll
  for (int u = 0; u < UNITS; u++) issue(u, u);
  wait_vmcnt<(UNITS - 1) * L>();
  meet();
  read(even, 0, 0);
  if constexpr (KIND == LIN_MX) gather_codes(0);
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
    auto row = [&](auto h_, auto i_, int e) {
      constexpr int h = decltype(h_)::value, i = decltype(i_)::value;
      auto one = [&](auto j_) {
        constexpr int j = decltype(j_)::value;
        if constexpr (i < TM && j < TN) {
          if constexpr (KIND == LIN_MX)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[set][h][j], fx[set][h][i], acc[i][j], 0, 0, j, (int)cw[h], i, (int)cx[h]);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_half(fw[set][h][j], e), bf16_half(fx[set][h][i], e), acc[i][j], 0, 0, 0);
        }
      };
      one(integral_constant<int, 0>()); one(integral_constant<int, 1>()); one(integral_constant<int, 2>()); one(integral_constant<int, 3>());
    };
    auto half = [&](auto h_) {
#pragma unroll
      for (int e = 0; e < (KIND == LIN_MX ? 1 : 2); e++) {
        row(h_, integral_constant<int, 0>(), e); row(h_, integral_constant<int, 1>(), e);
        row(h_, integral_constant<int, 2>(), e); row(h_, integral_constant<int, 3>(), e);
      }
    };
    half(even);
    half(odd);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (KIND == LIN_MX) gather_codes(u + 1);
    __builtin_amdgcn_s_waitcnt(0xc07f);
    wait_vmcnt<(UNITS - 2) * L>();
    meet();
    slot = next;
  };
  for (int u = 0;;) {
    unit(even, u);
    if (++u >= nu) break;
    unit(odd, u);
    if (++u >= nu) break;
  }
  wait_vmcnt<0>();  // (the zeros of the units behind the last)
  meet();
  linear_epilogue<TM, TN, MX_OUT>(a, acc, reinterpret_cast<float *>(lds) + w * kEpilogueFloats<TN>, m0 + wm * WTM, n0 + wn * WTN, lane);
}

template <int KIND, int BM, int BN, int WM, int WN, int UNITS>
static void go(const LinArgs &a, bool mx_out, hipStream_t st) {
  const int tm = (a.rows + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  const dim3 grid((unsigned)(tm * (long long)tn)), block(64 * WM * WN);
  const bool ragged = a.K % (KIND == LIN_MX ? 128 : 64) != 0;
  auto run = [&](auto out) {
    constexpr bool o = decltype(out)::value;
    if (ragged) hipLaunchKernelGGL((k_linear_small<KIND, BM, BN, WM, WN, UNITS, o, true>), grid, block, 0, st, a, tm, tn);
    else hipLaunchKernelGGL((k_linear_small<KIND, BM, BN, WM, WN, UNITS, o, false>), grid, block, 0, st, a, tm, tn);
  };
  if constexpr (KIND == LIN_MX) {
    if (mx_out) return run(std::true_type());
  }
  run(std::false_type());
}

int launch_linear_small(int kind, int which, int, const LinArgs &a, bool mx_out, hipStream_t st) {
#define TILES(KIND) \
  if (which == 2) go<KIND, 64, 64, 2, 2, 2>(a, mx_out, st); \
  else if (which == 3) go<KIND, 64, 64, 2, 2, 4>(a, mx_out, st); \
  else if (which == 4) go<KIND, 64, 128, 2, 2, 2>(a, mx_out, st); \
  else if (which == 5) go<KIND, 64, 128, 2, 2, 3>(a, mx_out, st); \
  else go<KIND, 128, 128, 2, 2, 2>(a, mx_out, st);
  if (kind == LIN_MX) { TILES(LIN_MX) } else { TILES(LIN_BF16) }
  return launch_status();
}

}  // namespace toma
