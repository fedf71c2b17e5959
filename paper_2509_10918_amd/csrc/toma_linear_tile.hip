// Tiled product of the linear layer for many rows: bf16, and 8 bits with a power-of-two scale per 32 channels.
//
// A workgroup computes BM x BN outputs, a wave WTM x WTN of them with the 16 x 16 matrix instructions (the 32 x 32 ones reach 1.79
// instead of 2.10 PFLOP/s in bf16 on random data, 4.1 instead of 4.5 in 8 bits), the weights as first operand, so that a lane holds
// one row and four consecutive columns of each.  K advances by 128 bytes of a row of X per step (128 channels in 8 bits, 64 in
// bf16: whole cache lines), through stages in LDS that the load-to-LDS path fills.  256 x 256 outputs and 128 x 128 take two stages,
// one and two workgroups on a CU.  128 x 128 with at most one workgroup for every CU take four: nobody else runs while a load is on
// its way (two and four stages, us: bf16 4096 x 2560 x 640 26.8 and 22.7, 2048 x 2048 x 2048 23.2 and 21.1; 1024 x 1280 x 5120, 320
// workgroups, 23.7 and 28.9.  Four waves instead of eight: 29.6 and 28.8, 25.3 and 24.4, 24.7 and 35.2).
// A 128-byte row of a stage is eight 16-byte packets; packet p of row r lies at place p ^ (r >> 1 & 7), which spreads the 16 rows
// that a fragment read takes over all banks.
#include "toma_linear.h"

namespace toma {

template <int KIND, int BM, int BN, int WM, int WN, int STAGES, bool MX_OUT>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_linear_tile(const LinArgs a, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  constexpr int ES = KIND == LIN_MX ? 1 : 2, BK = 128 / ES;
  constexpr int NIA = BM / 16 / NW, NIB = BN / 8 / NW;  // load instructions (1 KiB) per wave and step: half of X's rows, W
  constexpr int NS = (BM + BN) / 16, NIS = KIND == LIN_MX ? (NS + 4 * NW - 1) / (4 * NW) : 0;  // and a quarter of four steps' scale codes
  constexpr int PPR = BN / 8;                          // packets per k-row of a k-major stage
  static_assert(NIA >= 1 && NIB >= 1, "every wave loads its share");
  static_assert(TM % 4 == 0 && NIB % 2 == 0 && TN % (TM / 4) == 0, "row blocks in pairs and halves");
  static_assert(TN <= 4 && TM <= 8, "column and row blocks spelled out below");
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_BYTES = KIND == LIN_MX ? (BM + BN) * 16 : 0;
  constexpr int AHEAD = STAGES - 2;  // steps that loads run ahead of what two stages allow
  constexpr int SLOTS = AHEAD ? 4 : 2;  // of four steps' codes
  constexpr int B_AT = STAGES * A_BYTES, S_AT = B_AT + STAGES * B_BYTES, LDS_BYTES = S_AT + SLOTS * S_BYTES;
  __shared__ __align__(1024) uint8_t lds[LDS_BYTES];

  int tile_m, tile_n;
  tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w / WN, wn = w % WN;
  const int g = lane >> 4, c = lane & 15;
  const int K = a.K, nk = (K + BK - 1) / BK;

  // ---- loads: wave-uniform bases that advance with K, fixed byte offsets per lane -----------------------------------
  const uint8_t *xb = static_cast<const uint8_t *>(a.X) + (size_t)m0 * K * ES;
  const uint8_t *wb = static_cast<const uint8_t *>(a.W) + (KIND == LIN_MX ? (size_t)n0 * K : (size_t)n0 * 2);
  const size_t w_step = KIND == LIN_MX ? 128 : (size_t)BK * a.N * 2;
  // first row of the wave's t-th group of eight rows of X in the lower (upper) half of the row blocks of each wave row
  auto x_row = [&](int t, bool upper) {
    const int q = w * NIA + t;
    return q / (WTM / 16) * WTM + q % (WTM / 16) * 8 + (upper ? WTM / 2 : 0);
  };
  // (rows and columns behind the end repeat the last: their results are not stored)
  uint32_t xo[2][NIA], wo[NIB];
#pragma unroll
  for (int h = 0; h < 2; h++)
#pragma unroll
    for (int t = 0; t < NIA; t++) {
      const int row = x_row(t, h) + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
      xo[h][t] = (uint32_t)min(row, a.rows - 1 - m0) * (uint32_t)(K * ES) + p * 16;
    }
#pragma unroll
  for (int t = 0; t < NIB; t++) {
    if constexpr (KIND == LIN_MX) {
      const int row = (w * NIB + t) * 8 + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
      wo[t] = (uint32_t)min(row, a.N - 1 - n0) * (uint32_t)K + p * 16;
    } else {
      constexpr int RPI = 64 / PPR;  // k-rows per load instruction
      const int k = (w * NIB + t) * RPI + lane / PPR, p = km_place<PPR>(k, lane % PPR);
      wo[t] = (uint32_t)k * (uint32_t)(a.N * 2) + (uint32_t)min(p * 16, (a.N - n0 - 8) * 2);
    }
  }
  // Scale codes come four steps (16 bytes a row) at a time, a quarter of the rows with every step: taken step by step, every load
  // would fetch a cache line for four bytes, as many lines as all elements together.  A load instruction brings 16 rows, a
  // lane's four bytes are those of one step.  Codes behind the end of a row repeat its last.
  const uint32_t l0 = lds_addr_of(lds);
  auto issue_codes = [&](int chunk, int part) {
#pragma unroll
    for (int t = 0; t < NIS; t++) {
      const int sr = ((part * NW + w) * NIS + t) % NS * 16;
      const bool of_x = sr < BM;
      const uint8_t *base = of_x ? a.Xs + (size_t)m0 * a.xs_stride : a.Ws + (size_t)n0 * a.xs_stride;
      const int row = min(sr + (lane >> 2) - (of_x ? 0 : BM), of_x ? a.rows - 1 - m0 : a.N - 1 - n0);
      const uint32_t off = (uint32_t)row * (uint32_t)a.xs_stride + (uint32_t)min(16 * chunk + 4 * (lane & 3), a.xs_stride - 4);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(l0 + S_AT + (uint32_t)(chunk % SLOTS * S_BYTES + sr * 16)),
                   "v"(off), "s"(base)
                   : "memory", "m0");
    }
  };

  // Loads of a step into its stage: the lower and the upper half of X's row blocks, and W with the scale codes.  Packets behind the
  // end of K, and all of a step behind the last, are zeros that nothing is read for.
  auto issue_x = [&](uint32_t st, int j, auto upper_) {
    constexpr int h = decltype(upper_)::value;
    const uint32_t bytes = j < nk ? kAllPackets : 0u;
    const int left = K - j * BK;
#pragma unroll
    for (int t = 0; t < NIA; t++) {
      const int k = ((lane & 7) ^ (((x_row(t, h) + (lane >> 3)) >> 1) & 7)) * (16 / ES);
      buffer_to_lds16(xb + (size_t)j * 128, bytes, k < left ? xo[h][t] : kNoPacket, l0 + st * A_BYTES + (uint32_t)(x_row(t, h) * 128));
    }
  };
  auto issue_w = [&](uint32_t st, int j, auto half_) {
    constexpr int h = decltype(half_)::value;
    const uint32_t bytes = j < nk ? kAllPackets : 0u;
    const int left = K - j * BK;
#pragma unroll
    for (int t = h * NIB / 2; t < (h + 1) * NIB / 2; t++) {
      const int k = KIND == LIN_MX ? ((lane & 7) ^ ((((w * NIB + t) * 8 + (lane >> 3)) >> 1) & 7)) * 16 : (w * NIB + t) * (64 / PPR) + lane / PPR;
      buffer_to_lds16(wb + (size_t)j * w_step, bytes, k < left ? wo[t] : kNoPacket, l0 + B_AT + st * B_BYTES + (uint32_t)((w * NIB + t) * 1024));
    }
  };
  // ---- fragments: a lane takes packets g and 4 + g of its row (bf16: one of each half of the step) ------------------------
  // LDS addresses of the stage that is read; they move to the other stage at the end of a step
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
  auto read_x = [&](int i) { return join_halves(*(lds_u32x4_ptr)(rx[0] + i * 2048), *(lds_u32x4_ptr)(rx[1] + i * 2048)); };
  auto read_w = [&](int j) {
    if constexpr (KIND == LIN_MX) {
      return join_halves(*(lds_u32x4_ptr)(rw[0] + j * 2048), *(lds_u32x4_ptr)(rw[1] + j * 2048));
    } else {
      u32x4 f[2];
#pragma unroll
      for (int e = 0; e < 2; e++) {
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(rw[j] + 32 * e * PPR * 16)));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(rw[j] + (32 * e + 4) * PPR * 16)));
        f[e] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
      }
      return join_halves(f[0], f[1]);
    }
  };
  // scale codes of a step: byte b of word q is the code of row block 4 q + b for this lane's block of 32 channels (g); read as a
  // word per row (its four blocks) by lane group b, then turned over between the lane groups (8192^3 425 us; every lane reading
  // the words of all its row blocks, four times as many LDS reads, 447)
  constexpr int QX = (TM + 3) / 4, QW = (TN + 3) / 4;
  uint32_t cx[QX], cw[QW], raw_x[QX], raw_w[QW];
  const int block_x = 16 * (g % TM), block_w = 16 * (g % TN);
  auto read_codes = [&](int j) {  // of step j
    const lds_ptr at = (lds_ptr)(lds + S_AT) + ((j >> 2) % SLOTS * S_BYTES + (j & 3) * 4) + c * 16;
#pragma unroll
    for (int q = 0; q < QX; q++) raw_x[q] = *(lds_u32_ptr)(at + (wm * WTM + 64 * q + block_x) * 16);
#pragma unroll
    for (int q = 0; q < QW; q++) raw_w[q] = *(lds_u32_ptr)(at + (BM + wn * WTN + 64 * q + block_w) * 16);
  };
  const uint32_t tail_mask = K % 128 ? 0xffffffffu >> (32 - (K >> 5) % 4 * 8) : 0u;  // codes of the last group that stand for channels
  const uint32_t turn_pairs = turn_selector(g & 2), turn_own = turn_selector((g & 1) * 2);
  auto gather_codes = [&](int j) {  // of step j
    const uint32_t mask = j < (K >> 7) ? 0xffffffffu : j == (K >> 7) ? tail_mask : 0u;
#pragma unroll
    for (int q = 0; q < QX; q++) cx[q] = turn_bytes(raw_x[q] & mask, turn_pairs, turn_own);
#pragma unroll
    for (int q = 0; q < QW; q++) cw[q] = turn_bytes(raw_w[q] & mask, turn_pairs, turn_own);
  };

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  // ---- K loop -----------------------------------------------------------------------------------------------------------
  using std::integral_constant;
  constexpr bool TURNS = BM == 256;
  auto product = [&](auto i_, auto j_, const i32x8 &x, const i32x8 &v, int e) {
    constexpr int i = decltype(i_)::value, j = decltype(j_)::value;
    if constexpr (KIND == LIN_MX) {
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v, x, acc[i][j], 0, 0, j % 4, (int)cw[j / 4], i % 4, (int)cx[i / 4]);
    } else {
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_half(v, e), bf16_half(x, e), acc[i][j], 0, 0, 0);
    }
  };
  constexpr integral_constant<int, 0> lower{};
  constexpr integral_constant<int, 1> upper{};
  auto next_codes = [&](int j) {  // with the loads of step j: the codes of a chunk are complete with those of its first step
    if constexpr (KIND == LIN_MX) issue_codes(((j - 1) >> 2) + 1, (j - 1) & 3);
  };
  // A step goes through TP pairs of row blocks of X, each in two phases: memory (the pair's fragments from LDS, in the second half
  // of the pairs those of W and the codes for the next step, and loads) and products.  With eight waves the two waves of a SIMD take
  // turns: a barrier stands behind every phase, and waves 4 .. 7 run one phase behind, so that one wave of a SIMD feeds the
  // matrix core while the other one waits for memory.  (Both in the same phase at the same time, the matrix cores were busy 53 % of
  // the time: 8192^3 in 8 bits 506 us, with turns 442 then.)  The 128 x 128 tiles do without: two workgroups on a CU take turns by
  // themselves, and a lone one gains nothing (bf16 4096 x 2560 x 640 with turns 24.0 us, without 22.7).  A lone one takes 0.42 us a
  // step where its products take 0.21; four waves with fewer fragment reads, fragments read a step ahead between the products, one
  // barrier a step (23.3 us) left that as it is.
  // What a phase may read or overwrite, with two stages (s: step; four only load two steps further ahead): X's lower pairs are read
  // in the first half of the pairs, so in the second half their place takes the loads of step s + 2; the upper pairs, and W of step
  // s + 1, in the second half: in the step behind, their places take the loads of the upper pairs of step s + 2 and W of step s + 3.
  // The loads are spread over the phases (28 at once kept the address unit busy for longer than a phase).  A wave waits for its
  // loads of a half before the barrier in front of that half; every load has a step or more to land.
  constexpr int TP = TM / 2, HP = TP / 2;
  i32x8 fx[2], fw[2][TN];
  if constexpr (KIND == LIN_MX) {
    issue_codes(0, 0);
    issue_codes(0, 1);
    issue_codes(0, 2);
  }
#pragma unroll
  for (int j = 0; j < STAGES; j++) {
    next_codes(j);
    issue_w(j, j, lower);
    issue_w(j, j, upper);
    issue_x(j, j, lower);
    if (j < STAGES - 1) issue_x(j, j, upper);
  }
  constexpr int PER_STEP = 2 * NIA + NIB + NIS, EARLY = AHEAD * PER_STEP;  // loads
  wait_vmcnt<EARLY + PER_STEP>();  // W and the lower half of step 0
  meet();
#pragma unroll
  for (int j = 0; j < TN; j++) fw[0][j] = read_w(j);
  if constexpr (KIND == LIN_MX) {
    read_codes(0);
    gather_codes(0);
  }
#pragma unroll
  for (int e = 0; e < NRW; e++) rw[e] += B_BYTES;
  __builtin_amdgcn_s_waitcnt(0xc07f);
  meet();  // every wave has W of step 0
  if (TURNS && w >= 4) meet();
  auto step = [&](auto st_, int kt) {
    constexpr int st = decltype(st_)::value;
    auto pair = [&](auto p_) {
      constexpr int p = decltype(p_)::value;
      if constexpr (p < TP) {
        fx[0] = read_x(2 * p);
        fx[1] = read_x(2 * p + 1);
        if constexpr (p >= HP) {
#pragma unroll
          for (int j = 0; j < TN; j++)
            if (j / (TN / HP) == p - HP) fw[(st + 1) & 1][j] = read_w(j);
          if constexpr (KIND == LIN_MX && p == TP - 1) read_codes(kt + 1);
        }
        if constexpr (p == 0) {
          issue_x((st + STAGES - 1) % STAGES, kt + 1 + AHEAD, upper);
          next_codes(kt + 2 + AHEAD);
        }
        if constexpr (p == HP - 1) issue_w(st, kt + 2 + AHEAD, lower);
        if constexpr (p == HP) issue_w(st, kt + 2 + AHEAD, upper);
        if constexpr (p == TP - 1) issue_x(st, kt + 2 + AHEAD, lower);
        if constexpr (p == TP - 1) {  // the addresses move to the other stage
          constexpr int da = st == STAGES - 1 ? -(STAGES - 1) * A_BYTES : A_BYTES;
          constexpr int db = st == STAGES - 2 ? -(STAGES - 1) * B_BYTES : B_BYTES;  // (W is read a step ahead)
          rx[0] += da;
          rx[1] += da;
#pragma unroll
          for (int e = 0; e < NRW; e++) rw[e] += db;
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (TURNS || p == HP - 1 || p == TP - 1) {
          __builtin_amdgcn_s_waitcnt(0xc07f);
          if constexpr (p == HP - 1) wait_vmcnt<EARLY + PER_STEP - NIB / 2>();
          if constexpr (p == TP - 1) wait_vmcnt<EARLY + PER_STEP>();
          meet();
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        auto column = [&](auto j_) {
          constexpr int j = decltype(j_)::value;
          if constexpr (j < TN) {
#pragma unroll
            for (int e = 0; e < (KIND == LIN_MX ? 1 : 2); e++) {
              product(integral_constant<int, 2 * p>(), j_, fx[0], fw[st & 1][j], e);
              product(integral_constant<int, 2 * p + 1>(), j_, fx[1], fw[st & 1][j], e);
            }
          }
        };
        column(integral_constant<int, 0>()); column(integral_constant<int, 1>()); column(integral_constant<int, 2>()); column(integral_constant<int, 3>());
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (KIND == LIN_MX && p == TP - 1) gather_codes(kt + 1);
        if constexpr (TURNS) meet();
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    pair(integral_constant<int, 0>()); pair(integral_constant<int, 1>()); pair(integral_constant<int, 2>()); pair(integral_constant<int, 3>());
  };
  for (int kt = 0;;) {
    step(lower, kt);
    if (++kt >= nk) break;
    step(upper, kt);
    if (++kt >= nk) break;
    if constexpr (STAGES == 4) {
      step(integral_constant<int, 2>(), kt);
      if (++kt >= nk) break;
      step(integral_constant<int, 3>(), kt);
      if (++kt >= nk) break;
    }
  }
  if (TURNS && w < 4) meet();
  wait_vmcnt<0>();  // (the zeros of the steps behind the last)
  __builtin_amdgcn_s_waitcnt(0xc07f);
  meet();

  linear_epilogue<TM, TN, MX_OUT>(a, acc, reinterpret_cast<float *>(lds) + w * kEpilogueFloats<TN>, m0 + wm * WTM, n0 + wn * WTN, lane);
}

template <int KIND, int BM, int BN, int WM, int WN, int STAGES>
static void go(const LinArgs &a, bool mx_out, hipStream_t st) {
  const int tm = (a.rows + BM - 1) / BM;
  const int tn = (a.N + BN - 1) / BN;
  const dim3 grid((unsigned)(tm * (long long)tn)), block(64 * WM * WN);
  if constexpr (KIND == LIN_MX) {
    if (mx_out) {
      hipLaunchKernelGGL((k_linear_tile<KIND, BM, BN, WM, WN, STAGES, true>), grid, block, 0, st, a, tm, tn);
      return;
    }
  }
  hipLaunchKernelGGL((k_linear_tile<KIND, BM, BN, WM, WN, STAGES, false>), grid, block, 0, st, a, tm, tn);
}

template <int KIND> static void pick(bool large, const LinArgs &a, bool mx_out, hipStream_t st) {
  if (large) return go<KIND, 256, 256, 2, 4, 2>(a, mx_out, st);
  if (medium_alone(a.rows, a.N)) return go<KIND, 128, 128, 2, 4, 4>(a, mx_out, st);
  go<KIND, 128, 128, 2, 4, 2>(a, mx_out, st);
}

void launch_linear_tile(int kind, bool large, const LinArgs &a, bool mx_out, hipStream_t st) {
  if (kind == LIN_MX) pick<LIN_MX>(large, a, mx_out, st);
  else pick<LIN_BF16>(large, a, mx_out, st);
}

}  // namespace toma
