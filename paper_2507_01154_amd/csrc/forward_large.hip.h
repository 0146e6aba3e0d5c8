// The forward product on large tiles, for rows of whole 16-byte chunks: 256 tokens x 256 features by eight waves of 128 x 64, or
// 128 x 128 by four waves of 64 x 64, two workgroups to a compute unit.
//
// k-tiles of 128 bytes a row (whole cache lines) go from memory straight to LDS (buffer_load ... lds), into one of
// two stages: while k-tile k is multiplied, k + 1 is on its way.  One direct load of a wave writes 1 KB of LDS, eight rows,
// so rows cannot be padded; instead the 16-byte chunk c of row r is kept at position c ^ ((r / 2) % 8): the 16 rows of a fragment read at one
// chunk then lie in 16 different groups of four banks.  The lane that fills position p fetches chunk p ^ ((r / 2) % 8).
//
// A k-step (64 bytes) is walked in four quadrants of half the blocks each way in an order that lets every half-set of fragments be overwritten as
// soon as its last quadrant is issued - lo x first, lo x second, hi x second, hi x first, the halves of W changing roles from step to step -
// with the reads of a quadrant issued one to two quadrants ahead.  The order is held by scheduling barriers; the waits for LDS are the
// compiler's, those for the direct loads, which it does not see, are written by hand.
//
// Bound by the matrix cores at the clock they hold: bf16 8192 x 5120 -> 13824 with SiLU and Z 948 us = 1.22 PFLOP/s on 256 x 256.  Short
// rows by the epilogues, which workgroups that started together reach together: 8192 x 768 -> 3072 on 128 x 128 51 us, with GELU and Z
// in 8 bits 62 (every second workgroup started 4 us late: 1.6 us more).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "forward_common.hip.h"
#include "gemm_mfma_dma.hip.h"

namespace flashdp {

template <int FM_, int FN_, int WAVES_M_, int WAVES_N_>
struct ForwardLargeCfg {
  static constexpr int FM = FM_, FN = FN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WAVES = WAVES_M * WAVES_N;
  static constexpr int BM = 16 * FM * WAVES_M, BN = 16 * FN * WAVES_N, NT = 64 * WAVES, ROW = 128;      // ROW: bytes of a k-tile's row
  static constexpr int X_STAGE = BM * ROW, W_STAGE = BN * ROW, OPERANDS = 2 * (X_STAGE + W_STAGE);    // X stages 0, 1, then W stages 0, 1
  static constexpr int EPILOGUE = WAVES * ForwardStage<FM, FN>::BYTES;
  static constexpr int LDS_BYTES = EPILOGUE > OPERANDS ? EPILOGUE : OPERANDS;
  static constexpr int X_LOADS = BM / 8 / WAVES, W_LOADS = BN / 8 / WAVES;       // direct loads of 8 rows, per wave and k-tile
  static_assert(FM % 2 == 0 && FN == 4 && WAVES % 2 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "quadrants, whole loads");
};

__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <typename Cfg, int DT>
__global__ __launch_bounds__(Cfg::NT, 2) void forward_large_kernel(const ForwardArgs a) {
  constexpr int ROW = Cfg::ROW, FM = Cfg::FM, FN = Cfg::FN, BM = Cfg::BM, BN = Cfg::BN, HALF = FM / 2;
  extern __shared__ __attribute__((aligned(16))) char large_lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave % Cfg::WAVES_M, wave_n = wave / Cfg::WAVES_M;
  int tm, tn;
  tile_coords<8>(xcd_remap(blockIdx.x, a.tiles_m * a.tiles_n), a.tiles_m, a.tiles_n, &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;

  // ---- direct loads: instruction q of this wave fills rows 8 (WAVES q + wave) .. + 7 of an operand's tile
  const uint32_t kb = (uint32_t)a.K * Chunk<DT>::BYTES;                    // bytes of a row
  const int l_row = 8 * wave + (lane >> 3);
  const uint32_t l_col = (uint32_t)(((lane & 7) ^ ((l_row >> 1) & 7)) * 16);   // (the same for every q: 8 WAVES is a multiple of 16)
  const uint32_t x_rows = (uint32_t)min((int64_t)BM, a.rows - m0), w_rows = (uint32_t)min(BN, a.D - n0);
  const u32x4_t x_rsrc = make_rsrc_words((const char*)a.X + m0 * kb, x_rows * kb);
  const u32x4_t w_rsrc = make_rsrc_words((const char*)a.W + (int64_t)n0 * kb, w_rows * kb);
  const uint32_t l_off = (uint32_t)l_row * kb + l_col, l_stride = 8u * Cfg::WAVES * kb;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)large_lds;
  const uint32_t l_dst = lds_base + (uint32_t)wave * 1024u;
  const int nk = (int)((kb + ROW - 1) / ROW);
  uint32_t l_k = 0;                                                        // bytes into the rows of the next k-tile to fetch
  auto issue_loads = [&](int stage) {
    // beyond the row's end (or the last k-tile): out of the buffer, reads zeros
    const uint32_t off = l_k + l_col < kb ? l_off + l_k : 0x80000000u;
#pragma unroll
    for (int q = 0; q < Cfg::X_LOADS; ++q) load_to_lds(x_rsrc, off + q * l_stride, l_dst + stage * Cfg::X_STAGE + q * (Cfg::WAVES * 1024));
#pragma unroll
    for (int q = 0; q < Cfg::W_LOADS; ++q)
      load_to_lds(w_rsrc, off + q * l_stride, l_dst + 2 * Cfg::X_STAGE + stage * Cfg::W_STAGE + q * (Cfg::WAVES * 1024));
    l_k += ROW;
  };

  // ---- fragments: row lane % 16 of a block of 16, chunk 4 step + lane / 16
  const int f_row = lane & 15, f_pos = ((lane >> 4) ^ ((f_row >> 1) & 7)) * 16;
  const char* x_rd[2];
  const char* w_rd[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    x_rd[s] = large_lds + (wave_m * 16 * FM + f_row) * ROW + (f_pos ^ (64 * s));
    w_rd[s] = large_lds + 2 * Cfg::X_STAGE + (wave_n * 16 * FN + f_row) * ROW + (f_pos ^ (64 * s));
  }

  f32x4v_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4v_t{0.0f, 0.0f, 0.0f, 0.0f};

  u32x4_t xlo[HALF], xhi[HALF], wa[2], wb[2], wc[2];
  auto read_x = [&](int cur, int half, int f) { return *(const u32x4_t*)(x_rd[cur & 1] + (cur >> 1) * Cfg::X_STAGE + (HALF * half + f) * 16 * ROW); };
  auto read_w = [&](int cur, int half, int f) { return *(const u32x4_t*)(w_rd[cur & 1] + (cur >> 1) * Cfg::W_STAGE + (2 * half + f) * 16 * ROW); };
  auto quadrant = [&](const u32x4_t* x, int i0, const u32x4_t* w, int j0, auto&& after) {
    static_for<2 * HALF>([&](auto m_c) {
      constexpr int m = decltype(m_c)::value, i = m / 2, j = m % 2;
      acc[i0 + i][j0 + j] = k_step<DT>(w[j], x[i], acc[i0 + i][j0 + j]);
      after(m_c);
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  issue_loads(0);
  wait_loads_outstanding<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int f = 0; f < 2; ++f) wa[f] = read_w(0, 0, f);
#pragma unroll
  for (int f = 0; f < HALF; ++f) xlo[f] = read_x(0, 0, f);
#pragma unroll
  for (int f = 0; f < 2; ++f) wb[f] = read_w(0, 1, f);
  __builtin_amdgcn_sched_barrier(0);

  // k-step `cur` = 2 stage + step.  Even steps: first half of W = columns 0-1 (in wa), second = 2-3 (wb); the next step's first half, its
  // columns 2-3, goes to wc, and its second half, columns 0-1, to wb.  Odd steps: first = columns 2-3 (wc), second = 0-1 (wb), next to wa, wb.
  auto step = [&](auto cur_c) {
    constexpr int cur = decltype(cur_c)::value, PARITY = cur & 1, nxt = (cur + 1) & 3;
    u32x4_t* const first = PARITY == 0 ? wa : wc;
    u32x4_t* const next_first = PARITY == 0 ? wc : wa;
    constexpr int j1 = 2 * PARITY, j2 = 2 - 2 * PARITY;
    quadrant(xlo, 0, first, j1, [&](auto m_c) {
      constexpr int m = decltype(m_c)::value;
      if constexpr (m < HALF) xhi[m] = read_x(cur, 1, m);
      if constexpr (PARITY == 0 && m == HALF) issue_loads((cur >> 1) ^ 1);
    });
    quadrant(xlo, 0, wb, j2, [&](auto) {});
    if constexpr (PARITY == 1) wait_loads_outstanding<0>();
    quadrant(xhi, HALF, wb, j2, [&](auto m_c) {
      constexpr int m = decltype(m_c)::value;
      if constexpr (PARITY == 1 && m == 0) {
        wait_lds_reads();                      // of the stage that is refilled next
        __builtin_amdgcn_s_barrier();          // every wave's loads of the next k-tile have landed
        asm volatile("" ::: "memory");
      }
      if constexpr (m < 2) next_first[m] = read_w(nxt, 1 - PARITY, m);
      if constexpr (m >= 2 && m < 2 + HALF) xlo[m - 2] = read_x(nxt, 0, m - 2);
      if constexpr (HALF < 4 && m == 2 * HALF - 1)      // (quadrants of four instructions: the rest of the reads at their end)
#pragma unroll
        for (int f = 2 * HALF - 2; f < HALF; ++f) xlo[f] = read_x(nxt, 0, f);
    });
    quadrant(xhi, HALF, first, j1, [&](auto m_c) {
      constexpr int m = decltype(m_c)::value;
      if constexpr (m < 2) wb[m] = read_w(nxt, PARITY, m);
    });
  };
  // two k-tiles a trip; an odd one out is multiplied with the zeros that loads beyond the end deliver
  for (int k = 0; k < nk; k += 2) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }
  wait_loads_outstanding<0>();                 // (zeros on their way to the stages)
  wait_lds_reads();
  __syncthreads();
  forward_epilogue<DT, FM, FN>(a, acc, m0 + wave_m * 16 * FM, n0 + wave_n * 16 * FN, (float*)(large_lds + wave * ForwardStage<FM, FN>::BYTES));
}

using ForwardLarge256 = ForwardLargeCfg<8, 4, 2, 4>;
using ForwardLarge128 = ForwardLargeCfg<4, 4, 2, 2>;

}  // namespace flashdp
