// The forward product on small tiles with many k-tiles in flight, for rows of whole 16-byte chunks: some tens to hundreds of rows, where the tiles
// of a layer do not fill the chip and a workgroup waits for memory, not for the matrix cores.
//
// k-tiles of 128 bytes a row go straight to LDS (buffer_load ... lds) into a ring of STAGES; UNROLL of them are multiplied between two barriers,
// and the loads that refill a stage are issued right behind the barrier after it was read, so STAGES - UNROLL k-tiles are on their
// way at any time.  The waves share out the k-steps among themselves before they share out the tile: a wave that multiplies a whole
// 64 x 64 tile reads 8 fragments of LDS for 16 instructions, one that multiplies a quarter of it 4 for 4, and LDS is what bounds
// small tiles.  Their partial sums are joined in LDS at the end, in a fixed order.  Swizzle and fragments as in forward_large.hip.h.
//
// bf16 1 x 4096 -> 4096: 7.2 us = 4.7 TB/s of W; fp16 8 x 768 -> 50257: 16.3 us = 4.7 TB/s; bf16 256 x 4096 -> 4096: 15.9 us (operands in the caches; from memory 21), bound by the rate at which
// direct loads fill LDS (about 33 bytes a clock and compute unit).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "forward_large.hip.h"

namespace flashdp {

template <int BM_, int BN_, int WAVES_K_, int WAVES_N_, int STAGES_, int UNROLL_>
struct ForwardDeepCfg {
  static constexpr int BM = BM_, BN = BN_, WAVES_K = WAVES_K_, WAVES_N = WAVES_N_, STAGES = STAGES_, UNROLL = UNROLL_;
  static constexpr int WAVES = WAVES_K * WAVES_N, NT = 64 * WAVES, ROW = 128;
  static constexpr int FM = BM / 16, FN = BN / 16 / WAVES_N, STAGE = (BM + BN) * ROW;
  static constexpr int LOADS = (BM + BN) / 8 / WAVES;            // direct loads of 8 rows per wave and k-tile
  static constexpr int STEPS = 2 * UNROLL / WAVES_K;             // k-steps per wave between two barriers
  static constexpr int PITCH = BN + 4, PARTIAL = BM * PITCH;     // floats
  static constexpr int EPILOGUE = WAVES_K * PARTIAL * 4;
  static constexpr int LDS_BYTES = EPILOGUE > STAGES * STAGE ? EPILOGUE : STAGES * STAGE;
  static_assert((BM + BN) % (8 * WAVES) == 0 && BM % 16 == 0 && 2 * UNROLL % WAVES_K == 0 && STAGES % UNROLL == 0 && STAGES >= 2 * UNROLL, "whole loads and steps");
  static_assert(LOADS * (STAGES - UNROLL) < 64, "the counter of loads in flight has six bits");
};

template <int N>
__device__ __forceinline__ void wait_loads_left() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

template <typename Cfg, int DT>
__global__ __launch_bounds__(Cfg::NT) void forward_deep_kernel(const ForwardArgs a) {
  constexpr int N = Chunk<DT>::N, ROW = Cfg::ROW, FM = Cfg::FM, FN = Cfg::FN, BM = Cfg::BM, BN = Cfg::BN, STAGES = Cfg::STAGES, UNROLL = Cfg::UNROLL;
  extern __shared__ __attribute__((aligned(16))) char deep_lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_k = wave % Cfg::WAVES_K, wave_n = wave / Cfg::WAVES_K;
  int tm, tn;
  tile_coords<8>(xcd_remap(blockIdx.x, a.tiles_m * a.tiles_n), a.tiles_m, a.tiles_n, &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;

  // ---- direct loads: instruction q of this wave fills rows 8 (LOADS wave + q) .. + 7 of the tile pair, tokens first
  const uint32_t kb = (uint32_t)a.K * Chunk<DT>::BYTES;
  const uint32_t x_rows = (uint32_t)min((int64_t)BM, a.rows - m0), w_rows = (uint32_t)min(BN, a.D - n0);
  const u32x4_t x_rsrc = make_rsrc_words((const char*)a.X + m0 * kb, x_rows * kb);
  const u32x4_t w_rsrc = make_rsrc_words((const char*)a.W + (int64_t)n0 * kb, w_rows * kb);
  uint32_t l_off[Cfg::LOADS], l_col[Cfg::LOADS];
#pragma unroll
  for (int q = 0; q < Cfg::LOADS; ++q) {
    const int block = Cfg::LOADS * wave + q, r = 8 * block + (lane >> 3), row = r < BM ? r : r - BM;
    l_col[q] = (uint32_t)(((lane & 7) ^ ((row >> 1) & 7)) * 16);
    l_off[q] = (uint32_t)row * kb + l_col[q];
  }
  const uint32_t l_dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)deep_lds + (uint32_t)(Cfg::LOADS * wave) * 1024u;
  const int nk = (int)((kb + ROW - 1) / ROW);
  uint32_t l_k = 0;
  int l_stage = 0;
  auto issue_loads = [&]() {       // of the next UNROLL k-tiles; beyond the last one zeros, so that the count of loads stays what the waits expect
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
      for (int q = 0; q < Cfg::LOADS; ++q) {
        const uint32_t off = l_k + l_col[q] < kb ? l_off[q] + l_k : 0x80000000u;
        load_to_lds(8 * (Cfg::LOADS * wave + q) < BM ? x_rsrc : w_rsrc, off, l_dst + (uint32_t)((l_stage + u) * Cfg::STAGE + q * 1024));
      }
      l_k += ROW;
    }
    l_stage = l_stage + UNROLL == STAGES ? 0 : l_stage + UNROLL;
  };

  const int f_row = lane & 15, f_pos = ((lane >> 4) ^ ((f_row >> 1) & 7)) * 16;
  const char* x_rd = deep_lds + f_row * ROW;
  const char* w_rd = deep_lds + (BM + wave_n * 16 * FN + f_row) * ROW;

  f32x4v_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4v_t{0.0f, 0.0f, 0.0f, 0.0f};

#pragma unroll
  for (int s = 0; s < STAGES / UNROLL - 1; ++s) issue_loads();
  int cur = 0;
  for (int k = 0; k < nk; k += UNROLL) {
    wait_lds_reads();                                              // of the k-tiles whose stages are refilled below
    wait_loads_left<Cfg::LOADS * (STAGES - 2 * UNROLL)>();         // k-tiles k .. k + UNROLL - 1 have landed
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    issue_loads();
    u32x4_t x[Cfg::STEPS][FM], w[Cfg::STEPS][FN];
#pragma unroll
    for (int s = 0; s < Cfg::STEPS; ++s) {
      const int step = s * Cfg::WAVES_K + wave_k;                  // of the 2 UNROLL between the barriers
      const int at = (cur + (step >> 1)) * Cfg::STAGE + (f_pos ^ (64 * (step & 1)));
#pragma unroll
      for (int j = 0; j < FN; ++j) w[s][j] = *(const u32x4_t*)(w_rd + at + j * 16 * ROW);
#pragma unroll
      for (int i = 0; i < FM; ++i) x[s][i] = *(const u32x4_t*)(x_rd + at + i * 16 * ROW);
    }
#pragma unroll
    for (int s = 0; s < Cfg::STEPS; ++s)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = k_step<DT>(w[s][j], x[s][i], acc[i][j]);
    cur = cur + UNROLL == STAGES ? 0 : cur + UNROLL;
  }
  wait_loads_left<0>();                                            // (zeros on their way to the stages)
  wait_lds_reads();
  __syncthreads();

  float* part = (float*)deep_lds;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *(f32x4v_t*)(part + wave_k * Cfg::PARTIAL + (16 * i + (lane & 15)) * Cfg::PITCH + (wave_n * FN + j) * 16 + 4 * (lane >> 4)) = acc[i][j];
  __syncthreads();
  finish_partials<DT, Cfg::NT, Cfg::WAVES_K, BM, BN>(a, part, m0, n0);
}

}  // namespace flashdp
