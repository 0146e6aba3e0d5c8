// The forward product on tiles of BM tokens x BN features, for rows that may start anywhere (K no multiple of 16 bytes).
//
// Four waves, 2 x 2; k-tiles of 128 bytes a row go through registers (loads of any alignment, zeros beyond the ends) into one of two LDS
// buffers, one barrier per k-tile.  Rows of LDS are 144 bytes apart, so that the 16 rows that a fragment read meets at one 16-byte column
// start in 16 different groups of four banks.
//
// Bound by the loads, 16 bytes at any address: bf16 64 x 4097 -> 4096 66 us, 64 x 4098 -> 4096 60, 8 x 769 -> 50257 24 us = 3.2 TB/s of W; on 128 x 128
// tiles 1024 x 4097 -> 4096 103 us = 0.33 PFLOP/s.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "forward_common.hip.h"

namespace flashdp {

template <int BM_, int BN_>
struct ForwardTileCfg {
  static constexpr int BM = BM_, BN = BN_, NT = 256, PITCH = 144, ROWS = BM + BN;
  static constexpr int CHUNKS = ROWS * 8 / NT;               // 16-byte chunks per thread and k-tile
  static constexpr int LDS_BYTES = 2 * ROWS * PITCH;
  static constexpr int FM = BM / 32, FN = BN / 32;           // 16 x 16 blocks per wave
  static_assert(4 * ForwardStage<FM, FN>::BYTES <= LDS_BYTES, "the epilogue's stages lie in the operand buffers");
};

template <typename Cfg, int DT>
__global__ __launch_bounds__(Cfg::NT) void forward_tile_kernel(const ForwardArgs a) {
  constexpr int N = Chunk<DT>::N, BM = Cfg::BM, BN = Cfg::BN, PITCH = Cfg::PITCH, FM = Cfg::FM, FN = Cfg::FN;
  extern __shared__ __attribute__((aligned(16))) char tiles_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int tm, tn;
  tile_coords<8>(xcd_remap(blockIdx.x, a.tiles_m * a.tiles_n), a.tiles_m, a.tiles_n, &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;
  const int nk = (a.K + 8 * N - 1) / (8 * N);

  // chunk q of this thread: row (tid + 256 q) / 8 of the tile pair (tokens first), 16-byte column (tid + 256 q) % 8
  const char* src[Cfg::CHUNKS];
  bool in[Cfg::CHUNKS];
  const int c8 = tid & 7;
#pragma unroll
  for (int q = 0; q < Cfg::CHUNKS; ++q) {
    const int r = (tid >> 3) + 32 * q;
    const bool x = r < BM;
    const int64_t row = x ? m0 + r : n0 + r - BM;
    in[q] = row < (x ? a.rows : a.D);
    src[q] = (const char*)(x ? a.X : a.W) + (in[q] ? row : 0) * a.K * Chunk<DT>::BYTES;
  }
  u32x4_t stage[Cfg::CHUNKS];
  auto fetch = [&](int kt) {
    const int col = (kt * 8 + c8) * N;
#pragma unroll
    for (int q = 0; q < Cfg::CHUNKS; ++q) stage[q] = load_chunk<DT>(src[q], col, in[q] ? a.K - col : 0);
  };
  auto put = [&](int buf) {
    char* to = tiles_lds + buf * Cfg::ROWS * PITCH + (tid >> 3) * PITCH + c8 * 16;
#pragma unroll
    for (int q = 0; q < Cfg::CHUNKS; ++q) *(u32x4_t*)(to + 32 * q * PITCH) = stage[q];
  };

  f32x4v_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4v_t{0.0f, 0.0f, 0.0f, 0.0f};
  const int wm = (wave & 1) * (BM / 2), wn = (wave >> 1) * (BN / 2);
  const int x_rd = (wm + (lane & 15)) * PITCH + (lane >> 4) * 16, w_rd = (BM + wn + (lane & 15)) * PITCH + (lane >> 4) * 16;

  fetch(0);
  put(0);
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const char* cur = tiles_lds + (kt & 1) * Cfg::ROWS * PITCH;
    if (kt + 1 < nk) fetch(kt + 1);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4_t x[FM], w[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) x[i] = *(const u32x4_t*)(cur + x_rd + 16 * i * PITCH + 64 * ks);
#pragma unroll
      for (int j = 0; j < FN; ++j) w[j] = *(const u32x4_t*)(cur + w_rd + 16 * j * PITCH + 64 * ks);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = k_step<DT>(w[j], x[i], acc[i][j]);
    }
    if (kt + 1 < nk) put((kt + 1) & 1);      // the buffer that k-tile kt - 1 was read from, before the last barrier
    __syncthreads();
  }
  forward_epilogue<DT, FM, FN>(a, acc, m0 + wm, n0 + wn, (float*)(tiles_lds + wave * ForwardStage<FM, FN>::BYTES));
}

}  // namespace flashdp
