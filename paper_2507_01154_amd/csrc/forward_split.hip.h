// The forward product of fp32 operands on the bfloat16 matrix cores.
//
// A float is cut into three parts of 8 significant bits, a = a1 + a2 + a3 exactly: a1 is its upper half as it stands (rounded, the largest
// floats would become infinite), a2 the rounding of the rest, a3 what is left, each a bfloat16 number, and X W^T is the sum of six of the nine products of
// parts: 1 1, 1 2, 2 1, 2 2, 1 3, 3 1.  The other three are below 2^-22 of a product of operands together and of either sign (with a2 cut off as
// well they would be up to 2^-21 and of the product's sign).
//
// Matrix instructions cut small products off beside a large accumulator, always towards zero: with all of a sum in one accumulator, a row of
// products of one sign came out 8e-6 too small at K = 4096.  So the six products of a k-tile start from zero, that of the upper halves last, and their sum is
// added to the total by the vector unit, which rounds to nearest.  Off by at most some 8 times 2^-24 of the sum of magnitudes for the k-tiles and
// one for each of the K / 32 additions.  Relative errors in norm, fp32 instruction on 128 x 128 tiles, on 32 x 32 ones, where four waves share K, and
// here: normal operands, K = 64: 1.4e-7, 8.5e-8, 5.2e-8; K = 768: 5.0e-7, 2.5e-7, 1.1e-7; K = 4096: 1.1e-6, 5.8e-7, 2.2e-7; rectified
// normal times uniform, K = 64: 8.6e-8, 4.5e-8, 3.6e-8; K = 768: 3.0e-7, 8.5e-8, 7.8e-8; K = 4096: 6.6e-7, 1.7e-7, 1.7e-7.
// Parts below 2^-133 are lost (of numbers below 2^-110); an operand that is not finite has parts that are NaN.
//
// Six products at 16 times the rate of the fp32 instruction; what bounds it is the matrix cores and the clock they hold, with the vector unit's
// cutting and adding beside them (2048 x 4096 -> 4096: 317 us; in one accumulator and with all parts cut, 304; with a1 rounded, 330).
//
// Tiles of 128 tokens x 256 features by eight waves of 64 x 64, or 64 x 128 by four of 32 x 64, two workgroups to a compute unit.  k-tiles of 32 go through registers, where they are cut, into one of two LDS stages of
// three planes with rows of 64 bytes; the 16-byte chunk c of row r is kept at c ^ ((r / 4) % 4), so that the 16 rows of a fragment read lie in 16
// different groups of four banks.  The next k-tile is cut beside the matrix instructions, a chunk to each sixth of them, in an order that is
// asked of the compiler (before the sums had two levels: 395 us with the cutting behind the products, 303 so).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "forward_common.hip.h"

namespace flashdp {

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_>
struct ForwardSplitCfg {
  static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WAVES = WAVES_M * WAVES_N, NT = 64 * WAVES;
  static constexpr int FM = BM / 16 / WAVES_M, FN = BN / 16 / WAVES_N;
  static constexpr int ROW = 64, PLANE = (BM + BN) * ROW, STAGE = 3 * PLANE;
  static constexpr int X_LOADS = BM * 8 / NT, LOADS = (BM + BN) * 8 / NT;   // chunks of four floats per thread and k-tile, X's first
  static constexpr int EPILOGUE = WAVES * ForwardStage<FM, FN>::BYTES;
  static constexpr int LDS_BYTES = 2 * STAGE > EPILOGUE ? 2 * STAGE : EPILOGUE;
  static_assert(LOADS == 6 && BM * 8 % NT == 0 && NT % 128 == 0, "one chunk is cut beside each of the six products; rows 16 apart share a swizzle");
};

// ANY: rows are no whole chunks of four floats, the last of a row is cut off element by element.
template <typename Cfg, bool ANY>
__global__ __launch_bounds__(Cfg::NT, 2) void forward_split_kernel(const ForwardArgs a) {
  constexpr int LOADS = Cfg::LOADS, X_LOADS = Cfg::X_LOADS, FM = Cfg::FM, FN = Cfg::FN, BLOCKS = FM * FN;
  extern __shared__ __attribute__((aligned(16))) char split_lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave % Cfg::WAVES_M, wave_n = wave / Cfg::WAVES_M;
  int tm, tn;
  tile_coords<8>(xcd_remap(blockIdx.x, a.tiles_m * a.tiles_n), a.tiles_m, a.tiles_n, &tm, &tn);
  const int64_t m0 = (int64_t)tm * Cfg::BM;
  const int n0 = tn * Cfg::BN;

  const uint32_t kb = (uint32_t)a.K * 4u;
  const uint32_t x_rows = (uint32_t)min((int64_t)Cfg::BM, a.rows - m0), w_rows = (uint32_t)min(Cfg::BN, a.D - n0);
  const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc((const char*)a.X + m0 * kb, x_rows * kb);
  const __amdgpu_buffer_rsrc_t w_rsrc = make_rsrc((const char*)a.W + (int64_t)n0 * kb, w_rows * kb);
  const uint32_t l_col = (uint32_t)(tid & 7) * 16u, l_off = (uint32_t)(tid >> 3) * kb + l_col, l_stride = (uint32_t)(Cfg::NT / 8) * kb;
  u32x4_t raw[LOADS];
  // Chunk q of k-tile kt.  Rows that do not exist and chunks beyond a row's end lie outside the buffer (or are sent there) and read zeros.
  auto fetch = [&](int q, int kt) {
    const uint32_t at = (uint32_t)kt * 128u, off = at + l_col < kb ? l_off + at : 0x80000000u;
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(q < X_LOADS ? x_rsrc : w_rsrc, (int)(off + (uint32_t)(q < X_LOADS ? q : q - X_LOADS) * l_stride), 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) raw[q][e] = v[e];
  };
  const int s_at = (tid >> 3) * Cfg::ROW + ((((tid & 7) >> 1) ^ ((tid >> 5) & 3)) * 16) + (tid & 1) * 8;
  auto cut = [&](int q, int kt) {      // chunk q of k-tile kt, into stage kt % 2
    uint2 p[3];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) v[e] = !ANY || (uint32_t)kt * 128u + l_col + 8u * h + 4u * e < kb ? as_float(raw[q][2 * h + e]) : 0.0f;
      const uint32_t p1 = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[0]), 0x07060302u);
      const float r0 = v[0] - as_float(p1 << 16), r1 = v[1] - as_float(p1 & 0xFFFF0000u);
      const uint32_t p2 = pack2_16bit<DT_BF16>(r0, r1);
      const uint32_t p3 = pack2_16bit<DT_BF16>(r0 - as_float(p2 << 16), r1 - as_float(p2 & 0xFFFF0000u));
      (h ? p[0].y : p[0].x) = p1;
      (h ? p[1].y : p[1].x) = p2;
      (h ? p[2].y : p[2].x) = p3;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *(uint2*)(split_lds + (kt & 1) * Cfg::STAGE + k * Cfg::PLANE + q * (Cfg::NT / 8) * Cfg::ROW + s_at) = p[k];
  };

  const int f_at = (lane & 15) * Cfg::ROW + (((lane >> 4) ^ ((lane >> 2) & 3)) * 16);
  const char* x_rd = split_lds + wave_m * 16 * FM * Cfg::ROW + f_at;
  const char* w_rd = split_lds + (Cfg::BM + wave_n * 16 * FN) * Cfg::ROW + f_at;
  f32x4v_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4v_t{0.0f, 0.0f, 0.0f, 0.0f};

  const int nk = (a.K + 31) / 32;
#pragma unroll
  for (int q = 0; q < LOADS; ++q) fetch(q, 0);
#pragma unroll
  for (int q = 0; q < LOADS; ++q) cut(q, 0);
#pragma unroll
  for (int q = 0; q < LOADS; ++q) fetch(q, 1);      // (k-tiles beyond the last: zeros)
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const int cur = (kt & 1) * Cfg::STAGE;
    u32x4_t x[3][FM], w[3][FN];
    auto read_x = [&](int p) {
#pragma unroll
      for (int i = 0; i < FM; ++i) x[p][i] = *(const u32x4_t*)(x_rd + cur + p * Cfg::PLANE + i * 16 * Cfg::ROW);
    };
    auto read_w = [&](int p, int j) { w[p][j] = *(const u32x4_t*)(w_rd + cur + p * Cfg::PLANE + j * 16 * Cfg::ROW); };
    // in the order of their use
    read_w(2, 0);
    read_x(0);
    read_w(1, 0);
    read_x(1);
    read_w(0, 0);
    read_x(2);
#pragma unroll
    for (int j = 1; j < FN; ++j)
#pragma unroll
      for (int p = 2; p >= 0; --p) read_w(p, j);
    // A column of blocks at a time: its six products from zero on, the largest last, then added to the sums by the vector
    // unit, among the next column's.  Beside every sixth of them a chunk of the next k-tile is cut and one of the k-tile after it loaded.
    constexpr int WP[6] = {2, 1, 1, 0, 0, 0}, XP[6] = {0, 0, 1, 1, 2, 0};
    f32x4v_t part[2][FM];
    static_for<6 * BLOCKS>([&](auto m_c) {
      constexpr int m = decltype(m_c)::value, j = m / (6 * FM), t = m / FM % 6, i = m % FM;
      part[j & 1][i] = k_step<DT_BF16>(w[WP[t]][j], x[XP[t]][i], t == 0 ? f32x4v_t{0.0f, 0.0f, 0.0f, 0.0f} : part[j & 1][i]);
      if constexpr (j > 0 && t == 1) acc[i][j - 1] += part[(j & 1) ^ 1][i];
      if constexpr (m % BLOCKS == BLOCKS - 1) {
        cut(m / BLOCKS, kt + 1);      // into the stage that k-tile kt - 1 was read from, before the last barrier
        fetch(m / BLOCKS, kt + 2);
      }
    });
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[i][FN - 1] += part[(FN - 1) & 1][i];
    __builtin_amdgcn_sched_group_barrier(0x100, FM + 1, 0);      // the first product's fragments, then one instruction after the other
    static_for<6 * BLOCKS>([&](auto g_c) {
      constexpr int g = decltype(g_c)::value;
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                   // matrix
      __builtin_amdgcn_sched_group_barrier(0x002, BLOCKS >= 16 ? 2 : 3, 0);                // vector
      if constexpr (g < 3 * (FM + FN) - FM - 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);       // LDS read
      if constexpr (g % BLOCKS == BLOCKS - 1) {
        __builtin_amdgcn_sched_group_barrier(0x200, 3, 0);                                 // LDS write
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);                                 // load
      }
    });
    __syncthreads();
  }
  forward_epilogue<DT_F32, FM, FN>(a, acc, m0 + wave_m * 16 * FM, n0 + wave_n * 16 * FN, (float*)(split_lds + wave * ForwardStage<FM, FN>::BYTES));
}

}  // namespace flashdp
