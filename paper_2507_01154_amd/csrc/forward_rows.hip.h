// The forward product of few rows (tokens of a generating model) whose K no 16-byte chunk divides, so that rows of W start anywhere: W is
// read once, and that is the time.
//
// A workgroup owns 16 NF features.  Its waves share out the k-steps (64 bytes of every row) in turn, so that together they walk along
// the rows of W in whole cache lines; every wave multiplies 16 NF features with 16 MT tokens straight from memory, up to eight k-steps' loads in
// flight, and the waves' partial sums are joined in LDS in a fixed order.  Rows that do not exist repeat the last one that does: a sum
// belongs to one row of each operand, and those are not kept.
//
// Bound by the loads, 16 bytes at any address: bf16 1 x 4097 -> 4096, where every other row starts at an odd multiple of two bytes, 28 us, 64 rows 76;
// 1 x 4098 -> 4096, at multiples of four, 16 us = 2.1 TB/s of W, 64 rows 34; fp32 1 x 4097 -> 4096 28 us = 2.4 TB/s.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "forward_common.hip.h"

namespace flashdp {

template <int NF_, int MT_, int WAVES_>
struct ForwardRowsCfg {
  static constexpr int NF = NF_, MT = MT_, WAVES = WAVES_, NT = 64 * WAVES;
  static constexpr int UNROLL = 8 / (NF > MT ? NF : MT) > 1 ? 8 / (NF > MT ? NF : MT) : 2;   // k-steps in flight
  static constexpr int PITCH = 16 * NF + 4;                                                 // floats
  static constexpr int LDS_BYTES = WAVES * 16 * MT * PITCH * 4;
};

template <typename Cfg, int DT>
__global__ __launch_bounds__(Cfg::NT) void forward_rows_kernel(const ForwardArgs a) {
  constexpr int NF = Cfg::NF, MT = Cfg::MT, WAVES = Cfg::WAVES, UNROLL = Cfg::UNROLL, PITCH = Cfg::PITCH;
  extern __shared__ __attribute__((aligned(16))) float rows_lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16 * NF;
  const int64_t kb = (int64_t)a.K * Chunk<DT>::BYTES;
  const int c = (lane >> 4) * 16;                        // bytes into a k-step
  const char* w[NF];
  const char* x[MT];
#pragma unroll
  for (int f = 0; f < NF; ++f) w[f] = (const char*)a.W + min(n0 + 16 * f + (lane & 15), a.D - 1) * kb + c;
#pragma unroll
  for (int t = 0; t < MT; ++t) x[t] = (const char*)a.X + min((int64_t)(16 * t + (lane & 15)), a.rows - 1) * kb + c;
  f32x4v_t acc[NF][MT];
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[f][t] = f32x4v_t{0.0f, 0.0f, 0.0f, 0.0f};

  const int full = (int)(kb / 64);                       // whole k-steps
  int s = wave;
  if (s + (UNROLL - 1) * WAVES < full) {                 // batches of UNROLL k-steps, the next one's loads in flight while one is multiplied
    u32x4_t wr[2][UNROLL][NF], xr[2][UNROLL][MT];
    auto fetch = [&](int buf, int at) {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
        for (int f = 0; f < NF; ++f) wr[buf][u][f] = *(const u32x4_any_t*)(w[f] + (int64_t)(at + u * WAVES) * 64);
#pragma unroll
        for (int t = 0; t < MT; ++t) xr[buf][u][t] = *(const u32x4_any_t*)(x[t] + (int64_t)(at + u * WAVES) * 64);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](int buf) {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[f][t] = k_step<DT>(wr[buf][u][f], xr[buf][u][t], acc[f][t]);
      __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int BATCH = UNROLL * WAVES;
    fetch(0, s);
    s += BATCH;
    while (s + (UNROLL - 1) * WAVES < full) {
      fetch(1, s);
      s += BATCH;
      multiply(0);
      if (s + (UNROLL - 1) * WAVES >= full) {
        multiply(1);
        goto rest;
      }
      fetch(0, s);
      s += BATCH;
      multiply(1);
    }
    multiply(0);
  }
rest:
  for (; (int64_t)s * 64 < kb; s += WAVES) {                    // what is left, the last k-step in part perhaps
    const int64_t left = (kb - (int64_t)s * 64 - c) / Chunk<DT>::BYTES;
    u32x4_t wr[NF], xr[MT];
#pragma unroll
    for (int f = 0; f < NF; ++f) wr[f] = load_chunk<DT>(w[f] + (int64_t)s * 64, 0, left);
#pragma unroll
    for (int t = 0; t < MT; ++t) xr[t] = load_chunk<DT>(x[t] + (int64_t)s * 64, 0, left);
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[f][t] = k_step<DT>(wr[f], xr[t], acc[f][t]);
  }

  float* part = rows_lds + wave * 16 * MT * PITCH;
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int t = 0; t < MT; ++t) *(f32x4v_t*)(part + (16 * t + (lane & 15)) * PITCH + 16 * f + 4 * (lane >> 4)) = acc[f][t];
  __syncthreads();
  finish_partials<DT, Cfg::NT, WAVES, 16 * MT, 16 * NF>(a, rows_lds, 0, n0);
}

}  // namespace flashdp
