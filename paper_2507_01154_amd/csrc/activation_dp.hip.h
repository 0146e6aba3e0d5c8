// Backward pass of a linear layer's activation and bias: dZ = dY act'(Z) and the bias's per-sample gradient g_i = sum_t dZ_it, as
// partial sums over chunks of tokens for vector_dp.hip.h.  The bias's sums are taken before dZ is rounded.
//
// Memory bound: dY and Z in, dZ out, 6 bytes an element in 16-bit types and 5 with Z in 8 bits.  A thread owns one chunk of 16 bytes of
// a row and goes down the tokens of its workgroup's chunk, so the sums over tokens stay in registers; the rows of
// threads join theirs in LDS at the end.  Four rows' loads are in flight per thread.
//
// 8192 x 3072 bf16, GELU (tanh form), Z in 8 bits, 8 samples: 25 us = 5.0 TB/s, the vector instructions close behind the bytes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "activations.hip.h"
#include "checkpoint8.hip.h"
#include "vector_io.hip.h"

namespace flashdp {

enum : int { Z_NONE = 0, Z_SAME = 1, Z_EIGHT = 2 };   // how Z is kept

struct ActivationArgs {
  const void* dY;                 // [B][T][d]
  const void* Z;                  // [B * T][d], or the q of a checkpoint
  const unsigned char* scales;    // of a checkpoint
  void* dZ;                       // may be null, may be dY
  float* partial;                 // [B][chunks][d]; may be null
  double* squares;                // [B][col_tiles] sums of squares, where chunks == 1
  int64_t B, T, d;
  int chunks, rows_per_chunk;
  int col_tiles, log_ct;          // threads side by side: 1 << log_ct, chunks of 16 bytes each
};

// TOKEN: T == 1, a row is a sample and its gradient dZ itself: the rows of threads take a sample each (and nothing is joined).
template <int DT, int ACT, int ZK, bool TOKEN>
__global__ __launch_bounds__(256) void activation_dp_kernel(const ActivationArgs a) {
  constexpr int N = Chunk<DT>::N, UNROLL = 4;
  __shared__ float part[TOKEN ? 1 : 256 * N];
  __shared__ double square[4];
  const int ct = 1 << a.log_ct, rt = 256 >> a.log_ct;
  const int c = threadIdx.x & (ct - 1), r = threadIdx.x >> a.log_ct;
  const int64_t unit = blockIdx.x / a.col_tiles;                       // (sample, chunk of tokens), or rt samples
  const int64_t col = ((int64_t)(blockIdx.x - unit * a.col_tiles) * ct + c) * N, left = a.d - col;
  int64_t row0, row1;                                                  // rows of [B * T]
  if constexpr (TOKEN) {
    row0 = unit * rt;
    row1 = row0 + rt < a.B ? row0 + rt : a.B;
  } else {
    const int64_t i = unit / a.chunks, k = unit - i * a.chunks;
    row0 = i * a.T + k * a.rows_per_chunk;
    row1 = (k + 1) * a.rows_per_chunk < a.T ? row0 + a.rows_per_chunk : (i + 1) * a.T;
  }
  const int64_t nb = checkpoint8_blocks(a.d);
  float sum[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = 0.0f;
  if (TOKEN || left > 0) {      // (TOKEN: threads beyond the row's end take part in its sum of squares, with zeros)
    const int64_t at = (row0 + r) * a.d + col, step = (int64_t)rt * a.d;          // elements; from row to row of this thread
    const char* dyp = (const char*)a.dY + at * Chunk<DT>::BYTES;
    const char* zp = (const char*)a.Z + at * (ZK == Z_EIGHT ? 1 : Chunk<DT>::BYTES);
    const unsigned char* sp = a.scales + (row0 + r) * nb + col / CKPT8_BLOCK;
    char* dzp = (char*)a.dZ + at * Chunk<DT>::BYTES;
    const int64_t step_b = step * Chunk<DT>::BYTES, step_z = ZK == Z_EIGHT ? step : step_b, step_s = rt * nb;
    for (int64_t row = row0 + r; row < row1; row += (int64_t)rt * UNROLL) {
      u32x4_t dy[UNROLL], zr[UNROLL];
      uint32_t zq[UNROLL][N / 4];
      int sc[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (row + (int64_t)u * rt < row1) {
          dy[u] = load_chunk<DT>(dyp + u * step_b, 0, left);
          if constexpr (ZK == Z_SAME) zr[u] = load_chunk<DT>(zp + u * step_z, 0, left);
          if constexpr (ZK == Z_EIGHT) {
            load_q<N>((const signed char*)zp + u * step_z, left, zq[u]);
            sc[u] = !TOKEN || left > 0 ? sp[u * step_s] : 127;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (row + (int64_t)u * rt < row1) {
          float f[N], z[N];
          widen_chunk<DT>(dy[u], f);
          if constexpr (ZK == Z_SAME) widen_chunk<DT>(zr[u], z);
          if constexpr (ZK == Z_EIGHT) checkpoint8_values<N>(zq[u], power_of_two(sc[u] - 127), z);
#pragma unroll
          for (int k = 0; k < N; ++k) {
            if constexpr (ZK != Z_NONE) f[k] *= act_slope<ACT>(z[k]);
            sum[k] += f[k];
          }
          if (a.dZ) store_chunk<DT>(dzp + u * step_b, 0, left, round_chunk<DT>(f));
          if constexpr (TOKEN) {
            if (a.partial) {
#pragma unroll
              for (int q = 0; q < N / 4; ++q)
                store_chunk<DT_F32>(a.partial + at + u * step, 4 * q, left - 4 * q,
                                    u32x4_t{__builtin_bit_cast(uint32_t, f[4 * q]), __builtin_bit_cast(uint32_t, f[4 * q + 1]),
                                            __builtin_bit_cast(uint32_t, f[4 * q + 2]), __builtin_bit_cast(uint32_t, f[4 * q + 3])});
              double q = 0.0;
#pragma unroll
              for (int k = 0; k < N; ++k) q += (double)f[k] * (double)f[k];
              for (int off = ct >> 1; off > 0; off >>= 1) q += __shfl_xor(q, off, 64);
              if (c == 0) a.squares[(row + (int64_t)u * rt) * a.col_tiles + (blockIdx.x - unit * a.col_tiles)] = q;
            }
          }
        }
      }
      dyp += UNROLL * step_b;
      zp += UNROLL * step_z;
      sp += UNROLL * step_s;
      dzp += UNROLL * step_b;
    }
  }
  if constexpr (!TOKEN) {
    if (!a.partial) return;
#pragma unroll
    for (int k = 0; k < N; ++k) part[k * 256 + threadIdx.x] = sum[k];
    __syncthreads();
    // element e of the column tile: its N ct sums lie at [e % N][.. e / N ..]; one thread per element, neighbours side by side
    float* to = a.partial + unit * a.d;
    const int64_t first = (int64_t)(blockIdx.x - unit * a.col_tiles) * ct * N;
    double q = 0.0;
    for (int e = threadIdx.x; e < ct * N; e += 256) {
      if (first + e >= a.d) break;
      const float* p = part + (e % N) * 256 + e / N;
      float s = 0.0f;
      for (int k = 0; k < rt; ++k) s += p[k * ct];
      to[first + e] = s;
      q += (double)s * (double)s;
    }
    if (a.chunks > 1) return;
    q = wave_sum(q);
    if ((threadIdx.x & 63) == 0) square[threadIdx.x >> 6] = q;
    __syncthreads();
    if (threadIdx.x == 0) a.squares[blockIdx.x] = (square[0] + square[1]) + (square[2] + square[3]);
  }
}

}  // namespace flashdp
