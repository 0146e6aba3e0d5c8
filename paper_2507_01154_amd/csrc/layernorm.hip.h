// Layer normalisation, forward and backward.
//
//   forward   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh gamma + beta
//   backward  a = dy gamma, dx = r (a - mean(a) - xh mean(a xh));  per sample dgamma_i = sum_t dy xh, dbeta_i = sum_t dy
//
// Memory bound: 2 (backward: 3) values of the storage type an element.  A row is held in the registers of a wave (rows of up to 4 chunks of 16
// bytes a lane) or of a workgroup and read once; the mean is known before deviations are squared, since sums of squares cancel
// in a stream with an offset.  Backward, a thread holds the same columns of every row it meets, so the sums over tokens of dgamma and
// dbeta stay in registers too: one workgroup goes through a chunk of a sample's tokens and leaves one partial sum
// (vector_dp.hip.h adds them up).  Rows that no register file holds are read again for every sum.
//
// 16384 x 5120 bf16: forward 64 us = 5.2 TB/s; backward 113 us = 4.5 TB/s with 16 waves a compute unit, which is what 111 registers leave.  8168 x 768
// fp16, 8 samples: 7.8 and 12.4 us, two rounds of rows a workgroup (the next round's loads ahead of a row's sums: 2 us more).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vector_io.hip.h"

namespace flashdp {

struct NormArgs {
  const void* X;          // [rows][d]
  const void* gamma;      // [d]
  const void* beta;       // [d] or null
  void* Y;
  float* mean;            // [rows] or null
  float* rstd;
  int64_t rows, d;
  float eps;
};

struct NormGradArgs {
  const void* X;          // [B][T][d]
  const void* dY;
  const void* gamma;
  const float* mean;      // [B * T]
  const float* rstd;
  void* dX;               // may be null, may be dY
  float* partial;         // [B][chunks][2 d] (d without a bias); may be null
  double* squares;        // of the held rows' kernel, where chunks == 1: [B][waves of a sample] sums of squares
  int64_t B, T, d;
  int chunks, rows_per_chunk;
  int bias;
};

// Sums of NV values over 256 threads, the same bits in each; several such groups of a workgroup meet at the same barrier.  lds: 4 * NV floats of
// the group that no thread still reads (two buffers in turn need one barrier per sum).
template <int NV>
__device__ __forceinline__ void group_sum(float (&v)[NV], float* lds) {
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) & 3;
#pragma unroll
  for (int k = 0; k < NV; ++k) v[k] = wave_sum(v[k]);
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < NV; ++k) lds[k * 4 + wave] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NV; ++k) v[k] = (lds[k * 4] + lds[k * 4 + 1]) + (lds[k * 4 + 2] + lds[k * 4 + 3]);
}

// NT threads (64 or 256) share a row, CH chunks each.  EVEN: d is whole chunks.
template <int DT, int NT, int CH, bool EVEN>
__global__ __launch_bounds__(256) void layernorm_forward_kernel(const NormArgs a) {
  constexpr int N = Chunk<DT>::N;
  __shared__ float lds[2][4];
  const int t = threadIdx.x % NT;
  const int64_t row = (int64_t)blockIdx.x * (256 / NT) + __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  if (row >= a.rows) return;     // NT = 64: a whole wave, and there are no barriers; NT = 256: never
  const char* x = (const char*)a.X + row * a.d * Chunk<DT>::BYTES;
  u32x4_t raw[CH];
  float s[1] = {0.0f};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = (int64_t)(c * NT + t) * N;
    raw[c] = load_chunk<DT, EVEN>(x, col, a.d - col);
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float f[N];
    widen_chunk<DT>(raw[c], f);
#pragma unroll
    for (int k = 0; k < N; ++k) s[0] += f[k];
  }
  if constexpr (NT == 64) s[0] = wave_sum(s[0]); else group_sum(s, lds[0]);
  const float mu = s[0] / (float)a.d;
  s[0] = 0.0f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t left = a.d - (int64_t)(c * NT + t) * N;
    float f[N];
    widen_chunk<DT>(raw[c], f);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float v = k < left ? f[k] - mu : 0.0f;     // (EVEN: all or none of a chunk)
      s[0] = fmaf(v, v, s[0]);
    }
  }
  if constexpr (NT == 64) s[0] = wave_sum(s[0]); else group_sum(s, lds[1]);
  const float r = 1.0f / sqrtf(s[0] / (float)a.d + a.eps);
  char* y = (char*)a.Y + row * a.d * Chunk<DT>::BYTES;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = (int64_t)(c * NT + t) * N, left = a.d - col;
    if (left > 0) {
      float f[N], w[N], b[N];
      widen_chunk<DT>(raw[c], f);
      widen_chunk<DT>(load_chunk<DT, EVEN>(a.gamma, col, left), w);
      widen_chunk<DT>(a.beta ? load_chunk<DT, EVEN>(a.beta, col, left) : u32x4_t{0u, 0u, 0u, 0u}, b);
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] = fmaf((f[k] - mu) * r, w[k], b[k]);
      store_chunk<DT, EVEN>(y, col, left, round_chunk<DT>(f));
    }
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
}

// Rows longer than the registers of a workgroup hold: one workgroup per row, read three times.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_forward_long_kernel(const NormArgs a) {
  constexpr int N = Chunk<DT>::N;
  __shared__ float lds[2][4];
  const int64_t row = blockIdx.x;
  const char* x = (const char*)a.X + row * a.d * Chunk<DT>::BYTES;
  float s[1] = {0.0f}, f[N];
  for (int64_t col = (int64_t)threadIdx.x * N; col < a.d; col += 256 * N) {
    widen_chunk<DT>(load_chunk<DT>(x, col, a.d - col), f);
#pragma unroll
    for (int k = 0; k < N; ++k) s[0] += f[k];
  }
  group_sum(s, lds[0]);
  const float mu = s[0] / (float)a.d;
  s[0] = 0.0f;
  for (int64_t col = (int64_t)threadIdx.x * N; col < a.d; col += 256 * N) {
    widen_chunk<DT>(load_chunk<DT>(x, col, a.d - col), f);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float v = k < a.d - col ? f[k] - mu : 0.0f;
      s[0] = fmaf(v, v, s[0]);
    }
  }
  group_sum(s, lds[1]);
  const float r = 1.0f / sqrtf(s[0] / (float)a.d + a.eps);
  char* y = (char*)a.Y + row * a.d * Chunk<DT>::BYTES;
  for (int64_t col = (int64_t)threadIdx.x * N; col < a.d; col += 256 * N) {
    float w[N], b[N];
    widen_chunk<DT>(load_chunk<DT>(x, col, a.d - col), f);
    widen_chunk<DT>(load_chunk<DT>(a.gamma, col, a.d - col), w);
    widen_chunk<DT>(a.beta ? load_chunk<DT>(a.beta, col, a.d - col) : u32x4_t{0u, 0u, 0u, 0u}, b);
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = fmaf((f[k] - mu) * r, w[k], b[k]);
    store_chunk<DT>(y, col, a.d - col, round_chunk<DT>(f));
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
}

template <bool EVEN = false>
__device__ __forceinline__ void store_sums4(float* to, int64_t col, int64_t left, const float* s) {
  store_chunk<DT_F32, EVEN>(to, col, left, u32x4_t{__builtin_bit_cast(uint32_t, s[0]), __builtin_bit_cast(uint32_t, s[1]),
                                             __builtin_bit_cast(uint32_t, s[2]), __builtin_bit_cast(uint32_t, s[3])});
}

// NT threads share a row, CH chunks each, THREADS / NT rows side by side.  One workgroup per (sample, chunk of tokens), or with TOKEN
// (T == 1, a row is a sample) one sample per row of threads, whose sums are the sample's gradient.
template <int DT, int NT, int CH, int THREADS, bool TOKEN, bool EVEN>
__global__ __launch_bounds__(THREADS) void layernorm_grad_kernel(const NormGradArgs a) {
  constexpr int N = Chunk<DT>::N, ROWS = THREADS / NT, PITCH = THREADS + 8;
  constexpr int JOIN = TOKEN || ROWS == 1 ? 0 : N * PITCH, SUMS = NT == 64 ? 0 : 2 * ROWS * 8;
  __shared__ float lds[JOIN > SUMS ? JOIN : SUMS > 0 ? SUMS : 1];
  const int t = threadIdx.x % NT, g = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);   // (whole waves share a row)
  int64_t first, last;
  if constexpr (TOKEN) {
    first = (int64_t)blockIdx.x * ROWS;
    last = first + ROWS < a.B ? first + ROWS : a.B;
  } else {
    const int64_t i = blockIdx.x / a.chunks, k0 = blockIdx.x - i * a.chunks;
    first = i * a.T + k0 * a.rows_per_chunk;
    last = (k0 + 1) * a.rows_per_chunk < a.T ? first + a.rows_per_chunk : (i + 1) * a.T;
  }
  const float per_d = 1.0f / (float)a.d;
  const int64_t pitch = a.d * Chunk<DT>::BYTES;
  u32x4_t w[CH];
  float sg[CH][N], sb[CH][N];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = (int64_t)(c * NT + t) * N;
    w[c] = load_chunk<DT, EVEN>(a.gamma, col, a.d - col);
#pragma unroll
    for (int k = 0; k < N; ++k) sg[c][k] = sb[c][k] = 0.0f;
  }
  int turn = 0;
  for (int64_t row0 = first; row0 < last; row0 += ROWS) {     // the same number of times for all rows of threads: they meet at barriers
    const int64_t row = row0 + g;      // (scalar, so that addresses cost no vector registers)
    const bool in = row < last;
    const char* x = (const char*)a.X + row * pitch;
    const char* dy = (const char*)a.dY + row * pitch;
    u32x4_t xr[CH], gr[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t col = (int64_t)(c * NT + t) * N, left = in ? a.d - col : 0;
      xr[c] = load_chunk<DT, EVEN>(x, col, left);
      gr[c] = load_chunk<DT, EVEN>(dy, col, left);
    }
    const float mu = in ? a.mean[row] : 0.0f, r = in ? a.rstd[row] : 0.0f;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float f[N], e[N], v[N];
      widen_chunk<DT>(xr[c], f);
      widen_chunk<DT>(gr[c], e);
      widen_chunk<DT>(w[c], v);
      // (columns and rows that do not exist have dy = 0, and need xh = 0 as well: the mean alone times rstd may be infinite)
      const int64_t left = a.d - (int64_t)(c * NT + t) * N;
      const float here = EVEN && left <= 0 ? 0.0f : mu;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float xh = EVEN || k < left ? (f[k] - here) * r : 0.0f, p = e[k] * v[k];
        s[0] += p;
        s[1] = fmaf(p, xh, s[1]);
        sg[c][k] = fmaf(e[k], xh, sg[c][k]);
        sb[c][k] += e[k];
      }
      // (added up here: left to the compiler, the sums over tokens wait behind the barrier, with the widened row in registers)
#pragma unroll
      for (int k = 0; k < N; ++k) asm volatile("" : "+v"(sg[c][k]), "+v"(sb[c][k]));
    }
    if constexpr (NT == 64) { s[0] = wave_sum(s[0]); s[1] = wave_sum(s[1]); }
    else { group_sum(s, lds + (turn * ROWS + g) * 8); turn ^= 1; }
    // (kept as they were loaded, and widened again: the widened row beside the sums would not fit the registers)
#pragma unroll
    for (int c = 0; c < CH; ++c) asm volatile("" : "+v"(xr[c]), "+v"(gr[c]), "+v"(w[c]));
    if (a.dX && in) {
      const float m0 = s[0] * per_d, m1 = s[1] * per_d;
      char* dx = (char*)a.dX + row * pitch;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int64_t col = (int64_t)(c * NT + t) * N, left = a.d - col;
        if (left > 0) {
          float f[N], e[N], v[N];
          widen_chunk<DT>(xr[c], f);
          widen_chunk<DT>(gr[c], e);
          widen_chunk<DT>(w[c], v);
#pragma unroll
          for (int k = 0; k < N; ++k) f[k] = r * (fmaf(e[k], v[k], -m0) - (f[k] - mu) * r * m1);
          store_chunk<DT, EVEN>(dx, col, left, round_chunk<DT>(f));
        }
      }
    }
  }
  if (!a.partial) return;
  if constexpr (TOKEN || ROWS == 1) {
    if (TOKEN && first + g >= last) return;
    float* to = a.partial + (TOKEN ? first + g : (int64_t)blockIdx.x) * a.d * (a.bias ? 2 : 1);
    double square = 0.0;      // (columns that do not exist have sums of zero)
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int k = 0; k < N; ++k) square += (double)sg[c][k] * (double)sg[c][k] + (a.bias ? (double)sb[c][k] * (double)sb[c][k] : 0.0);
      const int64_t col = (int64_t)(c * NT + t) * N, left = a.d - col;
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        store_sums4<EVEN>(to, col + q, left - q, sg[c] + q);
        if (a.bias) store_sums4<EVEN>(to + a.d, col + q, left - q, sb[c] + q);
      }
    }
    if (TOKEN || a.chunks == 1) {
      square = wave_sum(square);
      if ((t & 63) == 0) a.squares[(TOKEN ? first + g : (int64_t)blockIdx.x) * (NT / 64) + t / 64] = square;
    }
  } else {
    // the rows of threads join their sums, NT * N columns of one of the two vectors at a time
    float* to = a.partial + (int64_t)blockIdx.x * a.d * (a.bias ? 2 : 1);
    double square = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        if (part == 1 && !a.bias) break;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) lds[k * PITCH + threadIdx.x] = part ? sb[c][k] : sg[c][k];
        __syncthreads();
        for (int e = threadIdx.x; e < NT * N; e += THREADS) {
          const int64_t col = (int64_t)c * NT * N + e;
          if (col >= a.d) break;
          float s = 0.0f;
#pragma unroll
          for (int q = 0; q < ROWS; ++q) s += lds[(e % N) * PITCH + q * NT + e / N];
          to[part * a.d + col] = s;
          square += (double)s * (double)s;
        }
      }
    }
    if (a.chunks == 1) {
      square = wave_sum(square);
      if ((threadIdx.x & 63) == 0) a.squares[(int64_t)blockIdx.x * (THREADS / 64) + threadIdx.x / 64] = square;
    }
  }
}

// Rows longer than the registers of a workgroup hold.  First the sums over tokens, a thread per chunk of columns down the tokens of its
// workgroup's chunk ...
template <int DT>
__global__ __launch_bounds__(256) void layernorm_grad_long_sums_kernel(const NormGradArgs a, int col_tiles) {
  constexpr int N = Chunk<DT>::N;
  const int64_t unit = blockIdx.x / col_tiles;
  const int64_t col = ((int64_t)(blockIdx.x - unit * col_tiles) * 256 + threadIdx.x) * N, left = a.d - col;
  if (left <= 0) return;
  const int64_t i = unit / a.chunks, k0 = unit - i * a.chunks;
  const int64_t first = i * a.T + k0 * a.rows_per_chunk;
  const int64_t last = (k0 + 1) * a.rows_per_chunk < a.T ? first + a.rows_per_chunk : (i + 1) * a.T;
  float sg[N], sb[N], f[N], g[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sg[k] = sb[k] = 0.0f;
#pragma unroll 2
  for (int64_t row = first; row < last; ++row) {
    widen_chunk<DT>(load_chunk<DT>((const char*)a.X + row * a.d * Chunk<DT>::BYTES, col, left), f);
    widen_chunk<DT>(load_chunk<DT>((const char*)a.dY + row * a.d * Chunk<DT>::BYTES, col, left), g);
    const float mu = a.mean[row], r = a.rstd[row];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      sg[k] = fmaf(g[k], (f[k] - mu) * r, sg[k]);
      sb[k] += g[k];
    }
  }
  float* to = a.partial + unit * a.d * (a.bias ? 2 : 1);
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    store_sums4(to, col + 4 * q, left - 4 * q, sg + 4 * q);
    if (a.bias) store_sums4(to + a.d, col + 4 * q, left - 4 * q, sb + 4 * q);
  }
}

// ... then dX (which may be dY, so not before the sums), one workgroup per row, read twice.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_grad_long_rows_kernel(const NormGradArgs a) {
  constexpr int N = Chunk<DT>::N;
  __shared__ float lds[8];
  const int64_t row = blockIdx.x;
  const char* x = (const char*)a.X + row * a.d * Chunk<DT>::BYTES;
  const char* dy = (const char*)a.dY + row * a.d * Chunk<DT>::BYTES;
  const float mu = a.mean[row], r = a.rstd[row], per_d = 1.0f / (float)a.d;
  float s[2] = {0.0f, 0.0f}, f[N], g[N], v[N];
  for (int64_t col = (int64_t)threadIdx.x * N; col < a.d; col += 256 * N) {
    widen_chunk<DT>(load_chunk<DT>(x, col, a.d - col), f);
    widen_chunk<DT>(load_chunk<DT>(dy, col, a.d - col), g);
    widen_chunk<DT>(load_chunk<DT>(a.gamma, col, a.d - col), v);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float p = g[k] * v[k];
      s[0] += p;
      s[1] = fmaf(p, k < a.d - col ? (f[k] - mu) * r : 0.0f, s[1]);
    }
  }
  group_sum(s, lds);
  const float m0 = s[0] * per_d, m1 = s[1] * per_d;
  char* dx = (char*)a.dX + row * a.d * Chunk<DT>::BYTES;
  for (int64_t col = (int64_t)threadIdx.x * N; col < a.d; col += 256 * N) {
    widen_chunk<DT>(load_chunk<DT>(x, col, a.d - col), f);
    widen_chunk<DT>(load_chunk<DT>(dy, col, a.d - col), g);
    widen_chunk<DT>(load_chunk<DT>(a.gamma, col, a.d - col), v);
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = r * (fmaf(g[k], v[k], -m0) - (f[k] - mu) * r * m1);
    store_chunk<DT>(dx, col, a.d - col, round_chunk<DT>(f));
  }
}

}  // namespace flashdp
