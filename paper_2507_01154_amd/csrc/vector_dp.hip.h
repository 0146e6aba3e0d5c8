// Per-layer DP gradients of vectors of parameters (a bias; weight and bias of a normalisation): the steps of Algorithm 1 after
// the sum over tokens, for parameter vectors of n elements,
//     g_i = sum over token chunks of partial[i][k][n]      n_i = |g_i|      out = sum_i g_i / max(1, n_i / C) + sigma C z.
//
// The kernels that go over the tokens leave one partial sum per chunk of tokens; their order is fixed, nothing is added
// atomically, so results repeat to the bit.  Squares are added up in fp64 (an element of 1e20 does not overflow its norm).
// Bound by launches and latency: B (chunks + 1) n floats, a few MB at most next to the activations that were read before.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clip_factor.hip.h"
#include "philox_gauss.h"
#include "vector_io.hip.h"

namespace flashdp {

struct VectorArgs {
  const float* partial;   // [B][chunks][n]
  float* g;               // [B][n]; partial itself where chunks == 1
  double* squares;        // [B][blocks] sums of squares of 64 elements each
  float* factors;         // [B] clip factors, where they come from a launch of their own
  int64_t n, B;
  int chunks, blocks;     // blocks = ceil(n / 64)
  float C, noise_scale;
  uint64_t seed;
  uint32_t layer, field;
  float* out;             // [n]
  float* out_norms;       // [B] or null
  int accumulate;
};

// One workgroup per 64 elements of one sample's vector, its four waves taking every fourth chunk.
__global__ __launch_bounds__(256) void vector_sum_kernel(const VectorArgs a) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = blockIdx.x / a.blocks;
  const int64_t col = (int64_t)(blockIdx.x - i * a.blocks) * 64 + lane;
  float s = 0.0f;
  if (col < a.n) {
    const float* p = a.partial + i * a.chunks * a.n + col;
#pragma unroll 4
    for (int k = wave; k < a.chunks; k += 4) s += p[(int64_t)k * a.n];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0) return;
  s = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
  if (col < a.n && a.chunks > 1) a.g[i * a.n + col] = s;
  const double q = wave_sum((double)s * (double)s);
  if (lane == 0) a.squares[blockIdx.x] = q;
}

__device__ __forceinline__ double vector_norm(const double* __restrict__ squares_i, int blocks, int lane) {
  double s = 0.0;
#pragma unroll 4
  for (int k = lane; k < blocks; k += 64) s += squares_i[k];
  return sqrt(wave_sum(s));
}

// Clip factors in a launch of their own, one wave per sample.
__global__ __launch_bounds__(256) void vector_factors_kernel(const VectorArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= a.B) return;
  const double n = vector_norm(a.squares + i * a.blocks, a.blocks, lane);
  if (lane == 0) {
    a.factors[i] = clip_factor_of(n, a.C);
    if (a.out_norms) a.out_norms[i] = (float)n;
  }
}

// out for 16 elements per workgroup: 16 threads of it side by side, the samples dealt to 16 rows of threads and their sums
// joined in a fixed order.  FOLD: every workgroup works the clip factors out for itself.
constexpr int VECTOR_FOLD_B = 1024;             // factors kept in LDS
constexpr int64_t VECTOR_FOLD_SQUARES = 8192;   // B * blocks doubles that every workgroup reads: 64 KB from the caches
template <bool FOLD>
__global__ __launch_bounds__(256) void vector_clip_kernel(const VectorArgs a) {
  __shared__ float fac[FOLD ? VECTOR_FOLD_B : 1];
  __shared__ float part[16][16];
  if constexpr (FOLD) {
    const int lane = threadIdx.x & 63;
    for (int64_t i = threadIdx.x >> 6; i < a.B; i += 4) {
      const double n = vector_norm(a.squares + i * a.blocks, a.blocks, lane);
      if (lane == 0) {
        fac[i] = clip_factor_of(n, a.C);
        if (blockIdx.x == 0 && a.out_norms) a.out_norms[i] = (float)n;
      }
    }
    __syncthreads();
  }
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t col = (int64_t)blockIdx.x * 16 + c;
  float s = 0.0f;
  if (col < a.n) {
#pragma unroll 4
    for (int64_t i = r; i < a.B; i += 16) s = fmaf(FOLD ? fac[i] : a.factors[i], a.g[i * a.n + col], s);
  }
  part[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= a.n) return;
  s = 0.0f;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += part[k][c];
  if (a.accumulate) s += a.out[col];
  if (a.noise_scale != 0.0f) {
    const Normals4 z = noise_group(a.seed, a.layer, (uint64_t)(col >> 2), a.field);
    const int e = (int)(col & 3);
    s = fmaf(a.noise_scale, e == 0 ? z.z[0] : e == 1 ? z.z[1] : e == 2 ? z.z[2] : z.z[3], s);
  }
  a.out[col] = s;
}

}  // namespace flashdp
