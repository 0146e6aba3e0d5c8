// Per-layer DP gradients of vectors of parameters (a bias; weight and bias of a normalisation): the steps of Algorithm 1 after
// the sum over tokens, for parameter vectors of n elements,
//     g_i = sum over token chunks of partial[i][k][n]      n_i = |g_i|      out = sum_i g_i / max(1, n_i / C) + sigma C z.
//
// The kernels that go over the tokens leave one partial sum per chunk of tokens; their order is fixed, nothing is added
// atomically, so results repeat to the bit.  Squares are added up in fp64 (an element of 1e20 does not overflow its norm).
// Bound by launches and latency: B (chunks + 1) n floats, a few MB at most next to the activations that were read before.  8 samples of 3072
// in 32 chunks: 4.6 us for the sums, 4.4 for the rest, some 2 of each the launch; where the kernel before has all of a sample's
// tokens in one workgroup it leaves the squares as well and the first of the two falls away (256 samples of 512: 11.0 us in all, 9.5 so).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "clip_factor.hip.h"
#include "philox_gauss.h"
#include "vector_io.hip.h"

namespace flashdp {

struct VectorArgs {
  const float* partial;   // [B][chunks][n]
  float* g;               // [B][n]; partial itself where chunks == 1
  double* squares;        // [B][blocks] sums of squares: of 64 elements each, or from the kernel before where chunks == 1
  float* factors;         // [B] clip factors, where they come from a launch of their own
  int64_t n, B;
  int chunks, blocks;
  float C, noise_scale;
  uint64_t seed;
  uint32_t layer, field;
  float* out;             // [n]
  float* out_norms;       // [B] or null
  int accumulate;
};

// One workgroup per 64 elements of one sample's vector (blocks = ceil(n / 64)), its four waves taking every fourth chunk.
__global__ __launch_bounds__(256) void vector_sum_kernel(const VectorArgs a) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = blockIdx.x / a.blocks;
  const int64_t col = (int64_t)(blockIdx.x - i * a.blocks) * 64 + lane;
  float s = 0.0f;
  if (col < a.n) {
    const float* p = a.partial + i * a.chunks * a.n + col;
#pragma unroll 8
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

// The norm of sample i by `lanes` (a power of two) neighbouring lanes, of which this one is number `lane`; the same in all of them.
__device__ __forceinline__ double vector_norm(const VectorArgs& a, int64_t i, int lane, int lanes) {
  const double* q = a.squares + i * a.blocks;
  double s = 0.0;
#pragma unroll 4
  for (int k = lane; k < a.blocks; k += lanes) s += q[k];
  for (int off = lanes >> 1; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  return sqrt(s);
}

// Clip factors in a launch of their own, one wave per sample.
__global__ __launch_bounds__(256) void vector_factors_kernel(const VectorArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= a.B) return;
  const double n = vector_norm(a, i, lane, 64);
  if (lane == 0) {
    a.factors[i] = clip_factor_of(n, a.C);
    if (a.out_norms) a.out_norms[i] = (float)n;
  }
}

// out for COLS elements per workgroup: COLS threads of it side by side, the samples dealt to 256 / COLS rows of threads and their sums
// joined in a fixed order.  COLS = 64, for at most 16 samples: a thread adds up four.  COLS = 16:
// up to 2^16, one after the other, and so in fp64 (in fp32, 2^14 equal ones lost eleven bits).  FOLD: every workgroup works the clip factors out for itself, all samples at a time (256 / B lanes each;
// a wave for one sample after the other takes a microsecond each: 256 samples of 512 elements 40 us, 3 so).
constexpr int VECTOR_FOLD_B = 1024;             // factors kept in LDS
constexpr int64_t VECTOR_FOLD_SQUARES = 8192;   // B * blocks doubles that every workgroup reads: 64 KB from the caches
__device__ __forceinline__ float fma_of(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double fma_of(double a, double b, double c) { return fma(a, b, c); }
template <bool FOLD, int COLS>
__global__ __launch_bounds__(256) void vector_clip_kernel(const VectorArgs a) {
  constexpr int ROWS = 256 / COLS, EARLY = 4;
  using Sum = std::conditional_t<COLS == 64, float, double>;
  __shared__ float fac[FOLD ? VECTOR_FOLD_B : 1];
  __shared__ Sum part[ROWS][COLS];
  const int c = threadIdx.x % COLS, r = threadIdx.x / COLS;
  const int64_t col = (int64_t)blockIdx.x * COLS + c;
  // what does not depend on the factors goes first: the first samples' elements, the old output, the noise
  float early[EARLY], old = 0.0f, noise = 0.0f;
#pragma unroll
  for (int k = 0; k < EARLY; ++k) early[k] = col < a.n && r + k * ROWS < a.B ? a.g[(int64_t)(r + k * ROWS) * a.n + col] : 0.0f;
  if (r == 0 && col < a.n) {
    if (a.accumulate) old = a.out[col];
    if (a.noise_scale != 0.0f) {
      const Normals4 z = noise_group(a.seed, a.layer, (uint64_t)(col >> 2), a.field);
      const int e = (int)(col & 3);
      noise = e == 0 ? z.z[0] : e == 1 ? z.z[1] : e == 2 ? z.z[2] : z.z[3];
    }
  }
  if constexpr (FOLD) {
    int lanes = 64;
    while (lanes > 1 && lanes * a.B > 256) lanes >>= 1;
    const int lane = threadIdx.x & (lanes - 1);
    for (int64_t i0 = 0; i0 < a.B; i0 += 256 / lanes) {      // (whole waves take part in the sums of lanes)
      const int64_t i = i0 + threadIdx.x / lanes;
      const double n = vector_norm(a, i < a.B ? i : a.B - 1, lane, lanes);
      if (lane == 0 && i < a.B) {
        fac[i] = clip_factor_of(n, a.C);
        if (blockIdx.x == 0 && a.out_norms) a.out_norms[i] = (float)n;
      }
    }
    __syncthreads();
  }
  Sum s = 0;
  if (col < a.n) {
#pragma unroll
    for (int k = 0; k < EARLY; ++k)
      if (r + k * ROWS < a.B) s = fma_of((Sum)(FOLD ? fac[r + k * ROWS] : a.factors[r + k * ROWS]), (Sum)early[k], s);
#pragma unroll 8
    for (int64_t i = r + EARLY * ROWS; i < a.B; i += ROWS) s = fma_of((Sum)(FOLD ? fac[i] : a.factors[i]), (Sum)a.g[i * a.n + col], s);
  }
  part[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= a.n) return;
  s = 0;
#pragma unroll
  for (int k = 0; k < ROWS; ++k) s += part[k][c];
  if (a.accumulate) s += (Sum)old;
  if (a.noise_scale != 0.0f) s = fma_of((Sum)a.noise_scale, (Sum)noise, s);
  a.out[col] = (float)s;
}

}  // namespace flashdp
