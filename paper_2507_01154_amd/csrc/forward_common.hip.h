// What the kernels of the forward product share: Y = act(Z) + R, Z = X W^T + bias, for X [rows][K], W [D][K].
//
// Both operands have the reduction index contiguous, which is what the matrix cores want: a lane of v_mfma_f32_16x16x32
// holds eight consecutive k (16 bytes) of one row, lane l of row l % 16 and k = 8 (l / 16) + 0..7.  The fp32 instruction
// 16x16x4 holds one k per lane, k = l / 16; four of them take a lane's 16 bytes element by element, which pairs k = 4 (l / 16) + s of
// both operands in step s.  So all kernels see rows of bytes: a k-step is 64 bytes of every row, whatever the type.
//
// W is the first operand and X the second: register r of lane l is then feature 4 (l / 16) + r of token l % 16, four
// consecutive features of one token.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "activations.hip.h"
#include "checkpoint8.hip.h"
#include "gemm_mfma.hip.h"
#include "vector_io.hip.h"

namespace flashdp {

enum : int { KEEP_NONE = 0, KEEP_SAME = 1, KEEP_EIGHT = 2 };   // Z

struct ForwardArgs {
  const void* X;           // [rows][K]
  const void* W;           // [D][K]
  const void* bias;        // [D] or null
  const void* residual;    // [rows][D] or null; may be Y
  void* Y;                 // [rows][D]
  void* Z;                 // [rows][D], or the q of a checkpoint
  unsigned char* scales;   // of a checkpoint
  int64_t rows;
  int K, D;
  int act, keep;
  int tiles_m, tiles_n;    // tiles of tokens and of features
};

typedef float f32x4v_t __attribute__((ext_vector_type(4)));

// acc += W fragment x X fragment over one k-step
template <int DT>
__device__ __forceinline__ f32x4v_t k_step(const u32x4_t w, const u32x4_t x, f32x4v_t acc) {
  if constexpr (DT == DT_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), acc, 0, 0, 0);
  } else if constexpr (DT == DT_F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, w), __builtin_bit_cast(f16x8_t, x), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(as_float(w[s]), as_float(x[s]), acc, 0, 0, 0);
    return acc;
  }
}

template <int N>
__device__ __forceinline__ void act_chunk(int act, const float (&z)[N], float (&y)[N]) {
  auto each = [&](auto act_c) {
#pragma unroll
    for (int k = 0; k < N; ++k) y[k] = act_value<decltype(act_c)::value>(z[k]);
  };
  switch (act) {
    case ACT_RELU: each(std::integral_constant<int, ACT_RELU>{}); break;
    case ACT_GELU: each(std::integral_constant<int, ACT_GELU>{}); break;
    case ACT_GELU_TANH: each(std::integral_constant<int, ACT_GELU_TANH>{}); break;
    case ACT_SILU: each(std::integral_constant<int, ACT_SILU>{}); break;
    default: each(std::integral_constant<int, ACT_NONE>{}); break;
  }
}

// What becomes of a chunk of sums Z, `left` of which exist (none: the lane only takes part): element `at` of [rows][D] on, block `block` of
// the 8-bit form.  The lanes of a block of 32 features are neighbours, all of the same token.
template <int DT>
__device__ __forceinline__ void finish_chunk(const ForwardArgs& a, int64_t at, int64_t block, int left, const float (&z)[Chunk<DT>::N]) {
  constexpr int N = Chunk<DT>::N, PER = CKPT8_BLOCK / N;
  u32x4_t res = {0u, 0u, 0u, 0u};
  if (a.residual && left > 0) res = load_chunk<DT>(a.residual, at, left);
  if (a.keep == KEEP_EIGHT) {
    float there[N];
#pragma unroll
    for (int k = 0; k < N; ++k) there[k] = z[k];
    if (left < N) {
#pragma unroll
      for (int k = 0; k < N; ++k) there[k] = k < left ? z[k] : 0.0f;
    }
    const uint32_t top = checkpoint8_top<N, PER>(there);
    if (left > 0) {
      const int e = checkpoint8_keep<DT>((signed char*)a.Z + at, left, z, top);
      if ((threadIdx.x & (PER - 1)) == 0) a.scales[block] = (unsigned char)(e + 127);
    }
  }
  if (left <= 0) return;
  if (a.keep == KEEP_SAME) store_chunk<DT>(a.Z, at, left, round_chunk<DT>(z));
  float y[N];
  act_chunk<N>(a.act, z, y);
  if (a.residual) {
    float w[N];
    widen_chunk<DT>(res, w);
#pragma unroll
    for (int k = 0; k < N; ++k) y[k] += w[k];
  }
  store_chunk<DT>(a.Y, at, left, round_chunk<DT>(y));
}

// The end of kernels whose waves share out the k-steps: PARTS partial sums of M tokens x F features in LDS (rows of F + 4 floats) are joined in
// order, one chunk per thread and step.  Whole waves stay together (lanes of a block of 32 features exchange its largest magnitude).
template <int DT, int NT, int PARTS, int M, int F>
__device__ __forceinline__ void finish_partials(const ForwardArgs& a, const float* part, int64_t m0, int n0) {
  constexpr int N = Chunk<DT>::N, PITCH = F + 4, PER_ROW = F / N, CHUNKS = M * PER_ROW;
  for (int e = threadIdx.x; e < (CHUNKS + 63) / 64 * 64; e += NT) {
    const int r = CHUNKS % 64 == 0 ? e / PER_ROW : min(e / PER_ROW, M - 1), c = (e % PER_ROW) * N;
    const int64_t m = m0 + r;
    const int col = n0 + c, left = e < CHUNKS && m < a.rows ? a.D - col : 0;
    float z[N];
    widen_chunk<DT>(a.bias ? load_chunk<DT>(a.bias, col, left) : u32x4_t{0u, 0u, 0u, 0u}, z);
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      f32x4v_t sum = *(const f32x4v_t*)(part + r * PITCH + c + k);
#pragma unroll
      for (int v = 1; v < PARTS; ++v) sum += *(const f32x4v_t*)(part + (v * M + r) * PITCH + c + k);
#pragma unroll
      for (int q = 0; q < 4; ++q) z[k + q] += sum[q];
    }
    finish_chunk<DT>(a, m * a.D + col, m * checkpoint8_blocks(a.D) + col / CKPT8_BLOCK, left, z);
  }
}

// What happens to finished sums.  acc[i][j] is the 16 x 16 block of tokens m0 + 16 i .. and features n0 + 16 j .. of this wave (n0 a
// multiple of 32).  They pass through `stage`, LDS of this wave alone, 64 tokens at a time, and leave as whole rows of chunks of 16 bytes: full
// cache lines, one chunk per lane and step, so that the code of the epilogue exists once and not once per block.  Rows of the stage are
// 16 bytes longer than their values, which spreads the 16 tokens that a store of sums meets over all banks.
template <int FM, int FN>
struct ForwardStage {
  static constexpr int FEATURES = 16 * FN, BLOCKS = FM < 4 ? FM : 4, PITCH = FEATURES + 4;   // floats
  static constexpr int BYTES = 16 * BLOCKS * PITCH * 4;                                     // per wave
};

template <int DT, int FM, int FN>
__device__ __forceinline__ void forward_epilogue(const ForwardArgs& a, const f32x4v_t (&acc)[FM][FN], int64_t m0, int n0, float* stage) {
  using S = ForwardStage<FM, FN>;
  constexpr int N = Chunk<DT>::N, PER_ROW = S::FEATURES / N, ROWS = 64 / PER_ROW;
  static_assert(FM % S::BLOCKS == 0 && S::FEATURES % CKPT8_BLOCK == 0, "whole phases, whole blocks of 32 features");
  const int lane = threadIdx.x & 63;
  const int c = (lane % PER_ROW) * N, r0 = lane / PER_ROW;
  const int col = n0 + c, left = a.D - col;
  const int64_t blocks = checkpoint8_blocks(a.D);
  int64_t at = (m0 + r0) * a.D + col, block = (m0 + r0) * blocks + col / CKPT8_BLOCK;
  float b[N];
  widen_chunk<DT>(a.bias ? load_chunk<DT>(a.bias, col, left) : u32x4_t{0u, 0u, 0u, 0u}, b);
#pragma unroll
  for (int phase = 0; phase < FM / S::BLOCKS; ++phase) {
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        *(f32x4v_t*)(stage + (16 * i + (lane & 15)) * S::PITCH + 16 * j + 4 * (lane >> 4)) = acc[phase * S::BLOCKS + i][j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll 2
    for (int it = 0; it < 16 * S::BLOCKS / ROWS; ++it) {
      const int r = it * ROWS + r0;
      float z[N];
#pragma unroll
      for (int k = 0; k < N; k += 4) {
        const f32x4v_t s = *(const f32x4v_t*)(stage + r * S::PITCH + c + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[k + e] = s[e] + b[k + e];
      }
      finish_chunk<DT>(a, at, block, m0 + 16 * S::BLOCKS * phase + r < a.rows ? left : 0, z);
      at += (int64_t)ROWS * a.D;
      block += ROWS * blocks;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace flashdp
