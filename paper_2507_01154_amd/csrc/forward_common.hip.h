// What the kernels of the forward product share: Y = act(Z) + R, Z = X W^T + bias, for X [rows][K], W [D][K].
//
// Both operands have the reduction index contiguous, which is what the matrix cores want: a lane of v_mfma_f32_16x16x32
// holds eight consecutive k (16 bytes) of one row, lane l of row l % 16 and k = 8 (l / 16) + 0..7.  The fp32 instruction
// 16x16x4 holds one k per lane, k = l / 16; four of them take a lane's 16 bytes element by element, which pairs k = 4 (l / 16) + s of
// both operands in step s.  So all kernels see rows of bytes: a k-step is 64 bytes of every row, whatever the type.
//
// W is the first operand and X the second: register r of lane l is then feature 4 (l / 16) + r of token l % 16, four
// consecutive features that leave in one store, and a block of 32 features that shares an 8-bit exponent is two registers' worth in the
// four lanes l, l + 16, l + 32, l + 48.
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

__device__ __forceinline__ float act_of(int act, float z) {
  switch (act) {
    case ACT_RELU: return act_value<ACT_RELU>(z);
    case ACT_GELU: return act_value<ACT_GELU>(z);
    case ACT_GELU_TANH: return act_value<ACT_GELU_TANH>(z);
    case ACT_SILU: return act_value<ACT_SILU>(z);
    default: return z;
  }
}

// Four consecutive elements from index `at` on (any alignment), `left` of which exist.
typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(2)));
template <int DT>
__device__ __forceinline__ void load4(const void* p, int64_t at, int left, float (&f)[4]) {
  if constexpr (DT == DT_F32) {
    const u32x4_t v = load_chunk<DT_F32>(p, at, left);
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = as_float(v[k]);
  } else {
    uint32_t v[2] = {0u, 0u};
    if (left >= 4) {
      const u32x2_any_t q = *(const u32x2_any_t*)((const unsigned short*)p + at);
      v[0] = q[0]; v[1] = q[1];
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (k < left) v[k >> 1] |= (uint32_t)((const unsigned short*)p)[at + k] << (16 * (k & 1));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t h = (v[k >> 1] >> (16 * (k & 1))) & 0xFFFFu;
      f[k] = DT == DT_BF16 ? __builtin_bit_cast(float, h << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)h);
    }
  }
}
template <int DT>
__device__ __forceinline__ void store4(void* p, int64_t at, int left, const float (&f)[4]) {
  if constexpr (DT == DT_F32) {
    store_chunk<DT_F32>(p, at, left, u32x4_t{__builtin_bit_cast(uint32_t, f[0]), __builtin_bit_cast(uint32_t, f[1]),
                                             __builtin_bit_cast(uint32_t, f[2]), __builtin_bit_cast(uint32_t, f[3])});
  } else {
    const u32x2_any_t q = {pack2_16bit<DT>(f[0], f[1]), pack2_16bit<DT>(f[2], f[3])};
    if (left >= 4) {
      *(u32x2_any_t*)((unsigned short*)p + at) = q;
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (k < left) ((unsigned short*)p)[at + k] = (unsigned short)(q[k >> 1] >> (16 * (k & 1)));
    }
  }
}

// The 8-bit form of a block of 32 features of token m that the lanes l, l + 16, l + 32, l + 48 hold: z[0] are features n .. n + 3 and
// z[1] n + 16 .. n + 19, n = the block's first + 4 (lane / 16).  ok: the token exists (all lanes take part all the same).
template <int DT>
__device__ __forceinline__ void keep_block8(const ForwardArgs& a, int64_t m, int n, bool ok, const float (&z)[2][4]) {
  float top = 0.0f;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, finite_f32(z[h][k]) && n + 16 * h + k < a.D ? fabsf(z[h][k]) : 0.0f);
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  if (!ok) return;
  const int e = checkpoint8_exponent<DT>(top);
  const float inv = power_of_two(-e);
  signed char* row = (signed char*)a.Z + m * a.D;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = n + 16 * h;
    uint32_t q = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) q |= checkpoint8_quantise(z[h][k], inv) << (8 * k);
    if (a.D - col >= 4) {
      *(u32_any_t*)(row + col) = q;
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (col + k < a.D) row[col + k] = (signed char)(q >> (8 * k));
    }
  }
  if ((threadIdx.x & 63) < 16 && n < a.D) a.scales[m * checkpoint8_blocks(a.D) + n / CKPT8_BLOCK] = (unsigned char)(e + 127);
}

// What happens to finished sums: acc[i][j] is the 16 x 16 block of tokens m0 + 16 i .. and features n0 + 16 j .. of this wave
// (n0 a multiple of 32).  Straight from the registers to memory.
template <int DT, int FM, int FN>
__device__ __forceinline__ void forward_epilogue(const ForwardArgs& a, f32x4v_t (&acc)[FM][FN], int64_t m0, int n0) {
  static_assert(FN % 2 == 0, "blocks of 32 features");
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < FN; j += 2) {
    const int n = n0 + 16 * j + 4 * (lane >> 4);
    float b[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int k = 0; k < 4; ++k) b[h][k] = 0.0f;
      if (a.bias) load4<DT>(a.bias, n + 16 * h, a.D - n - 16 * h, b[h]);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t m = m0 + 16 * i + (lane & 15);
      const bool ok = m < a.rows;
      float z[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) z[h][k] = acc[i][j + h][k] + b[h][k];
      if (a.keep == KEEP_EIGHT) keep_block8<DT>(a, m, n, ok, z);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int col = n + 16 * h, left = a.D - col;
        if (!ok || left <= 0) continue;
        if (a.keep == KEEP_SAME) store4<DT>(a.Z, m * a.D + col, left, z[h]);
        float y[4], r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (a.residual) load4<DT>(a.residual, m * a.D + col, left, r);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = act_of(a.act, z[h][k]) + r[k];
        store4<DT>(a.Y, m * a.D + col, left, y);
      }
    }
  }
}

}  // namespace flashdp
