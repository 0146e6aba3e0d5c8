// The activations of the linear layers' epilogue and their slopes, in fp32.
//
// All but ReLU are z times a smooth step, and each is written so that the step keeps its relative accuracy where it is small
// (for z << 0), without a cancelling 1 + tanh or 1 + erf:
//   GELU (tanh form)  z s(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3), since (1 + tanh u) / 2 is the logistic function s of 2 u
//   SiLU              z s(z)
//   GELU              z erfc(-z / sqrt(2)) / 2
// s(v) = 1 / (1 + e^-v): for v << 0 the exponential overflows to infinity and s is 0.  All of them have reached their limits
// in fp32 at |z| = 128, where the factors beside the step are cut off, so that infinities give the limit and not 0 times infinity; the step
// itself is taken of z as it is, so NaN stays NaN though minima and maxima drop it.
#pragma once
#include <hip/hip_runtime.h>

namespace flashdp {

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

// 1 / (1 + 2^u): s(v) for u = -v log2(e), a factor that folds into what v is made of
__device__ __forceinline__ float logistic_of_exp2(float u) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u)); }
constexpr float LOG2_E = 1.44269504f;
constexpr float GELU_1 = 1.59576912f, GELU_3 = 1.59576912f * 0.044715f;      // 2 u = GELU_1 z + GELU_3 z^3

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == ACT_NONE) return z;
  if constexpr (ACT == ACT_RELU) return z <= 0.0f ? 0.0f : z;     // (a comparison with NaN is false)
  const float c = fmaxf(z, -128.0f);
  if constexpr (ACT == ACT_GELU) return 0.5f * c * erfcf(-0.70710678f * z);
  if constexpr (ACT == ACT_GELU_TANH) return c * logistic_of_exp2(z * fmaf(z * z, -LOG2_E * GELU_3, -LOG2_E * GELU_1));
  if constexpr (ACT == ACT_SILU) return c * logistic_of_exp2(-LOG2_E * z);
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == ACT_NONE) return 1.0f;
  if constexpr (ACT == ACT_RELU) return z <= 0.0f ? 0.0f : z > 0.0f ? 1.0f : z;
  const float c = __builtin_amdgcn_fmed3f(z, -128.0f, 128.0f);
  if constexpr (ACT == ACT_GELU) return fmaf(0.39894228f * c, __expf(-0.5f * c * c), 0.5f * erfcf(-0.70710678f * z));
  if constexpr (ACT == ACT_GELU_TANH) {
    const float cc = c * c, s = logistic_of_exp2(z * fmaf(cc, -LOG2_E * GELU_3, -LOG2_E * GELU_1));
    return fmaf(c * fmaf(cc, 3.0f * GELU_3, GELU_1) * (1.0f - s), s, s);   // s + z s (1 - s) d(2 u)/dz
  }
  if constexpr (ACT == ACT_SILU) {
    const float s = logistic_of_exp2(-LOG2_E * z);
    return fmaf(c * (1.0f - s), s, s);
  }
}

}  // namespace flashdp
