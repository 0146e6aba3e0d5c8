// Rows of any length in 16-byte pieces: a row of n elements is cut into chunks of 16 bytes (8 16-bit elements or 4 floats),
// the last of which may be short.  Whole chunks are one access through a type of 2- resp. 4-byte alignment (the target's
// vector memory accesses need no more, and at aligned addresses it is the same instruction); short ones go element by element.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm_mfma.hip.h"

namespace flashdp {

// By value: applied to an element of a vector in place, the builtin reads the vector's first element.
__device__ __forceinline__ float as_float(uint32_t bits) { return __builtin_bit_cast(float, bits); }

template <int DT> struct Chunk {
  static constexpr int N = DT == DT_F32 ? 4 : 8;      // elements
  static constexpr int BYTES = DT == DT_F32 ? 4 : 2;  // of one
};

// Elements col .. of a row, `left` of which exist (none if left <= 0); what does not exist reads as zero.  EVEN: rows are whole chunks
// (the code for short ones costs registers where a thread holds several chunks).
template <int DT, bool EVEN = false>
__device__ __forceinline__ u32x4_t load_chunk(const void* row, int64_t col, int64_t left) {
  u32x4_t v = {0u, 0u, 0u, 0u};
  if constexpr (EVEN) {
    if (left > 0) v = *(const u32x4_t*)((const char*)row + col * Chunk<DT>::BYTES);
  } else if (left >= Chunk<DT>::N) {
    v = *(const u32x4_any_t*)((const char*)row + col * Chunk<DT>::BYTES);
  } else if constexpr (DT == DT_F32) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < left) v[k] = ((const uint32_t*)row)[col + k];
  } else {
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < left) v[k >> 1] |= (uint32_t)((const unsigned short*)row)[col + k] << (16 * (k & 1));
  }
  return v;
}

template <int DT, bool EVEN = false>
__device__ __forceinline__ void store_chunk(void* row, int64_t col, int64_t left, const u32x4_t v) {
  if constexpr (EVEN) {
    if (left > 0) *(u32x4_t*)((char*)row + col * Chunk<DT>::BYTES) = v;
  } else if (left >= Chunk<DT>::N) {
    *(u32x4_any_t*)((char*)row + col * Chunk<DT>::BYTES) = v;
  } else if constexpr (DT == DT_F32) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < left) ((uint32_t*)row)[col + k] = v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < left) ((unsigned short*)row)[col + k] = (unsigned short)(v[k >> 1] >> (16 * (k & 1)));
  }
}

template <int DT>
__device__ __forceinline__ void widen_chunk(const u32x4_t v, float (&f)[Chunk<DT>::N]) {
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = as_float(v[k]);
  } else if constexpr (DT == DT_BF16) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[2 * q] = __builtin_bit_cast(float, v[q] << 16);
      f[2 * q + 1] = __builtin_bit_cast(float, v[q] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[2 * q] = (float)__builtin_bit_cast(_Float16, (unsigned short)(v[q] & 0xFFFFu));
      f[2 * q + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(v[q] >> 16));
    }
  }
}

template <int DT>
__device__ __forceinline__ u32x4_t round_chunk(const float (&f)[Chunk<DT>::N]) {
  u32x4_t v;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (DT == DT_F32) v[q] = __builtin_bit_cast(uint32_t, f[q]);
    else v[q] = pack2_16bit<DT>(f[2 * q], f[2 * q + 1]);
  }
  return v;
}

// v of the lane whose number differs in the given way, inside rows of 16 lanes: in one vector-ALU instruction, where a general exchange
// goes through LDS.  A reversal within 8 or 16 lanes stands for lane ^ 4 or ^ 8 where all lanes of a quad (an eighth) hold the same value.
enum : int { LANE_XOR_1 = 0xB1, LANE_XOR_2 = 0x4E, LANE_REVERSE_8 = 0x141, LANE_REVERSE_16 = 0x140 };   // DPP controls
template <int CTRL>
__device__ __forceinline__ uint32_t lane_exchange(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ float lane_exchange(float v) { return __builtin_bit_cast(float, lane_exchange<CTRL>(__builtin_bit_cast(uint32_t, v))); }

// Sum over the 64 lanes of a wave, the same bits in every lane (every step adds the same two values in both partners).
__device__ __forceinline__ float wave_sum(float v) {
  v += lane_exchange<LANE_XOR_1>(v);
  v += lane_exchange<LANE_XOR_2>(v);
  v += lane_exchange<LANE_REVERSE_8>(v);
  v += lane_exchange<LANE_REVERSE_16>(v);
  // rows of 16 lanes, then halves of 32, change places between two copies
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  const auto rows = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  v = __builtin_bit_cast(float, (uint32_t)rows[0]) + __builtin_bit_cast(float, (uint32_t)rows[1]);
  const uint32_t c = __builtin_bit_cast(uint32_t, v);
  const auto halves = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  return __builtin_bit_cast(float, (uint32_t)halves[0]) + __builtin_bit_cast(float, (uint32_t)halves[1]);
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

}  // namespace flashdp
