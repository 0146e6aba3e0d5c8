// Activations in 8 bits between forward and backward pass.
//
// Blocks of 32 consecutive features of a row share an exponent e, an element is q 2^e, -127 <= q <= 127:
//   m = largest finite magnitude of the block, e = max(floor(log2 m) - 6, least), q = clamp(round(x 2^-e), -127, 127).
// So 64 <= m 2^-e < 128: an element is off by at most 2^e / 2 <= m / 128 (the clamp cuts what rounds to 128, which is then off by
// less than 2^e).  A power of two as scale, at the cost of up to one bit of resolution, makes both directions exact but for the
// one rounding: x 2^-e is exact in fp32, ties included, and q 2^e has 7 significant bits, so it is exact in bfloat16, fp16 and fp32
// alike and the backward pass contracts the very values that were kept.  The scale depends on one row alone: a sample's gradient
// is a function of that sample only, which the clipping needs.
// least = -126 keeps 2^e and 2^-e normal numbers (blocks below 2^-120 lose resolution); for fp16 -24, the step of its subnormals,
// of which every fp16 number is a multiple.  An element that is not finite is kept as q = -128 and comes back as NaN.
// Layout: q of all rows, [rows][d] int8, up to a multiple of 16 bytes; then e + 127 of all blocks, [rows][ceil(d / 32)] uint8.
//
// Memory bound: 2 (4) + 33/32 bytes an element; 16384 x 5120 bf16 packed in 52 us = 4.9 TB/s, unpacked in 38 (a part from the caches).  Four lanes (fp32: eight) hold a block and agree on m by exchanges inside the wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vector_io.hip.h"

namespace flashdp {

constexpr int CKPT8_BLOCK = 32;

__host__ __device__ __forceinline__ int64_t checkpoint8_blocks(int64_t d) { return (d + CKPT8_BLOCK - 1) / CKPT8_BLOCK; }
__host__ __device__ __forceinline__ int64_t checkpoint8_scales_at(int64_t rows, int64_t d) { return (rows * d + 15) / 16 * 16; }

template <int DT> struct Checkpoint8Least { static constexpr int EXP = DT == DT_F16 ? -24 : -126; };

__device__ __forceinline__ bool finite_f32(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// e of a block whose largest finite magnitude is m
template <int DT>
__device__ __forceinline__ int checkpoint8_exponent(float m) {
  const int e = (int)(__builtin_bit_cast(uint32_t, m) >> 23) - 127 - 6;
  return e < Checkpoint8Least<DT>::EXP ? Checkpoint8Least<DT>::EXP : e;
}
// The largest m of PER (4 or 8) neighbouring lanes, in all of them.
template <int PER>
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t m) {
  m = max(m, lane_exchange<LANE_XOR_1>(m));
  m = max(m, lane_exchange<LANE_XOR_2>(m));
  return PER == 8 ? max(m, lane_exchange<LANE_REVERSE_8>(m)) : m;
}

// Bits of the largest magnitude of N values of a block that PER neighbouring lanes hold, agreed on by them (magnitudes compare as integers).
// From CKPT8_NOT_FINITE on, the block has a value that is not finite: the top bit is set then, below it the bits of the largest finite one.
constexpr uint32_t CKPT8_NOT_FINITE = 0x80000000u;
template <int N, int PER>
__device__ __forceinline__ uint32_t checkpoint8_top(const float (&f)[N]) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) m = max(m, __builtin_bit_cast(uint32_t, f[k]) & 0x7FFFFFFFu);
  m = max_of_lanes<PER>(m);
  if (m >= 0x7F800000u) {     // the same in all lanes of the block
    m = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) m = max(m, finite_f32(f[k]) ? __builtin_bit_cast(uint32_t, f[k]) & 0x7FFFFFFFu : 0u);
    m = max_of_lanes<PER>(m) | CKPT8_NOT_FINITE;
  }
  return m;
}
// Four q, a byte each, of finite values in a block of scale 2^-e = inv.  Cut to -127 .. 127 and added to 1.5 * 2^23, a value is rounded to an
// integer, ties to even, and stands in the low byte of the sum.
__device__ __forceinline__ uint32_t checkpoint8_quantise4(const float* f, float inv) {
  uint32_t b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) b[k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(f[k] * inv, -127.0f, 127.0f) + 12582912.0f);
  const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0C0C0400u);
  return hi << 16 | lo;
}

// The values of N q, a byte each, of a block of the given scale 2^e: a byte with its sign bit turned is u = q + 128, which converts in one
// instruction, and u 2^e - 128 2^e is exact.  Gone through again are words with a zero among those bytes, which is q = -128, a value that was
// not finite, and blocks of e = 121, where 128 2^e overflows.
template <int N>
__device__ __forceinline__ void checkpoint8_values(const uint32_t (&v)[N / 4], float scale, float (&f)[N]) {
  const float offset = -128.0f * scale;
  uint32_t zero = 0;
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    const uint32_t u = v[k] ^ 0x80808080u;
    zero |= (u - 0x01010101u) & ~u & 0x80808080u;
#pragma unroll
    for (int b = 0; b < 4; ++b) f[4 * k + b] = fmaf((float)((u >> (8 * b)) & 0xFFu), scale, offset);
  }
  if (zero || !finite_f32(offset)) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t byte = (v[k >> 2] >> (8 * (k & 3))) & 0xFFu;
      f[k] = byte == 0x80u ? __builtin_bit_cast(float, 0x7FC00000u) : (float)(signed char)byte * scale;
    }
  }
}

typedef uint32_t u32_any_t __attribute__((aligned(1)));

// Up to n bytes of q (n = 8 or 4, one chunk) at q[col ..], `left` of which exist; what does not exist reads as zero.
template <int N>
__device__ __forceinline__ void load_q(const signed char* q, int64_t left, uint32_t (&v)[N / 4]) {
  if (left >= N) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) v[k] = ((const u32_any_t*)q)[k];
  } else {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) v[k] = 0u;
#pragma unroll
    for (int k = 0; k < N - 1; ++k)
      if (k < left) v[k >> 2] |= (uint32_t)(unsigned char)q[k] << (8 * (k & 3));
  }
}

// The q of a chunk of a block with the given top (checkpoint8_top) to q[0 ..], `left` > 0 of which exist; returns the block's e.
template <int DT>
__device__ __forceinline__ int checkpoint8_keep(signed char* q, int left, const float (&f)[Chunk<DT>::N], uint32_t top) {
  constexpr int N = Chunk<DT>::N;
  const int e = checkpoint8_exponent<DT>(__builtin_bit_cast(float, top & ~CKPT8_NOT_FINITE));
  const float inv = power_of_two(-e);
  uint32_t v[N / 4];
#pragma unroll
  for (int k = 0; k < N / 4; ++k) v[k] = checkpoint8_quantise4(f + 4 * k, inv);
  if (top >= CKPT8_NOT_FINITE) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (!finite_f32(f[k])) v[k >> 2] = (v[k >> 2] & ~(0xFFu << (8 * (k & 3)))) | 0x80u << (8 * (k & 3));
  }
  if (left >= N) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) ((u32_any_t*)q)[k] = v[k];
  } else {
#pragma unroll
    for (int k = 0; k < N - 1; ++k)
      if (k < left) q[k] = (signed char)(v[k >> 2] >> (8 * (k & 3)));
  }
  return e;
}

// One chunk of 16 bytes of x per thread (two or four, a workgroup apart: 16384 x 5120 bf16 packed and unpacked 97.7 us, 90.1 so).  The chunks of
// a row fill whole blocks (chunks past the row's end hold zeros and store nothing), so the lanes of a block are neighbours in one wave.
// FLAT: d is whole blocks, and chunk c is simply elements N c on; otherwise a chunk's place costs a division (93.5 us).
struct Checkpoint8Place { int64_t at, block; int left; };   // element, block, elements that exist
template <int N, bool FLAT>
__device__ __forceinline__ Checkpoint8Place checkpoint8_place(int64_t c, int64_t chunks, int64_t d) {
  constexpr int PER = CKPT8_BLOCK / N;   // chunks per block
  const int64_t block = c / PER;
  if (c >= chunks) return {0, 0, 0};
  if constexpr (FLAT) return {c * N, block, N};
  const int64_t nb = checkpoint8_blocks(d), row = block / nb;
  const int64_t col = (block - row * nb) * CKPT8_BLOCK + (c % PER) * N;
  return {row * d + col, block, (int)max((int64_t)0, min((int64_t)N, d - col))};
}

template <int DT, bool FLAT>
__global__ __launch_bounds__(256) void checkpoint8_pack_kernel(const void* x, int64_t chunks, int64_t d, signed char* q, unsigned char* scales) {
  constexpr int N = Chunk<DT>::N, PER = CKPT8_BLOCK / N;
  const Checkpoint8Place p = checkpoint8_place<N, FLAT>((int64_t)blockIdx.x * 256 + threadIdx.x, chunks, d);
  float f[N];
  widen_chunk<DT>(load_chunk<DT, FLAT>(x, p.at, p.left), f);
  const uint32_t top = checkpoint8_top<N, PER>(f);
  if (p.left <= 0) return;
  const int e = checkpoint8_keep<DT>(q + p.at, p.left, f, top);
  if ((threadIdx.x & (PER - 1)) == 0) scales[p.block] = (unsigned char)(e + 127);
}

// And back.
template <int DT, bool FLAT>
__global__ __launch_bounds__(256) void checkpoint8_unpack_kernel(const signed char* q, const unsigned char* scales, int64_t chunks, int64_t d, void* x) {
  constexpr int N = Chunk<DT>::N;
  const Checkpoint8Place p = checkpoint8_place<N, FLAT>((int64_t)blockIdx.x * 256 + threadIdx.x, chunks, d);
  if (p.left <= 0) return;
  uint32_t v[N / 4];
  load_q<N>(q + p.at, p.left, v);
  float f[N];
  checkpoint8_values<N>(v, power_of_two((int)scales[p.block] - 127), f);
  store_chunk<DT, FLAT>(x, p.at, p.left, round_chunk<DT>(f));
}

}  // namespace flashdp
