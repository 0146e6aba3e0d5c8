// C ABI of the layers around the DP weight gradient (see include/flashdp.h): the forward product with its epilogue, the backward pass
// of activation and bias, layer normalisation, 8-bit checkpoints.  Host code validates, sizes workspaces, picks kernels and
// enqueues them.
#include "../../include/flashdp.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "activation_dp.hip.h"
#include "api_internal.h"
#include "checkpoint8.hip.h"
#include "forward_deep.hip.h"
#include "forward_large.hip.h"
#include "forward_rows.hip.h"
#include "forward_split.hip.h"
#include "forward_tile.hip.h"
#include "layernorm.hip.h"
#include "vector_dp.hip.h"

using namespace flashdp;

namespace {

#define HIP_TRY(expr) do { if ((expr) != hipSuccess) { (void)hipGetLastError(); return FLASHDP_HIP_ERROR; } } while (0)

constexpr int64_t GRID_LIMIT = (int64_t(1) << 31) - 1;
constexpr int64_t FEATURE_LIMIT = int64_t(1) << 30;      // columns are computed in 32 bits
constexpr int64_t ROW_LIMIT = int64_t(1) << 40;
constexpr int64_t ELEMENT_LIMIT = int64_t(1) << 58;      // offsets and sizes in bytes are computed in 64 bits

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool valid_dtype(int d) { return d == FLASHDP_BF16 || d == FLASHDP_F32 || d == FLASHDP_F16; }
inline bool valid_act(int a) { return a >= FLASHDP_ACT_NONE && a <= FLASHDP_ACT_SILU; }
inline bool valid_clip(float C, float sigma) { return C > 0.0f && std::isfinite(C) && sigma >= 0.0f && std::isfinite(sigma); }

int check_rows(int64_t rows, int64_t d) {
  if (rows <= 0 || d <= 0) return FLASHDP_INVALID_ARGUMENT;
  return rows >= ROW_LIMIT || d > FEATURE_LIMIT || rows > ELEMENT_LIMIT / d ? FLASHDP_UNSUPPORTED_SHAPE : FLASHDP_OK;
}
int check_samples(int64_t B, int64_t T, int64_t d) {
  if (B <= 0 || T <= 0 || d <= 0) return FLASHDP_INVALID_ARGUMENT;
  return B >= (int64_t(1) << 20) || T >= (int64_t(1) << 31) ? FLASHDP_UNSUPPORTED_SHAPE : check_rows(B * T, d);
}

// f(integral_constant<DT>) for the storage type of a call
template <typename F>
auto by_dtype(int dtype, F&& f) {
  if (dtype == FLASHDP_BF16) return f(std::integral_constant<int, DT_BF16>{});
  if (dtype == FLASHDP_F16) return f(std::integral_constant<int, DT_F16>{});
  return f(std::integral_constant<int, DT_F32>{});
}
inline int chunk_elements(int dtype) { return dtype == FLASHDP_F32 ? 4 : 8; }

template <typename... Formal, typename... Actual>
hipError_t launch(void (*kernel)(Formal...), int64_t grid, int threads, size_t lds, hipStream_t st, Actual... args) {
  if (grid <= 0 || grid > GRID_LIMIT) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3((unsigned)threads), lds, st, args...);
  return hipGetLastError();
}

// ---- per-sample gradients of vectors ----------------------------------------------------------------

struct VectorWs { size_t partial, g, squares, factors, total; int blocks; };

// blocks: sums of squares per sample that the kernel before leaves, 0 if vector_sum_kernel does
VectorWs vector_ws(int64_t B, int64_t chunks, int64_t n, int64_t blocks) {
  VectorWs w;
  w.blocks = (int)(blocks ? blocks : (n + 63) / 64);
  w.partial = 0;
  w.g = align_up((size_t)B * chunks * n * 4, 256);
  w.squares = w.g + (chunks > 1 ? align_up((size_t)B * n * 4, 256) : 0);
  w.factors = w.squares + align_up((size_t)B * w.blocks * 8, 256);
  w.total = w.factors + align_up((size_t)B * 4, 256);
  return w;
}

// What comes after the partial sums: their sum (if summed is false), norms, clip factors, the clipped sum and its noise.
hipError_t run_vector(VectorArgs& v, char* ws, const VectorWs& w, bool summed, hipStream_t st) {
  v.partial = reinterpret_cast<const float*>(ws + w.partial);
  v.g = reinterpret_cast<float*>(ws + (v.chunks > 1 ? w.g : w.partial));
  v.squares = reinterpret_cast<double*>(ws + w.squares);
  v.factors = reinterpret_cast<float*>(ws + w.factors);
  v.blocks = w.blocks;
  hipError_t e = summed ? hipSuccess : launch(vector_sum_kernel, v.B * v.blocks, 256, 0, st, v);
  if (e != hipSuccess) return e;
  const bool fold = v.B <= VECTOR_FOLD_B && v.B * v.blocks <= VECTOR_FOLD_SQUARES;
  if (!fold && (e = launch(vector_factors_kernel, (v.B + 3) / 4, 256, 0, st, v)) != hipSuccess) return e;
  // few samples: whole cache lines of elements side by side; many: rows of threads to share them
  if (v.B <= 16) return launch(fold ? vector_clip_kernel<true, 64> : vector_clip_kernel<false, 64>, (v.n + 63) / 64, 256, 0, st, v);
  return launch(fold ? vector_clip_kernel<true, 16> : vector_clip_kernel<false, 16>, (v.n + 15) / 16, 256, 0, st, v);
}

struct ActivationPlan {
  int log_ct;
  int64_t col_tiles, chunks, rows_per_chunk;
  bool token;
  int64_t squares() const { return chunks == 1 ? col_tiles : 0; }      // per sample, from the kernel
};

ActivationPlan activation_plan(int64_t B, int64_t T, int64_t d, int dtype) {
  ActivationPlan p;
  const int64_t columns = (d + chunk_elements(dtype) - 1) / chunk_elements(dtype);
  p.log_ct = 3;
  while (p.log_ct < 6 && (int64_t(1) << p.log_ct) < columns) ++p.log_ct;
  p.col_tiles = (columns + (1 << p.log_ct) - 1) >> p.log_ct;
  p.token = T == 1;
  // tokens per partial sum: at most the six workgroups per compute unit that are there at a time (8192 x 3072, 8 samples, Z in 8 bits, all three
  // kernels: two 38.2, four 36.4, six 34.7, eight 37.5 us), and whole trips of the kernel's loop, 16 tokens or more, below which writing
  // and reading the partial sums shows
  const int64_t k = p.token ? 1 : std::max<int64_t>(1, 6 * 256 / (B * p.col_tiles)), trip = 4 * (256 >> p.log_ct);
  p.rows_per_chunk = std::min(T, ((T + k - 1) / k + trip - 1) / trip * trip);
  p.chunks = (T + p.rows_per_chunk - 1) / p.rows_per_chunk;
  return p;
}

template <int DT, int ZK>
auto activation_kernel(int act, bool token) {
  if constexpr (ZK == Z_NONE) return token ? activation_dp_kernel<DT, ACT_NONE, ZK, true> : activation_dp_kernel<DT, ACT_NONE, ZK, false>;
  else switch (act) {
    case FLASHDP_ACT_RELU: return token ? activation_dp_kernel<DT, ACT_RELU, ZK, true> : activation_dp_kernel<DT, ACT_RELU, ZK, false>;
    case FLASHDP_ACT_GELU: return token ? activation_dp_kernel<DT, ACT_GELU, ZK, true> : activation_dp_kernel<DT, ACT_GELU, ZK, false>;
    case FLASHDP_ACT_GELU_TANH: return token ? activation_dp_kernel<DT, ACT_GELU_TANH, ZK, true> : activation_dp_kernel<DT, ACT_GELU_TANH, ZK, false>;
    default: return token ? activation_dp_kernel<DT, ACT_SILU, ZK, true> : activation_dp_kernel<DT, ACT_SILU, ZK, false>;
  }
}

// ---- layer normalisation ----------------------------------------------------------------------------

// Chunks of 16 bytes a row has decide who holds it: a wave up to 4 chunks a lane, a workgroup up to 8, nobody beyond.  Rows that are no whole
// chunks have fewer kernels to choose from.
constexpr int64_t NORM_LONG = 256 * 8;

template <int DT>
void (*norm_kernel(int64_t columns, bool even))(const NormArgs) {
  if (!even) {
    if (columns <= 128) return layernorm_forward_kernel<DT, 64, 2, false>;
    if (columns <= 256) return layernorm_forward_kernel<DT, 64, 4, false>;
    if (columns <= 1024) return layernorm_forward_kernel<DT, 256, 4, false>;
    return layernorm_forward_kernel<DT, 256, 8, false>;
  }
  if (columns <= 64) return layernorm_forward_kernel<DT, 64, 1, true>;
  if (columns <= 128) return layernorm_forward_kernel<DT, 64, 2, true>;
  if (columns <= 256) return layernorm_forward_kernel<DT, 64, 4, true>;
  if (columns <= 512) return layernorm_forward_kernel<DT, 256, 2, true>;
  if (columns <= 768) return layernorm_forward_kernel<DT, 256, 3, true>;
  if (columns <= 1024) return layernorm_forward_kernel<DT, 256, 4, true>;
  return layernorm_forward_kernel<DT, 256, 8, true>;
}

struct NormGradKernel { void (*kernel)(const NormGradArgs); int threads, rows; };   // of a workgroup; rows: that it goes through side by side
template <int DT, int NT, int CH, int THREADS, bool EVEN>
NormGradKernel norm_grad_of(bool token) {
  return {token ? layernorm_grad_kernel<DT, NT, CH, THREADS, true, EVEN> : layernorm_grad_kernel<DT, NT, CH, THREADS, false, EVEN>, THREADS, THREADS / NT};
}
template <int DT>
NormGradKernel norm_grad_kernel(int64_t columns, bool even, bool token) {
  if (!even) {
    if (columns <= 128) return norm_grad_of<DT, 64, 2, 256, false>(token);
    if (columns <= 256) return norm_grad_of<DT, 64, 4, 256, false>(token);
    if (columns <= 1024) return norm_grad_of<DT, 256, 4, 256, false>(token);
    return norm_grad_of<DT, 256, 8, 256, false>(token);
  }
  if (columns <= 64) return norm_grad_of<DT, 64, 1, 1024, true>(token);
  if (columns <= 128) return norm_grad_of<DT, 64, 2, 1024, true>(token);
  if (columns <= 256) return norm_grad_of<DT, 64, 4, 512, true>(token);
  if (columns <= 512) return norm_grad_of<DT, 256, 2, 1024, true>(token);
  if (columns <= 768) return norm_grad_of<DT, 256, 3, 1024, true>(token);
  if (columns <= 1024) return norm_grad_of<DT, 256, 4, 512, true>(token);
  return norm_grad_of<DT, 256, 8, 256, true>(token);
}
NormGradKernel norm_grad_kernel_of(int64_t d, int dtype, bool token) {
  const int64_t n = chunk_elements(dtype), columns = (d + n - 1) / n;
  return by_dtype(dtype, [&](auto dt) { return norm_grad_kernel<decltype(dt)::value>(columns, d % n == 0, token); });
}

struct NormPlan { int64_t columns, col_tiles, chunks, rows_per_chunk, squares; bool token; };   // squares: per sample, from the kernel

NormPlan norm_plan(int64_t B, int64_t T, int64_t d, int dtype) {
  NormPlan p;
  p.columns = (d + chunk_elements(dtype) - 1) / chunk_elements(dtype);
  const bool held = p.columns <= NORM_LONG;
  p.col_tiles = held ? 1 : (p.columns + 255) / 256;
  p.token = held && T == 1;
  // about two times 16 waves per compute unit, every workgroup going through its rows at least twice, and no fewer than 16 tokens to a partial
  // sum, below which writing and reading them shows
  const NormGradKernel kernel = held ? norm_grad_kernel_of(d, dtype, p.token) : NormGradKernel{nullptr, 256, 8};
  const int64_t want = (2 * 256 * (1024 / kernel.threads) + B * p.col_tiles - 1) / (B * p.col_tiles), fewest = std::max(2 * kernel.rows, 16);
  const int64_t k = p.token ? 1 : std::max<int64_t>(1, std::min(want, (T + fewest - 1) / fewest));
  p.rows_per_chunk = (T + k - 1) / k;
  p.chunks = (T + p.rows_per_chunk - 1) / p.rows_per_chunk;
  p.squares = !held || p.chunks > 1 ? 0 : kernel.threads / (p.token ? kernel.rows : 1) / 64;
  return p;
}

// ---- the forward product ----------------------------------------------------------------------------

// Which kernel forms a product.  For rows of whole 16-byte chunks a ladder of tiles; a call takes the one whose rounds are
// the shortest.  A round of `per_cu` workgroups on every compute unit takes start + tile * (k-tiles of 128 bytes) microseconds, one
// of at most one workgroup per unit start + alone * k-tiles, and epilogue more where the epilogue has an activation or 8-bit sums (fitted to 170
// products of one to 8192 rows, 768 to 13824 features; 16-bit types, then fp32, whose k-tiles are half as deep).  us, tiles of 16 x 16, 16 x 32, 32 x 32,
// 64 x 64, 128 x 128, 128 x 128 with two workgroups per unit, 256 x 256 (- = not tried), operands in the caches (from memory the order is the
// same: 128 x 4096 -> 4096: -, -, 20, 21, 40, 64, 99; 512 x 4096 -> 4096: -, -, 61, 39, 40, 63, 103; 256 x 5120 -> 13824: -, -, 144, 100, 58, 89, 148):
// bf16 1 x 4096 -> 4096: 7.2, 10.0, 10.0, 14.7, 34, -, -; fp16 8 x 768 -> 50257: 23.3, 16.6, 18.4, 22.4, -, -, -; bf16 128 x 4096 -> 4096: -, -, 14.6, 15.2, 34.9, 46, 74;
// 256 x 4096 -> 4096: -, -, 26.2, 15.9, 35.1, 46, 76; 1024 x 4096 -> 4096: -, -, 89, 59, 38.9, 49, 76; fp16 2048 x 4096 -> 4096: -, -, 178, 120, 80, 62, 80;
// bf16 8192 x 5120 -> 13824: -, -, 3397, 2425, 1328, 1174, 907; 8192 x 768 -> 3072: -, -, 167, 109, 62, 51, 51, with GELU and Z in 8 bits -, -, -, 127, 80, 62, 69.
// fp32, 32 x 32, 64 x 64, 128 x 128 twice, then in bfloat16 parts on 64 x 128 and 128 x 256: 128 x 4096 -> 4096: 55, 78, 247, 153, 287; 512 x 4096 -> 4096: 173,
// 150, 249, 138, 292; 2048 x 4096 -> 4096: 663, 586, 478, 400, 318; 8192 x 768 -> 3072: 429, 382, 286, 239, 198 (errors: forward_split.hip.h).
// Rows that no 16-byte chunks divide: direct loads to LDS need 4-byte alignment.  Up to 64 rows the kernel that reads W straight into
// registers is the faster one until its workgroups of 32 features go in several rounds, sooner where rows start at odd multiples of two bytes; then tiles staged
// through registers are, and fp32 in parts (costs of these fitted to 760 products of 1 to 64 rows, 33 to 13825, 40 to 50257 features; us, straight
// from memory and tiles of 64 x 64, fp32 also parts on 64 x 128: bf16 1 x 4097 -> 4096: 28, 80; 64 x 4097 -> 4096: 76, 66; 64 x 4098 -> 4096: 34, 60;
// 8 x 769 -> 50257: 54, 24; 8 x 2050 -> 50257: 59, 52; fp32 64 x 4097 -> 4096: 66, 114, 181; 8 x 4097 -> 50257: 227, 338, 233; 64 x 1001 -> 50257: 123, 94, 71).
// Beyond, tiles of 64 x 64 or 128 x 128 and the parts where they are faster (fp32 1024 x 1001 -> 2304: 70, 59).
enum ForwardPath { FWD_16x16 = 0, FWD_16x32, FWD_32x32, FWD_64x64, FWD_128x128, FWD_128x128_TWO, FWD_256x256, FWD_ROWS, FWD_ANY_64, FWD_ANY_128, FWD_SPLIT, FWD_SPLIT_SMALL, FWD_PATHS };
struct ForwardCost { double start, tile, alone; };
struct ForwardRung { ForwardPath path; int bm, bn, per_cu; ForwardCost bits16, bits32; double epilogue; bool direct; };   // no tile: not for that type
constexpr ForwardRung FORWARD_LADDER[] = {
    {FWD_16x16, 16, 16, 2, {1.9, 0.115, 0.085}, {1.9, 0.115, 0.09}, 0.2, true},   {FWD_16x32, 16, 32, 3, {2.0, 0.15, 0.12}, {2.0, 0.3, 0.21}, 0.3, true},
    {FWD_32x32, 32, 32, 2, {1.6, 0.18, 0.1}, {1.6, 0.34, 0.2}, 0.4, true},        {FWD_64x64, 64, 64, 1, {2.6, 0.19, 0.19}, {2.6, 0.56, 0.56}, 0.7, true},
    {FWD_128x128, 128, 128, 1, {4.0, 0.54, 0.54}, {}, 2.9, true},                 {FWD_128x128_TWO, 128, 128, 2, {6.6, 0.87, 0.65}, {6.6, 3.7, 1.92}, 3.7, true},
    {FWD_256x256, 256, 256, 1, {7.0, 1.54, 1.54}, {}, 9.0, true},                 {FWD_SPLIT, 128, 256, 1, {}, {9.5, 2.43, 2.2}, 4.5, false},
    {FWD_SPLIT_SMALL, 64, 128, 2, {}, {5.6, 1.53, 0.98}, 2.0, false}};
constexpr int64_t SPLIT_LEAST = 64;   // fewest products of a sum formed from parts: from there on they are closer than the fp32 instruction in every way (forward_split.hip.h)

bool forward_direct(int64_t d_in, int dtype) { return d_in * (dtype == FLASHDP_F32 ? 4 : 2) % 16 == 0; }
// 256 rows lie within the 2 GiB that a buffer descriptor reaches
bool forward_described(int64_t d_in, int dtype) { return d_in * (dtype == FLASHDP_F32 ? 4 : 2) < (int64_t(1) << 23) - 4096; }
// tiles of a rung, or -1 where they are too many for a grid
int64_t forward_tiles(int64_t rows, int64_t d_out, int bm, int bn) {
  const int64_t tm = (rows + bm - 1) / bm, tn = (d_out + bn - 1) / bn;
  return tm * 8 > GRID_LIMIT || tn * 8 > GRID_LIMIT || tm * tn > GRID_LIMIT ? -1 : tm * tn;
}

// blocks_of_32: Z goes out in 8 bits; busy: the epilogue has more to do than to round and store.
ForwardPath forward_path(int64_t rows, int64_t d_in, int64_t d_out, int dtype, bool blocks_of_32, bool busy) {
  const int forced = api::forward_override();
  const bool f32 = dtype == FLASHDP_F32, described = forward_described(d_in, dtype), direct = described && forward_direct(d_in, dtype);
  const int64_t cus = api::compute_units(), nk = (d_in * (f32 ? 4 : 2) + 127) / 128;
  ForwardPath best = FWD_PATHS;
  double least = 0.0;
  auto offer = [&](ForwardPath path, int64_t tiles, int per_cu, const ForwardCost& c, double epilogue) {
    const int64_t slots = cus * per_cu, rest = tiles % slots;
    const double start = c.start + (busy ? epilogue : 0.0);
    double t = (double)(tiles / slots) * (start + c.tile * nk) + (rest == 0 ? 0.0 : start + (rest <= cus ? c.alone : c.tile) * nk);
    if (forced == path) t = -1.0;
    if (best == FWD_PATHS || t < least) { best = path; least = t; }
  };
  const bool few = !direct && rows <= 64;
  if (few) {      // k-tiles of 128 bytes
    const double c = f32 || d_in % 2 == 0 ? 0.24 + 0.0043 * rows : 0.39 + 0.0116 * rows;
    offer(FWD_ROWS, (d_out + 31) / 32, 1, ForwardCost{1.2, c, c}, 0.0);
  }
  if (!direct) {
    const int64_t t64 = forward_tiles(rows, d_out, 64, 64), t128 = forward_tiles(rows, d_out, 128, 128);
    const bool small = forced == FWD_ANY_64 || (forced != FWD_ANY_128 && (few || t128 < 256));
    const ForwardCost c64 = few ? f32 ? ForwardCost{2.0, 2.2, 0.95} : ForwardCost{2.0, 1.4, 0.95 - 0.004 * rows} : f32 ? ForwardCost{3.0, 2.2, 0.83} : ForwardCost{3.0, 1.0, 0.57};
    if (small && t64 >= 0) offer(FWD_ANY_64, t64, 4, c64, 0.0);
    else if (t128 >= 0) offer(FWD_ANY_128, t128, 2, f32 ? ForwardCost{6.6, 4.4, 2.2} : ForwardCost{6.6, 1.28, 0.9}, 0.0);
  }
  for (const ForwardRung& g : FORWARD_LADDER) {
    const ForwardCost c = few && f32 && g.path == FWD_SPLIT_SMALL ? ForwardCost{5.6, 1.75, 1.3} : f32 ? g.bits32 : g.bits16;
    if (c.tile == 0.0 || (g.direct ? !direct : !described || (d_in < SPLIT_LEAST && forced != g.path)) || (blocks_of_32 && g.bn % CKPT8_BLOCK != 0)) continue;
    const int64_t tiles = forward_tiles(rows, d_out, g.bm, g.bn);
    if (tiles >= 0) offer(g.path, tiles, g.per_cu, c, g.epilogue);
  }
  return best;
}

template <typename Cfg>
hipError_t launch_forward(void (*kernel)(ForwardArgs), ForwardArgs& a, int64_t grid, hipStream_t st) {
  const hipError_t e = api::allow_lds(reinterpret_cast<const void*>(kernel), Cfg::LDS_BYTES);
  return e != hipSuccess ? e : launch(kernel, grid, Cfg::NT, Cfg::LDS_BYTES, st, a);
}
template <typename Cfg>
hipError_t launch_forward_tiles(void (*kernel)(ForwardArgs), ForwardArgs& a, hipStream_t st) {
  a.tiles_m = (int)((a.rows + Cfg::BM - 1) / Cfg::BM);
  a.tiles_n = (int)(((int64_t)a.D + Cfg::BN - 1) / Cfg::BN);
  return launch_forward<Cfg>(kernel, a, (int64_t)a.tiles_m * a.tiles_n, st);
}
template <typename Cfg, int DT>
hipError_t launch_forward_rows(ForwardArgs& a, hipStream_t st) {
  return launch_forward<Cfg>(forward_rows_kernel<Cfg, DT>, a, ((int64_t)a.D + 16 * Cfg::NF - 1) / (16 * Cfg::NF), st);
}

using Deep16x16 = ForwardDeepCfg<16, 16, 4, 1, 16, 4>;
using Deep16x32 = ForwardDeepCfg<16, 32, 2, 1, 8, 2>;
using Deep32x32 = ForwardDeepCfg<32, 32, 4, 1, 8, 2>;
using Deep64x64 = ForwardDeepCfg<64, 64, 4, 2, 8, 2>;
using Deep128x128 = ForwardDeepCfg<128, 128, 2, 4, 4, 1>;

using Split128x256 = ForwardSplitCfg<128, 256, 2, 4>;
using Split64x128 = ForwardSplitCfg<64, 128, 2, 2>;
template <typename Cfg>
hipError_t launch_forward_split(ForwardArgs& a, hipStream_t st) {
  return launch_forward_tiles<Cfg>(a.K % 4 == 0 ? forward_split_kernel<Cfg, false> : forward_split_kernel<Cfg, true>, a, st);
}

template <int DT>
hipError_t run_forward(ForwardPath path, ForwardArgs& a, hipStream_t st) {
  switch (path) {
    case FWD_16x16: return launch_forward_tiles<Deep16x16>(forward_deep_kernel<Deep16x16, DT>, a, st);
    case FWD_16x32: return launch_forward_tiles<Deep16x32>(forward_deep_kernel<Deep16x32, DT>, a, st);
    case FWD_32x32: return launch_forward_tiles<Deep32x32>(forward_deep_kernel<Deep32x32, DT>, a, st);
    case FWD_64x64: return launch_forward_tiles<Deep64x64>(forward_deep_kernel<Deep64x64, DT>, a, st);
    case FWD_128x128: if constexpr (DT != DT_F32) return launch_forward_tiles<Deep128x128>(forward_deep_kernel<Deep128x128, DT>, a, st); else return hipErrorInvalidValue;
    case FWD_128x128_TWO: return launch_forward_tiles<ForwardLarge128>(forward_large_kernel<ForwardLarge128, DT>, a, st);
    case FWD_256x256: if constexpr (DT != DT_F32) return launch_forward_tiles<ForwardLarge256>(forward_large_kernel<ForwardLarge256, DT>, a, st); else return hipErrorInvalidValue;
    case FWD_ROWS:
      if (a.rows <= 16) return launch_forward_rows<ForwardRowsCfg<2, 1, 8>, DT>(a, st);
      if (a.rows <= 32) return launch_forward_rows<ForwardRowsCfg<2, 2, 8>, DT>(a, st);
      return launch_forward_rows<ForwardRowsCfg<2, 4, 8>, DT>(a, st);
    case FWD_SPLIT: if constexpr (DT == DT_F32) return launch_forward_split<Split128x256>(a, st); else return hipErrorInvalidValue;
    case FWD_SPLIT_SMALL: if constexpr (DT == DT_F32) return launch_forward_split<Split64x128>(a, st); else return hipErrorInvalidValue;
    case FWD_ANY_64: return launch_forward_tiles<ForwardTileCfg<64, 64>>(forward_tile_kernel<ForwardTileCfg<64, 64>, DT>, a, st);
    case FWD_ANY_128: return launch_forward_tiles<ForwardTileCfg<128, 128>>(forward_tile_kernel<ForwardTileCfg<128, 128>, DT>, a, st);
    default: return hipErrorInvalidValue;
  }
}

const char* forward_kernel_name(ForwardPath path) {
  return path == FWD_ROWS ? "forward_rows_kernel" : path == FWD_ANY_64 || path == FWD_ANY_128 ? "forward_tile_kernel"
         : path == FWD_SPLIT || path == FWD_SPLIT_SMALL ? "forward_split_kernel"
         : path == FWD_128x128_TWO || path == FWD_256x256 ? "forward_large_kernel" : "forward_deep_kernel";
}

}  // namespace

extern "C" {

int flashdp_linear_forward(const void* X, const void* W, const void* bias, const void* residual, int64_t rows, int64_t d_in, int64_t d_out,
                           int dtype, int activation, void* Y, void* Z, int z_8bit, void* stream) {
  if (!X || !W || !Y || !valid_dtype(dtype) || !valid_act(activation) || (z_8bit != 0 && z_8bit != 1) || (z_8bit && !Z)) return FLASHDP_INVALID_ARGUMENT;
  int st = check_rows(rows, d_in);
  if (st == FLASHDP_OK) st = check_rows(rows, d_out);
  if (st != FLASHDP_OK) return st;
  const ForwardPath path = forward_path(rows, d_in, d_out, dtype, z_8bit != 0, activation != FLASHDP_ACT_NONE || z_8bit != 0);
  if (path == FWD_PATHS) return FLASHDP_UNSUPPORTED_SHAPE;    // more tiles than a grid holds
  if (!aligned(X, 16) || !aligned(W, 16) || !aligned(bias, 16) || !aligned(residual, 16) || !aligned(Y, 16) || !aligned(Z, 16)) return FLASHDP_MISALIGNED;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  ForwardArgs a;
  a.X = X; a.W = W; a.bias = bias; a.residual = residual; a.Y = Y; a.Z = Z;
  a.scales = z_8bit ? static_cast<unsigned char*>(Z) + checkpoint8_scales_at(rows, d_out) : nullptr;
  a.rows = rows; a.K = (int)d_in; a.D = (int)d_out;
  a.act = activation; a.keep = !Z ? KEEP_NONE : z_8bit ? KEEP_EIGHT : KEEP_SAME;
  a.tiles_m = a.tiles_n = 0;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  HIP_TRY(by_dtype(dtype, [&](auto dt) { return run_forward<decltype(dt)::value>(path, a, hs); }));
  api::note_kernel(forward_kernel_name(path));
  return FLASHDP_OK;
}

size_t flashdp_activation_workspace_bytes(int64_t B, int64_t T, int64_t d_out, int dtype) {
  if (!valid_dtype(dtype) || check_samples(B, T, d_out) != FLASHDP_OK) return 0;
  const ActivationPlan p = activation_plan(B, T, d_out, dtype);
  return vector_ws(B, p.chunks, d_out, p.squares()).total;
}

int flashdp_activation_dp_grad(const void* dY, const void* Z, int z_8bit, int64_t B, int64_t T, int64_t d_out, int dtype, int activation,
                               float C, float sigma, uint64_t seed, uint32_t layer, void* dZ, float* out_grad, float* out_norms,
                               void* workspace, size_t workspace_bytes, void* stream, int accumulate, int add_noise) {
  if (!dY || !valid_dtype(dtype) || !valid_act(activation) || (z_8bit != 0 && z_8bit != 1) || (!dZ && !out_grad)) return FLASHDP_INVALID_ARGUMENT;
  if (activation != FLASHDP_ACT_NONE && !Z) return FLASHDP_INVALID_ARGUMENT;
  if (out_grad && !valid_clip(C, sigma)) return FLASHDP_INVALID_ARGUMENT;
  int st = check_samples(B, T, d_out);
  if (st != FLASHDP_OK) return st;
  const bool use_z = activation != FLASHDP_ACT_NONE;
  if (!aligned(dY, 16) || (use_z && !aligned(Z, 16)) || !aligned(dZ, 16) || !aligned(out_grad, 16) || !aligned(out_norms, 4) || !aligned(workspace, 16))
    return FLASHDP_MISALIGNED;
  const ActivationPlan p = activation_plan(B, T, d_out, dtype);
  const int64_t rt = 256 >> p.log_ct, units = p.token ? (B + rt - 1) / rt : B * p.chunks;
  const VectorWs w = vector_ws(B, p.chunks, d_out, p.squares());
  if (units * p.col_tiles > GRID_LIMIT || B * w.blocks > GRID_LIMIT) return FLASHDP_UNSUPPORTED_SHAPE;
  if (out_grad && workspace && workspace_bytes < w.total) return FLASHDP_WORKSPACE_TOO_SMALL;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (out_grad && !workspace && (st = api::library_workspace(w.total, hs, &workspace)) != FLASHDP_OK) return st;
  char* ws = static_cast<char*>(workspace);
  ActivationArgs a;
  a.dY = dY; a.Z = Z; a.dZ = dZ;
  a.scales = use_z && z_8bit ? static_cast<const unsigned char*>(Z) + checkpoint8_scales_at(B * T, d_out) : nullptr;
  a.partial = out_grad ? reinterpret_cast<float*>(ws + w.partial) : nullptr;
  a.squares = out_grad ? reinterpret_cast<double*>(ws + w.squares) : nullptr;
  a.B = B; a.T = T; a.d = d_out;
  a.chunks = (int)p.chunks; a.rows_per_chunk = (int)p.rows_per_chunk; a.col_tiles = (int)p.col_tiles; a.log_ct = p.log_ct;
  HIP_TRY(by_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    auto kernel = !use_z ? activation_kernel<DT, Z_NONE>(activation, p.token) : z_8bit ? activation_kernel<DT, Z_EIGHT>(activation, p.token)
                                                                                       : activation_kernel<DT, Z_SAME>(activation, p.token);
    return launch(kernel, units * p.col_tiles, 256, 0, hs, a);
  }));
  api::note_kernel("activation_dp_kernel");
  if (!out_grad) return FLASHDP_OK;
  VectorArgs v;
  v.n = d_out; v.B = B; v.chunks = a.chunks;
  v.C = C; v.noise_scale = add_noise ? sigma * C : 0.0f; v.seed = seed; v.layer = layer; v.field = FLASHDP_FIELD_BIAS;
  v.out = out_grad; v.out_norms = out_norms; v.accumulate = accumulate ? 1 : 0;
  HIP_TRY(run_vector(v, ws, w, p.squares() != 0, hs));
  return FLASHDP_OK;
}

int flashdp_layernorm_forward(const void* X, const void* gamma, const void* beta, int64_t rows, int64_t d, int dtype, float eps, void* Y,
                              float* mean, float* rstd, void* stream) {
  if (!X || !gamma || !Y || !valid_dtype(dtype) || !(eps > 0.0f) || !std::isfinite(eps)) return FLASHDP_INVALID_ARGUMENT;
  int st = check_rows(rows, d);
  if (st != FLASHDP_OK) return st;
  if (rows > GRID_LIMIT) return FLASHDP_UNSUPPORTED_SHAPE;
  if (!aligned(X, 16) || !aligned(gamma, 16) || !aligned(beta, 16) || !aligned(Y, 16) || !aligned(mean, 4) || !aligned(rstd, 4)) return FLASHDP_MISALIGNED;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  NormArgs a;
  a.X = X; a.gamma = gamma; a.beta = beta; a.Y = Y; a.mean = mean; a.rstd = rstd; a.rows = rows; a.d = d; a.eps = eps;
  const int64_t columns = (d + chunk_elements(dtype) - 1) / chunk_elements(dtype);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  HIP_TRY(by_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (columns > NORM_LONG) return launch(layernorm_forward_long_kernel<DT>, rows, 256, 0, hs, a);
    return launch(norm_kernel<DT>(columns, d % chunk_elements(dtype) == 0), columns <= 256 ? (rows + 3) / 4 : rows, 256, 0, hs, a);
  }));
  api::note_kernel(columns > NORM_LONG ? "layernorm_forward_long_kernel" : "layernorm_forward_kernel");
  return FLASHDP_OK;
}

size_t flashdp_layernorm_workspace_bytes(int64_t B, int64_t T, int64_t d, int dtype, int bias) {
  if (!valid_dtype(dtype) || check_samples(B, T, d) != FLASHDP_OK) return 0;
  const NormPlan p = norm_plan(B, T, d, dtype);
  return vector_ws(B, p.chunks, bias ? 2 * d : d, p.squares).total;
}

int flashdp_layernorm_dp_grad(const void* X, const void* dY, const void* gamma, const float* mean, const float* rstd, int64_t B, int64_t T, int64_t d,
                              int dtype, float C, float sigma, uint64_t seed, uint32_t layer, void* dX, float* out_grad, float* out_norms, int bias,
                              void* workspace, size_t workspace_bytes, void* stream, int accumulate, int add_noise) {
  if (!X || !dY || !gamma || !mean || !rstd || !valid_dtype(dtype) || (!dX && !out_grad)) return FLASHDP_INVALID_ARGUMENT;
  if (out_grad && !valid_clip(C, sigma)) return FLASHDP_INVALID_ARGUMENT;
  int st = check_samples(B, T, d);
  if (st != FLASHDP_OK) return st;
  if (!aligned(X, 16) || !aligned(dY, 16) || !aligned(gamma, 16) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dX, 16) || !aligned(out_grad, 16) ||
      !aligned(out_norms, 4) || !aligned(workspace, 16))
    return FLASHDP_MISALIGNED;
  const int64_t n = bias ? 2 * d : d;
  const NormPlan p = norm_plan(B, T, d, dtype);
  const VectorWs w = vector_ws(B, p.chunks, n, p.squares);
  if (B * p.chunks * p.col_tiles > GRID_LIMIT || B * w.blocks > GRID_LIMIT || (p.columns > NORM_LONG && B * T > GRID_LIMIT)) return FLASHDP_UNSUPPORTED_SHAPE;
  if (out_grad && workspace && workspace_bytes < w.total) return FLASHDP_WORKSPACE_TOO_SMALL;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (out_grad && !workspace && (st = api::library_workspace(w.total, hs, &workspace)) != FLASHDP_OK) return st;
  char* ws = static_cast<char*>(workspace);
  NormGradArgs a;
  a.X = X; a.dY = dY; a.gamma = gamma; a.mean = mean; a.rstd = rstd; a.dX = dX;
  a.partial = out_grad ? reinterpret_cast<float*>(ws + w.partial) : nullptr;
  a.squares = out_grad ? reinterpret_cast<double*>(ws + w.squares) : nullptr;
  a.B = B; a.T = T; a.d = d; a.chunks = (int)p.chunks; a.rows_per_chunk = (int)p.rows_per_chunk; a.bias = bias ? 1 : 0;
  if (p.columns <= NORM_LONG) {
    const NormGradKernel k = norm_grad_kernel_of(d, dtype, p.token);
    HIP_TRY(launch(k.kernel, p.token ? (B + k.rows - 1) / k.rows : B * p.chunks, k.threads, 0, hs, a));
  } else HIP_TRY(by_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    hipError_t e = hipSuccess;
    if (out_grad) e = launch(layernorm_grad_long_sums_kernel<DT>, B * p.chunks * p.col_tiles, 256, 0, hs, a, (int)p.col_tiles);
    if (e == hipSuccess && dX) e = launch(layernorm_grad_long_rows_kernel<DT>, B * T, 256, 0, hs, a);
    return e;
  }));
  api::note_kernel(p.columns <= NORM_LONG ? "layernorm_grad_kernel" : "layernorm_grad_long_rows_kernel");
  if (!out_grad) return FLASHDP_OK;
  VectorArgs v;
  v.n = n; v.B = B; v.chunks = a.chunks;
  v.C = C; v.noise_scale = add_noise ? sigma * C : 0.0f; v.seed = seed; v.layer = layer; v.field = FLASHDP_FIELD_NORM;
  v.out = out_grad; v.out_norms = out_norms; v.accumulate = accumulate ? 1 : 0;
  HIP_TRY(run_vector(v, ws, w, p.squares != 0, hs));
  return FLASHDP_OK;
}

// Chunks of 16 bytes that whole blocks of 32 features hold, and workgroups that go through them.
static int64_t checkpoint8_chunks(int64_t rows, int64_t d, int dtype) { return rows * checkpoint8_blocks(d) * (CKPT8_BLOCK / chunk_elements(dtype)); }
static int64_t checkpoint8_grid(int64_t chunks) { return (chunks + 255) / 256; }

size_t flashdp_checkpoint8_bytes(int64_t rows, int64_t d) {
  if (check_rows(rows, d) != FLASHDP_OK) return 0;
  return (size_t)(checkpoint8_scales_at(rows, d) + rows * checkpoint8_blocks(d));
}

int flashdp_checkpoint8_pack(const void* X, int64_t rows, int64_t d, int dtype, void* packed, void* stream) {
  if (!X || !packed || !valid_dtype(dtype)) return FLASHDP_INVALID_ARGUMENT;
  int st = check_rows(rows, d);
  if (st != FLASHDP_OK) return st;
  if (!aligned(X, 16) || !aligned(packed, 16)) return FLASHDP_MISALIGNED;
  const int64_t chunks = checkpoint8_chunks(rows, d, dtype);
  if (checkpoint8_grid(chunks) > GRID_LIMIT) return FLASHDP_UNSUPPORTED_SHAPE;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  signed char* q = static_cast<signed char*>(packed);
  unsigned char* scales = static_cast<unsigned char*>(packed) + checkpoint8_scales_at(rows, d);
  HIP_TRY(by_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    return launch(d % CKPT8_BLOCK == 0 ? checkpoint8_pack_kernel<DT, true> : checkpoint8_pack_kernel<DT, false>, checkpoint8_grid(chunks), 256, 0,
                  static_cast<hipStream_t>(stream), X, chunks, d, q, scales);
  }));
  return FLASHDP_OK;
}

int flashdp_checkpoint8_unpack(const void* packed, int64_t rows, int64_t d, int dtype, void* X, void* stream) {
  if (!X || !packed || !valid_dtype(dtype)) return FLASHDP_INVALID_ARGUMENT;
  int st = check_rows(rows, d);
  if (st != FLASHDP_OK) return st;
  if (!aligned(X, 16) || !aligned(packed, 16)) return FLASHDP_MISALIGNED;
  const int64_t chunks = checkpoint8_chunks(rows, d, dtype);
  if (checkpoint8_grid(chunks) > GRID_LIMIT) return FLASHDP_UNSUPPORTED_SHAPE;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  const signed char* q = static_cast<const signed char*>(packed);
  const unsigned char* scales = static_cast<const unsigned char*>(packed) + checkpoint8_scales_at(rows, d);
  HIP_TRY(by_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    return launch(d % CKPT8_BLOCK == 0 ? checkpoint8_unpack_kernel<DT, true> : checkpoint8_unpack_kernel<DT, false>, checkpoint8_grid(chunks), 256, 0,
                  static_cast<hipStream_t>(stream), q, scales, chunks, d, X);
  }));
  return FLASHDP_OK;
}

// Room for the unpacked activation of one layer, in front of the schedule's own workspace.
static size_t unpacked_bytes(const flashdp_layer_t* layers, int n_layers, int64_t B, int64_t T, int dtype) {
  size_t most = 0;
  for (int l = 0; l < n_layers; ++l) most = std::max(most, (size_t)B * T * layers[l].d_in * (dtype == FLASHDP_F32 ? 4 : 2));
  return align_up(most, 256);
}

size_t flashdp_workspace_bytes_checkpoint8(const flashdp_layer_t* layers, int n_layers, int64_t B, int64_t T, int dtype, int schedule) {
  const size_t need = flashdp_workspace_bytes(layers, n_layers, B, T, dtype, api::schedule_of_call(schedule));
  for (int l = 0; need != 0 && l < n_layers; ++l)
    if (check_samples(B, T, layers[l].d_in) != FLASHDP_OK) return 0;
  return need == 0 ? 0 : unpacked_bytes(layers, n_layers, B, T, dtype) + need;
}

int flashdp_block_dp_grad_checkpoint8(const flashdp_layer_t* layers, int n_layers, int64_t B, int64_t T, int dtype, int schedule, void* workspace,
                                      size_t workspace_bytes, void* stream, int accumulate, int add_noise) {
  if (!layers || n_layers <= 0 || !valid_dtype(dtype) || schedule < FLASHDP_SCHEDULE_AUTO || schedule > FLASHDP_SCHEDULE_FUSED) return FLASHDP_INVALID_ARGUMENT;
  // the layers as the ordinary call will see them; it repeats these checks, but after a layer has been unpacked
  for (int l = 0; l < n_layers; ++l) {
    const flashdp_layer_t& L = layers[l];
    if (!L.X || !L.dY || !L.out_grad || !valid_clip(L.C, L.sigma)) return FLASHDP_INVALID_ARGUMENT;
    if (!aligned(L.X, 16) || !aligned(L.dY, 16) || !aligned(L.out_grad, 16) || !aligned(L.out_norms, 4)) return FLASHDP_MISALIGNED;
  }
  if (!aligned(workspace, 16)) return FLASHDP_MISALIGNED;
  if (B <= 0 || T <= 0) return FLASHDP_INVALID_ARGUMENT;
  for (int l = 0; l < n_layers; ++l)
    if (layers[l].d_in <= 0 || layers[l].d_out <= 0) return FLASHDP_INVALID_ARGUMENT;
  for (int l = 0; l < n_layers; ++l)
    if (check_samples(B, T, layers[l].d_in) != FLASHDP_OK || checkpoint8_grid(checkpoint8_chunks(B * T, layers[l].d_in, dtype)) > GRID_LIMIT)
      return FLASHDP_UNSUPPORTED_SHAPE;
  schedule = api::schedule_of_call(schedule);
  const size_t inner = flashdp_workspace_bytes(layers, n_layers, B, T, dtype, schedule);
  if (inner == 0) return FLASHDP_UNSUPPORTED_SHAPE;
  int st = api::check_schedule_sizes(layers, n_layers, B, T, dtype, schedule);
  if (st != FLASHDP_OK) return st;
  const size_t room = unpacked_bytes(layers, n_layers, B, T, dtype);
  if (workspace && workspace_bytes < room + inner) return FLASHDP_WORKSPACE_TOO_SMALL;
  int dev = 0;
  if ((st = api::current_device(&dev)) != FLASHDP_OK) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  // The activation, and the workspace of the ordinary call: what is left of the caller's, or none, so that it takes the library's as it
  // does without checkpoints.
  void* unpacked = workspace;
  if (!workspace && (st = api::library_activation(room, hs, &unpacked)) != FLASHDP_OK) return st;
  void* rest = workspace ? static_cast<char*>(workspace) + room : nullptr;
  const size_t rest_bytes = workspace ? workspace_bytes - room : 0;
  // Layers in a row that share their activation (the projections of an attention block) are unpacked once and go to one call.
  constexpr int RUN = 16;
  for (int l = 0; l < n_layers;) {
    flashdp_layer_t run[RUN];
    int n = 0;
    while (l + n < n_layers && n < RUN && layers[l + n].X == layers[l].X && layers[l + n].d_in == layers[l].d_in) {
      run[n] = layers[l + n];
      run[n].X = unpacked;
      ++n;
    }
    st = flashdp_checkpoint8_unpack(layers[l].X, B * T, layers[l].d_in, dtype, unpacked, stream);
    if (st == FLASHDP_OK)
      st = flashdp_block_dp_grad_micro(run, n, B, T, dtype, schedule, rest, rest_bytes, stream, accumulate, add_noise);
    if (st != FLASHDP_OK) return st;
    l += n;
  }
  return FLASHDP_OK;
}

}  // extern "C"
