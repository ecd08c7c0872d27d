// Affine layers: the weights' layout, the product kernels and their epilogue, and their part of the C ABI.  See
// include/cbd.h for the contract of each call.
#include <cmath>
#include <new>
#include <type_traits>

#include "cbd_host.hpp"
#include "cbd_score.hpp"

using cbd::dmalloc;
using cbd::fail;

namespace cbd {
namespace {

// One application: pointers and strides as in cbd_layer_io, rows counted through (row r = channel r / frames, frame
// r % frames).
struct LayerParams {
  const void *x, *w, *residual;
  const float *bias;
  void *out;
  int64_t x_cs, x_fs, out_cs, out_fs, res_cs, res_fs;
  int32_t rows, frames, K, N;
  int32_t w_blocks, w_steps;   // the packed weights: blocks of 16 outputs, steps of 64 bytes along K
  int32_t act, out_dtype;
  float scale, residual_scale;
  uint32_t frames_mul, frames_shift;   // r / frames = r * frames_mul >> frames_shift for 0 <= r < 2^31
};

__device__ __forceinline__ int channel_of(const LayerParams &p, int r) {
  return (int)((uint64_t)(uint32_t)r * p.frames_mul >> p.frames_shift);
}

typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
// 16 bytes at any element's address: global loads and stores of this size need no more alignment than that.
typedef uint32_t uint4u __attribute__((ext_vector_type(4), aligned(2)));

// A fragment is 16 bytes a lane: lane l holds row l % 16 and the (l / 16)-th 16-byte piece of a step of 64 bytes along K
// (32 halves or 16 floats).  Both operands of a product use the same assignment of k to lanes, so the sum over the step
// is complete whatever the order within it.
template <typename T> struct Mma;   // kParts instructions make a step's product; part q of the pair a, b added to c
template <> struct Mma<bf16> {
  static constexpr int kParts = 1;
  typedef bf16 V __attribute__((ext_vector_type(8)));
  __device__ static float4v run(int, uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
};
template <> struct Mma<f16> {
  static constexpr int kParts = 1;
  typedef f16 V __attribute__((ext_vector_type(8)));
  __device__ static float4v run(int, uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
};
template <> struct Mma<float> {
  static constexpr int kParts = 4;
  __device__ static float4v run(int q, uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[q]), __uint_as_float(b[q]), c, 0, 0, 0);
  }
};

// exp by the hardware's base-2 exponential: relative error at most (1.25 |y| + 2) 2^-24.
__device__ __forceinline__ float fast_exp(float y) { return __builtin_amdgcn_exp2f(y * 1.44269504088896341f); }
__device__ __forceinline__ float fast_rcp(float y) { return __builtin_amdgcn_rcpf(y); }   // (1 unit in the last place)

__device__ __forceinline__ float activate(int act, float y) {
  switch (act) {
    case CBD_ACT_RELU: return y < 0.0f ? 0.0f : y;   // (NaN stays)
    case CBD_ACT_SIGMOID: return fast_rcp(1.0f + fast_exp(-y));
    case CBD_ACT_TANH: {
      // Near zero y + y^3 P(y^2), P fitted to a relative 3e-9 of the result up to |y| = 0.6; beyond, 1 - 2e / (1 + e) with
      // e = exp(-2|y|), whose last term, the only one with errors of its own, is below the result there.
      const float q = y * y;
      float near = fmaf(-0.00589513965f, q, 0.0207959544f);
      near = fmaf(near, q, -0.0537838265f);
      near = fmaf(near, q, 0.133319244f);
      near = fmaf(near, q, -0.333332986f);
      near = fmaf(y * q, near, y);
      const float e = __builtin_amdgcn_exp2f(fabsf(y) * -2.88539008177792681f);
      const float far = copysignf(fmaf(-2.0f * e, fast_rcp(1.0f + e), 1.0f), y);
      return fabsf(y) < 0.6f ? near : far;
    }
    case CBD_ACT_GELU: {
      // y Phi(y).  The tail Phi(-m), m = |y|, is exp(-m^2 / 2) g(m), and g falls from 1/2 like 1 / m: it is t = 1 / (1 + 0.3 m)
      // times a polynomial in t, fitted to a relative 1.2e-7 for m up to 13 (the tail leaves fp32's range there).  What
      // rounding takes from m^2 and from the exponent is put back in first order, or it would count some 50 times.  (12800 x
      // 1024 -> 4096 in bf16 129 us; with silu 107, with tanh 118.)
      const float m = fminf(fabsf(y), 16.0f), t = fast_rcp(fmaf(0.3f, m, 1.0f));
      float g = fmaf(0.0360896401f, t, -0.158936828f);
      g = fmaf(g, t, 0.209351301f);
      g = fmaf(g, t, -0.0564542599f);
      g = fmaf(g, t, 0.13003464f);
      g = fmaf(g, t, 0.0994645059f);
      g = fmaf(g, t, 0.120826401f);
      g = fmaf(g, t, 0.11962454f);
      constexpr float kLog = -0.72134752044448170f, kLogRest = (float)(-0.72134752044448170 - (double)kLog);   // -log2(e) / 2
      const float h = m * m, a = h * kLog;
      float rest = fmaf(h, kLog, -a);
      rest = fmaf(fmaf(m, m, -h), kLog, rest);
      rest = fmaf(h, kLogRest, rest);
      const float e = __builtin_amdgcn_exp2f(a), tail = g * t * fmaf(e * 0.693147180559945309f, rest, e);
      return y * (y < 0.0f ? tail : 1.0f - tail);
    }
    case CBD_ACT_SILU: return y * fast_rcp(1.0f + fast_exp(-y));
    default: return y;
  }
}

typedef float float8v __attribute__((ext_vector_type(8)));

template <int kAct, int n> __device__ __forceinline__ void activate_all(float (&v)[n]) {
#pragma unroll
  for (int j = 0; j < n; ++j) v[j] = activate(kAct, v[j]);
}

template <int n> __device__ __forceinline__ void activate_by(int act, float (&v)[n]) {
  switch (act) {   // (the same for all lanes)
    case CBD_ACT_RELU: activate_all<CBD_ACT_RELU>(v); break;
    case CBD_ACT_SIGMOID: activate_all<CBD_ACT_SIGMOID>(v); break;
    case CBD_ACT_TANH: activate_all<CBD_ACT_TANH>(v); break;
    case CBD_ACT_GELU: activate_all<CBD_ACT_GELU>(v); break;
    case CBD_ACT_SILU: activate_all<CBD_ACT_SILU>(v); break;
    default: break;
  }
}

// The layer's epilogue on neighbouring sums of one row: bias, activation, scale.
template <bool kActivation, int n> __device__ __forceinline__ void finish(const LayerParams &p, float (&v)[n], const float (&bias)[n]) {
#pragma unroll
  for (int j = 0; j < n; ++j) v[j] += bias[j];
  if (kActivation) activate_by(p.act, v);
#pragma unroll
  for (int j = 0; j < n; ++j) v[j] *= p.scale;
}

template <int n> __device__ __forceinline__ void load_bias(const LayerParams &p, int at, float (&bias)[n]) {
#pragma unroll
  for (int j = 0; j < n; ++j) bias[j] = p.bias && at + j < p.N ? p.bias[at + j] : 0.0f;
}

// Outputs `at` .. at + n - 1 of a row: the residual added, one rounding to the output's type, stored.  A row's end inside
// them is stored element by element.
template <typename O, int n> __device__ __forceinline__ void store_as(const LayerParams &p, int64_t out_row, int64_t res_row, int at, float (&v)[n]) {
  O *out = (O *)p.out + out_row + at;
  const O *res = p.residual ? (const O *)p.residual + res_row + at : nullptr;
  struct __attribute__((aligned(sizeof(O)))) Some { O v[n]; };   // (vector loads and stores need no more alignment)
  if (at + n <= p.N) {
    if (res) {
      const Some r = *(const Some *)res;
#pragma unroll
      for (int j = 0; j < n; ++j) v[j] += p.residual_scale * (float)r.v[j];
    }
    Some o;
#pragma unroll
    for (int j = 0; j < n; ++j) o.v[j] = (O)v[j];
    *(Some *)out = o;
    return;
  }
#pragma unroll
  for (int j = 0; j < n; ++j) {
    if (at + j < p.N) {
      float y = v[j];
      if (res) y += p.residual_scale * (float)res[j];
      out[j] = (O)y;
    }
  }
}

template <int n> __device__ __forceinline__ void store(const LayerParams &p, int64_t out_row, int64_t res_row, int at, float (&v)[n]) {
  if (at >= p.N) return;
  if (p.out_dtype == CBD_F32) store_as<float>(p, out_row, res_row, at, v);
  else if (p.out_dtype == CBD_F16) store_as<f16>(p, out_row, res_row, at, v);
  else store_as<bf16>(p, out_row, res_row, at, v);
}

// Eight neighbouring outputs of a row that lie within it, from sums with bias, activation and scale done.
template <typename O, bool kResidual> __device__ __forceinline__ void store_whole(const LayerParams &p, int64_t out_row, int64_t res_row, int at, float8v v) {
  typedef O V8 __attribute__((ext_vector_type(8)));
  typedef O V8u __attribute__((ext_vector_type(8), aligned(sizeof(O))));   // (vector accesses need no more alignment)
  if (kResidual) {
    const V8 r = *(const V8u *)((const O *)p.residual + res_row + at);
    v += p.residual_scale * __builtin_convertvector(r, float8v);
  }
  if (sizeof(O) == 4) {
    // fp32: a lane's eight outputs are two stores.  The four lanes of a row first exchange halves, so that each store
    // fills 64 bytes of the row instead of every other 16 (output layer of 12800 rows, 1024 -> 6000: 181 -> 173 us).
    float4v lo, hi;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[q]), __float_as_uint(v[q + 4]), false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(a[0], a[1], false, false);
      lo[q] = __uint_as_float(b[0]);
      hi[q] = __uint_as_float(b[1]);
    }
    typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
    const int g = (threadIdx.x >> 4) & 3;
    float *out = (float *)p.out + out_row + at - g * 4;
    *(float4u *)out = lo;
    *(float4u *)(out + 16) = hi;
    return;
  }
  *(V8u *)((O *)p.out + out_row + at) = __builtin_convertvector(v, V8);   // (the one rounding to the output's type)
}

// The end of a tile kernel: a wave's FM x FN blocks of sums become outputs.  With the packed weights' order of outputs a
// lane holds, of row lane % 16 of each row block, eight neighbouring outputs per pair of blocks, and the four lanes of a
// row 32: one 16-byte store (two for fp32) a lane fills 64 bytes of a row.
//
// A tile that lies within the rows and outputs: code for each row block.  A loop over them would be an eighth of it, but no
// running index reaches registers, and what picks a block's sums in their place spilled a third of those of 128 x 256 tiles:
// 12800 x 1024 -> 4096 with silu and residual 165 us, so 121.
template <typename O, bool kResidual, bool kActivation, int FM, int FN>
__device__ __forceinline__ void finish_whole(const LayerParams &p, float4v (&acc)[FM][FN], const longlong2 *rows_at, int n, int lane) {
  float bias[FN / 2][8];
#pragma unroll
  for (int j = 0; j < FN / 2; ++j) load_bias(p, n + j * 32, bias[j]);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    float v[FN * 4];
#pragma unroll
    for (int j = 0; j < FN * 4; ++j) v[j] = acc[i][j / 4][j % 4] + bias[j / 8][j % 8];
    if (kActivation) activate_by(p.act, v);
    const longlong2 at = rows_at[i * 16 + (lane & 15)];
#pragma unroll
    for (int j = 0; j < FN / 2; ++j) {
      float8v y;
#pragma unroll
      for (int q = 0; q < 8; ++q) y[q] = v[j * 8 + q] * p.scale;
      store_whole<O, kResidual>(p, at.x, at.y, n + j * 32, y);
    }
  }
}

template <typename O, bool kActivation, int FM, int FN>
__device__ __forceinline__ void finish_tile(const LayerParams &p, float4v (&acc)[FM][FN], const longlong2 *rows_at, int n0, int lane, bool whole) {
  const int n = n0 + (lane >> 4) * 8;
  if (whole) {
    if (p.residual) finish_whole<O, true, kActivation, FM, FN>(p, acc, rows_at, n, lane);
    else finish_whole<O, false, kActivation, FM, FN>(p, acc, rows_at, n, lane);
    return;
  }
  float bias[FN / 2][8];
#pragma unroll
  for (int j = 0; j < FN / 2; ++j) load_bias(p, n + j * 32, bias[j]);
#pragma unroll 1
  for (int i = 0; i < FM; ++i) {
    float v[FN / 2][8];
#pragma unroll
    for (int k = 0; k < FM; ++k)
      if (k == i) {
#pragma unroll
        for (int j = 0; j < FN * 4; ++j) v[j / 8][j % 8] = acc[k][j / 4][j % 4];
      }
    const longlong2 at = rows_at[i * 16 + (lane & 15)];   // (negative: beyond the last row)
    if (at.x >= 0) {
#pragma unroll
      for (int j = 0; j < FN / 2; ++j) {
        finish<kActivation>(p, v[j], bias[j]);
        if (n + j * 32 < p.N) store_as<O>(p, at.x, at.y, n + j * 32, v[j]);
      }
    }
  }
}

// Where the rows of a tile are in output and residual (elements), or a negative number beyond the last row.
__device__ __forceinline__ void place_rows(const LayerParams &p, int row0, int count, longlong2 *rows_at) {
  for (int i = threadIdx.x; i < count; i += blockDim.x) {
    const int r = row0 + i;
    longlong2 at = {-1, -1};
    if (r < p.rows) {
      const int c = channel_of(p, r), f = r - c * p.frames;
      at.x = c * p.out_cs + f * p.out_fs;
      at.y = c * p.res_cs + f * p.res_fs;
    }
    rows_at[i] = at;
  }
}

// The tile of a workgroup.  Consecutive workgroups go to the chip's eight dies in turn: each die gets a contiguous run of
// tiles, and the tiles of a run share weights and rows (eight row tiles below each other, then the next outputs).
__device__ __forceinline__ void place_tile(int b, int tiles_m, int tiles_n, int *tile_m, int *tile_n) {
  const int total = tiles_m * tiles_n, die = b & 7, q = total >> 3, rest = total & 7;
  int t = die * q + min(die, rest) + (b >> 3);
  constexpr int kGroup = 8;
  const int group = t / (kGroup * tiles_n), first = group * kGroup, height = min(kGroup, tiles_m - first);
  t -= group * kGroup * tiles_n;
  *tile_m = first + t % height;
  *tile_n = t / height;
}

// 16 bytes of an input row from element k on; beyond K there are zeros (and no reads).
template <typename T> __device__ __forceinline__ uint4v load_piece(const T *row, int k, int K) {
  constexpr int kElems = 16 / sizeof(T);
  if (k + kElems <= K) {
    const uint4u v = *(const uint4u *)(row + k);
    return v;
  }
  T e[kElems];
#pragma unroll
  for (int j = 0; j < kElems; ++j) e[j] = k + j < K ? row[k + j] : (T)0.0f;
  return __builtin_bit_cast(uint4v, e);
}

// Weights, packed once: block b of 16 outputs, step s: 64 lanes x 16 bytes in fragment order, so that a wave loads a
// fragment as one contiguous kilobyte.  Zeros beyond N and K.  Two blocks share 32 outputs so that the sums of four
// neighbouring rows of the first and of the second, which one lane holds, belong to eight neighbouring outputs: row q of
// block b is output packed_output(b, q).
__host__ __device__ __forceinline__ int packed_output(int b, int q) { return (b >> 1) * 32 + (q >> 2) * 8 + (b & 1) * 4 + (q & 3); }

template <typename T> __global__ __launch_bounds__(256) void pack_weight_kernel(const T *src, int64_t stride, uint4v *dst, int32_t K,
                                                                                 int32_t N, int32_t steps, int64_t total) {
  constexpr int kElems = 16 / sizeof(T);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;   // (block, step, lane)
  if (i >= total) return;
  const int lane = (int)(i & 63);
  const int64_t bs = i >> 6;
  const int n = packed_output((int)(bs / steps), lane & 15), k = (int)(bs % steps) * 4 * kElems + (lane >> 4) * kElems;
  uint4v v = {0u, 0u, 0u, 0u};
  if (n < N) v = load_piece<T>(src + (int64_t)n * stride, k, K);
  dst[i] = v;
}

// Tiles.  A workgroup of WM x WN waves makes (WM * FM * 16) rows x (WN * FN * 16) outputs; a wave FM x FN blocks of 16 x
// 16.  Input rows go through LDS, 128 bytes of K at a time, two buffers; weights come straight from the packed layout
// into registers, one such step ahead: no two waves of a workgroup read the same weights, so LDS would only delay them,
// and its bandwidth is left to the rows.  Measured (12800 rows): 1024 -> 6000 in bf16 to fp32 177 us, 1024 -> 4096 with
// silu 108 us (885 and 995 TFLOP/s; the matrix units are busy half of the cycles: the stores of a tile's results and its
// first loads are not covered by products), fp32 1600 x 512 -> 3000 49.5 us (99 TFLOP/s, busy 73 %: the last of 1200 tiles).
template <typename T, typename O, bool kActivation, int WM, int WN, int FM, int FN>
__global__ __launch_bounds__(64 * WM * WN, 2) void tile_kernel(LayerParams p, int first_m, int tiles_m, int tiles_n) {
  constexpr int kThreads = 64 * WM * WN, BM = WM * FM * 16, kElems = 16 / sizeof(T), kTileK = 8 * kElems;
  constexpr int kPieces = BM * 8 / kThreads;   // 16-byte pieces of a K tile per thread
  __shared__ uint4v lds[2][BM * 8];
  __shared__ longlong2 rows_at[BM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  int tile_m, tile_n;
  place_tile(blockIdx.x, tiles_m, tiles_n, &tile_m, &tile_n);
  tile_m += first_m;   // (the launch's first row of tiles)
  place_rows(p, tile_m * BM, BM, rows_at);
  // this thread's pieces of the input: rows tid / 8 + i * (threads / 8), piece tid % 8 of each K tile
  const T *src[kPieces];
  int dst[kPieces];
  const int piece = tid & 7;
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int row = (tid >> 3) + i * (kThreads / 8);
    const int r = min(tile_m * BM + row, p.rows - 1);   // (rows beyond the last repeat it and are not stored)
    const int c = channel_of(p, r), f = r - c * p.frames;
    src[i] = (const T *)p.x + c * p.x_cs + f * p.x_fs;
    dst[i] = row * 8 + (piece ^ (row & 7));   // (pieces of a row swapped by row: reads of 16 rows spread over all banks)
  }
  // (wave and block numbers are the same in all lanes: their addresses are kept in scalar registers)
  const uint4v *w[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int block = min((tile_n * WN + wn) * FN + j, p.w_blocks - 1);   // (blocks beyond the last repeat it)
    w[j] = (const uint4v *)p.w + (int64_t)block * p.w_steps * 64;
  }
  float4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  // A K tile is worked off in four groups: two steps of K, each in two halves of the row blocks.  While the products of a
  // group run, the next group's rows are on their way from LDS; a step's weights are replaced by the next tile's as soon
  // as its last product is issued; the next tile's rows wait in registers and go to the other LDS buffer ahead of the
  // barrier, behind which the last group's products cover the first reads.
  constexpr int G = FM / 2;
  uint4v stage[kPieces], wv[2][FN], xa[G], xb[G];
  const int x_at = (wm * FM * 16 + (lane & 15)) * 8, swap = lane & 7;   // (16-row blocks start at multiples of 8 rows)
  auto read_group = [&](int t, int g, uint4v *x) {
    const uint4v *buf = lds[t & 1] + x_at + (((g >> 1) * 4 + (lane >> 4)) ^ swap);
#pragma unroll
    for (int i = 0; i < G; ++i) x[i] = buf[((g & 1) * G + i) * 128];
  };
  auto load_weights = [&](int t, int step) {
#pragma unroll
    for (int j = 0; j < FN; ++j) wv[step][j] = w[j][(t * 2 + step) * 64 + lane];
  };
  auto products = [&](int g, const uint4v *x) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < Mma<T>::kParts; ++q)   // (outermost: neighbouring products go to different sums)
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[(g & 1) * G + i][j] = Mma<T>::run(q, wv[g >> 1][j], x[i], acc[(g & 1) * G + i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto write_stage = [&](int t) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) lds[t & 1][dst[i]] = stage[i];
  };
  auto load_whole = [&](int t) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) { const uint4u v = *(const uint4u *)(src[i] + t * kTileK + piece * kElems); stage[i] = v; }
  };
  auto load_end = [&](int t) {   // (the last tile may reach beyond K)
#pragma unroll
    for (int i = 0; i < kPieces; ++i) stage[i] = load_piece<T>(src[i], t * kTileK + piece * kElems, p.K);
  };
  const int n_tiles = p.w_steps / 2;
  auto tile = [&](int t, auto next) {   // next: 0 = a whole tile follows, 1 = the last one follows, 2 = none
    constexpr bool more = decltype(next)::value < 2;
    if constexpr (decltype(next)::value == 0) load_whole(t + 1);
    if constexpr (decltype(next)::value == 1) load_end(t + 1);
    read_group(t, 1, xb);
    products(0, xa);
    read_group(t, 2, xa);
    products(1, xb);
    if constexpr (more) load_weights(t + 1, 0);
    read_group(t, 3, xb);
    products(2, xa);
    if constexpr (more) {
      write_stage(t + 1);
      __syncthreads();
      read_group(t + 1, 0, xa);
    }
    products(3, xb);
    if constexpr (more) load_weights(t + 1, 1);
  };
  load_end(0);
  load_weights(0, 0);
  load_weights(0, 1);
  write_stage(0);
  __syncthreads();
  read_group(0, 0, xa);
  int t = 0;
  for (; t < n_tiles - 2; ++t) tile(t, std::integral_constant<int, 0>());
  if (n_tiles > 1) tile(t++, std::integral_constant<int, 1>());
  tile(t, std::integral_constant<int, 2>());
  finish_tile<O, kActivation>(p, acc, rows_at + wm * FM * 16, (tile_n * WN + wn) * FN * 16, lane,
                      (tile_m + 1) * BM <= p.rows && (tile_n + 1) * WN * FN * 16 <= p.N);
}

// Few outputs in all: a workgroup makes (FM * 16) rows x (FN * 16) outputs, its waves share K (wave w takes groups of
// kAhead steps w, w + kWaves, ...) and add their sums up in LDS, in the order of the waves.  Operands are used FM or FN
// times by one wave only, so both come straight from memory, kAhead steps in flight (two with 32 x 32: fp32 500 x 2048 ->
// 500 15.4 us, with four 18.1: half the registers, twice the workgroups on a compute unit).  Bound by the latency of its
// few loads: 1 x 1024 -> 6000 in bf16 5.1 us (12.3 MB, 2.4 TB/s), 32 x 2048 -> 512 5.5 us, a fill of one number 3.4.
constexpr int kNarrowWaves = 8;
template <typename T, int FM, int FN, int kAhead> __global__ __launch_bounds__(64 * kNarrowWaves) void narrow_kernel(LayerParams p) {
  constexpr int kElems = 16 / sizeof(T), kStep = 4 * kElems;
  __shared__ float4v sums[kNarrowWaves][FM][FN][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T *src[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int r = min((int)(blockIdx.y * FM + i) * 16 + (lane & 15), p.rows - 1);
    const int c = channel_of(p, r), f = r - c * p.frames;
    src[i] = (const T *)p.x + c * p.x_cs + f * p.x_fs + (lane >> 4) * kElems;
  }
  const uint4v *w[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j)   // (a block beyond the last repeats it and is not stored)
    w[j] = (const uint4v *)p.w + (int64_t)min((int)blockIdx.x * FN + j, p.w_blocks - 1) * p.w_steps * 64 + lane;
  float4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = wave * kAhead; s0 < p.w_steps; s0 += kNarrowWaves * kAhead) {
    uint4v wv[kAhead][FN], xv[kAhead][FM];
    if (s0 + kAhead <= p.w_steps && (s0 + kAhead) * kStep <= p.K) {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
#pragma unroll
        for (int j = 0; j < FN; ++j) wv[a][j] = w[j][(int64_t)(s0 + a) * 64];
#pragma unroll
        for (int i = 0; i < FM; ++i) { const uint4u v = *(const uint4u *)(src[i] + (s0 + a) * kStep); xv[a][i] = v; }
      }
    } else {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int s = min(s0 + a, p.w_steps - 1);
#pragma unroll
        for (int j = 0; j < FN; ++j) wv[a][j] = s0 + a < p.w_steps ? w[j][(int64_t)s * 64] : uint4v{0u, 0u, 0u, 0u};
        // (a step beyond the last counts as one beyond K: zeros on both sides, as zero times an infinite weight is NaN)
        const int k = (s0 + a) * kStep;
#pragma unroll
        for (int i = 0; i < FM; ++i) xv[a][i] = load_piece<T>(src[i], k, p.K - (lane >> 4) * kElems);
      }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
#pragma unroll
      for (int q = 0; q < Mma<T>::kParts; ++q)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = Mma<T>::run(q, wv[a][j], xv[a][i], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) sums[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  // a wave finishes a block: lane l has row l % 16 and the four outputs of the block's rows 4 (l / 16) ..
  for (int at = wave; at < FM * FN; at += kNarrowWaves) {
    const int i = at / FN, j = at % FN;
    float4v v = sums[0][i][j][lane];
#pragma unroll
    for (int k = 1; k < kNarrowWaves; ++k) v += sums[k][i][j][lane];
    const int r = (int)(blockIdx.y * FM + i) * 16 + (lane & 15), n = packed_output((int)blockIdx.x * FN + j, (lane >> 4) * 4);
    if (r >= p.rows) continue;
    const int c = channel_of(p, r), f = r - c * p.frames;
    float y[4] = {v[0], v[1], v[2], v[3]}, bias[4];
    load_bias(p, n, bias);
    finish<true>(p, y, bias);
    store(p, c * p.out_cs + f * p.out_fs, c * p.res_cs + f * p.res_fs, n, y);
  }
}

}  // namespace
}  // namespace cbd

struct cbd_layer {
  int device = 0;
  int32_t K = 0, N = 0, dtype = 0, act = 0;
  int32_t blocks = 0, steps = 0;   // of the packed weights
  void *w = nullptr;
  float *bias = nullptr;
};

namespace {

using cbd::LayerParams;

// calls f(O(), std::bool_constant<activation>()) for the output's type and whether there is an activation
template <typename F> void with_output(const LayerParams &p, F f) {
  auto with_type = [&](auto o) {
    if (p.act == CBD_ACT_NONE) f(o, std::false_type());
    else f(o, std::true_type());
  };
  if (p.out_dtype == CBD_F32) with_type(0.0f);
  else if (p.out_dtype == CBD_F16) with_type((cbd::f16)0.0f);
  else with_type((cbd::bf16)0.0f);
}

template <typename T, int WM, int WN, int FM, int FN> hipError_t launch_tiles(const LayerParams &p, hipStream_t st) {
  const int tiles_m = (p.rows + WM * FM * 16 - 1) / (WM * FM * 16), tiles_n = (p.N + WN * FN * 16 - 1) / (WN * FN * 16);
  const int most = (int)(0xFFFFFFFFll / (64 * WM * WN) / tiles_n);   // rows of tiles in a launch, which has fewer than 2^32 threads
  for (int first = 0; first < tiles_m; first += most) {
    const int n = std::min(most, tiles_m - first);
    with_output(p, [&](auto o, auto act) {
      hipLaunchKernelGGL((cbd::tile_kernel<T, decltype(o), decltype(act)::value, WM, WN, FM, FN>), dim3((unsigned)n * (unsigned)tiles_n),
                         dim3(64 * WM * WN), 0, st, p, first, n, tiles_n);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int FM, int FN, int kAhead> hipError_t launch_narrow(const LayerParams &p, hipStream_t st) {
  auto kernel = cbd::narrow_kernel<T, FM, FN, kAhead>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((p.w_blocks + FN - 1) / FN), (unsigned)((p.rows + FM * 16 - 1) / (FM * 16))),
                     dim3(64 * cbd::kNarrowWaves), 0, st, p);
  return hipGetLastError();
}

int64_t tiles_of(const LayerParams &p, int rows, int outputs) {
  return (int64_t)((p.rows + rows - 1) / rows) * ((p.N + outputs - 1) / outputs);
}

// A kernel's share of the choice: the time of a launch is close to K * (first + more * (n / 256 - 1)) ns for n > 256
// workgroups of `rows` x `outputs`, and K * first ns up to then (256 compute units; above, they overlap or queue).
struct Choice {
  int rows, outputs;
  float first, more;
  float cost(const LayerParams &p) const {
    if (outputs <= 64 && (p.rows - 1) / rows >= 65535) return 1e30f;   // (waves that share K: row blocks are the grid's second dimension)
    const float n = (float)tiles_of(p, rows, outputs) / 256.0f;
    return n <= 1.0f ? first : first + more * (n - 1.0f);
  }
};

// Which kernel.  Large tiles read less per product, small ones and those whose waves share K leave fewer compute units
// without work; which counts more follows from the number of workgroups alone, as all kernels' times grow with K.  The
// figures were fitted to 20 to 100,000 rows, 64 to 4096 inputs, 256 to 100,000 outputs; the choice is within 6 % of the best
// of all on average.  us for 16 x 16 / 32 x 32 / 32 x 64 by waves that share K, and tiles of 32 x 128 / 64 x 128:
//   bf16   64 x 1024 -> 1024    4.0 /  4.9 /  5.7 /  6.9 /  8.6      fp32   64 x 1024 -> 1024    5.0 /  8.7 /  -  / 23.6 / 38.3
//   bf16  231 x  771 -> 1021   10.7 /  7.4 /  7.8 /  7.3 /  9.3      fp32  500 x 2048 ->  500   22.4 / 15.4 /  -  / 43.9 / 73.4
//   bf16 1000 x 4096 ->  256   19.2 / 12.5 / 15.0 / 18.7 / 24.3      fp32  336 x 1272 -> 3653   66.1 / 49.0 /  -  / 49.4 / 55.3
//   bf16 2000 x 1024 -> 4000    140 /  77  /  80  / 32.8 / 25.0      fp32 1600 x  512 -> 3000   86.3 / 63.1 /  -  / 49.3 / 55.8
// (fp32: products take 16 times the time of bf16 ones, so that spreading them counts for more than reads.)
// Chip-filling 16-bit products with more than a few steps of K take larger tiles:
//   64 x 256 from 1000 tiles of 64 x 128  (1600 x 1024 -> 6000: 29.6; 64 x 128 32.9; but 6400 x 512 -> 2000: 26.3 and 24.1)
//   128 x 256 from 512 of its own tiles   (16384 x 1024 -> 4096: 144; 64 x 256 157)
template <typename T> hipError_t launch(const LayerParams &p, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (tiles_of(p, 64, 128) >= 1000 && p.K > 512)
      return tiles_of(p, 128, 256) < 512 ? launch_tiles<T, 1, 4, 4, 4>(p, st) : launch_tiles<T, 1, 4, 8, 4>(p, st);
    const Choice choices[] = {{16, 16, 0.55f, 1.1f}, {32, 32, 1.5f, 2.5f}, {32, 64, 2.0f, 3.8f}, {32, 128, 3.5f, 4.6f}, {64, 128, 5.2f, 8.1f}};
    int best = 0;
    for (int i = 1; i < 5; ++i)
      if (choices[i].cost(p) < choices[best].cost(p)) best = i;
    switch (best) {
      case 0: return launch_narrow<T, 1, 1, 4>(p, st);
      case 1: return launch_narrow<T, 2, 2, 2>(p, st);
      case 2: return launch_narrow<T, 2, 4, 2>(p, st);
      case 3: return launch_tiles<T, 1, 4, 2, 2>(p, st);
      default: return launch_tiles<T, 1, 4, 4, 2>(p, st);
    }
  } else {
    const Choice choices[] = {{16, 16, 1.9f, 2.5f}, {32, 32, 4.7f, 8.1f}, {32, 128, 21.0f, 27.0f}};
    int best = 0;
    for (int i = 1; i < 3; ++i)
      if (choices[i].cost(p) < choices[best].cost(p)) best = i;
    switch (best) {
      case 0: return launch_narrow<T, 1, 1, 4>(p, st);
      case 1: return launch_narrow<T, 2, 2, 2>(p, st);
      default: return launch_tiles<T, 1, 4, 2, 2>(p, st);
    }
  }
}

bool aligned(const void *ptr, int32_t dtype) { return ((uintptr_t)ptr & (cbd::dtype_size(dtype) - 1)) == 0; }

// Do rows of `width` elements at i * cs + f * fs (i < n, f < m) lie apart, channels outermost or frames outermost?
bool rows_apart(int64_t n, int64_t m, int64_t cs, int64_t fs, int64_t width) {
  if (n <= 1 && m <= 1) return true;
  if (n <= 1) return fs >= width;
  if (m <= 1) return cs >= width;
  const bool by_channel = fs >= width && (cs - width) / (m - 1) >= fs && cs >= width;
  const bool by_frame = cs >= width && (fs - width) / (n - 1) >= cs && fs >= width;
  return by_channel || by_frame;
}

// May the furthest row's address be computed in 64 bits?
bool strides_fit(int64_t n, int64_t m, int64_t cs, int64_t fs) {
  const int64_t top = (int64_t)1 << 60;
  return cs >= 0 && fs >= 0 && (n <= 1 || cs <= top / n) && (m <= 1 || fs <= top / m);
}

}  // namespace

extern "C" {

int32_t cbd_layer_create(const cbd_layer_desc *desc, void *hip_stream, cbd_layer **out) try {
  if (!desc || !out) return fail(CBD_E_INVALID, "layer: null argument");
  if (desc->in_features < 1 || desc->in_features > 65536) return fail(CBD_E_INVALID, "layer: in_features must be in [1, 65536]");
  if (desc->out_features < 1 || desc->out_features > 1048576)
    return fail(CBD_E_INVALID, "layer: out_features must be in [1, 1048576]");
  if (desc->dtype < CBD_F32 || desc->dtype > CBD_BF16) return fail(CBD_E_INVALID, "layer: dtype");
  if (desc->activation < CBD_ACT_NONE || desc->activation > CBD_ACT_SILU) return fail(CBD_E_INVALID, "layer: activation");
  if (!desc->weight) return fail(CBD_E_INVALID, "layer: null weight");
  const int64_t stride = desc->weight_stride ? desc->weight_stride : desc->in_features;
  if (stride < desc->in_features || stride > (int64_t)1 << 40) return fail(CBD_E_INVALID, "layer: weight_stride");
  if (!aligned(desc->weight, desc->dtype) || !aligned(desc->bias, CBD_F32))
    return fail(CBD_E_INVALID, "layer: weight or bias not aligned to its elements");
  const int32_t step = 64 / (int32_t)cbd::dtype_size(desc->dtype);
  const int32_t blocks = (desc->out_features + 31) / 32 * 2;
  const int32_t steps = (desc->in_features + 2 * step - 1) / (2 * step) * 2;   // (tiles take two steps at a time)
  const int64_t total = (int64_t)blocks * steps * 64;   // 16-byte pieces, one per thread of a launch
  if (total > 0xFFFFFF00ll) return fail(CBD_E_INVALID, "layer: more than 64 GB of weights");
  hipStream_t st = (hipStream_t)hip_stream;
  int device = 0;
  HIPCHK(hipGetDevice(&device));
  if (!cbd::stream_is_of(st, device)) return fail(CBD_E_INVALID, "layer: the stream belongs to another device");
  if (cbd::is_capturing(st)) return fail(CBD_E_INVALID, "layer: the stream is being captured");
  cbd_layer *l = new (std::nothrow) cbd_layer();
  if (!l) return fail(CBD_E_NOMEM, "layer: host allocation");
  struct Guard {   // frees the half-built layer on every early return
    cbd_layer *l;
    ~Guard() { if (l) cbd_layer_free(l); }
  } guard{l};
  l->device = device;
  l->K = desc->in_features; l->N = desc->out_features; l->dtype = desc->dtype; l->act = desc->activation;
  l->blocks = blocks; l->steps = steps;
  HIPCHK(dmalloc((char **)&l->w, (size_t)total * 16, nullptr));
  const dim3 grid((unsigned)((total + 255) / 256));
  cbd::uint4v *w = (cbd::uint4v *)l->w;
  if (l->dtype == CBD_F32)
    hipLaunchKernelGGL(cbd::pack_weight_kernel<float>, grid, dim3(256), 0, st, (const float *)desc->weight, stride, w, l->K, l->N, l->steps, total);
  else if (l->dtype == CBD_F16)
    hipLaunchKernelGGL(cbd::pack_weight_kernel<cbd::f16>, grid, dim3(256), 0, st, (const cbd::f16 *)desc->weight, stride, w, l->K, l->N, l->steps, total);
  else
    hipLaunchKernelGGL(cbd::pack_weight_kernel<cbd::bf16>, grid, dim3(256), 0, st, (const cbd::bf16 *)desc->weight, stride, w, l->K, l->N, l->steps, total);
  HIPCHK(hipGetLastError());
  if (desc->bias) {
    HIPCHK(dmalloc(&l->bias, (size_t)l->N, nullptr));
    HIPCHK(hipMemcpyAsync(l->bias, desc->bias, sizeof(float) * (size_t)l->N, hipMemcpyDeviceToDevice, st));
  }
  HIPCHK(hipStreamSynchronize(st));
  *out = l;
  guard.l = nullptr;
  return CBD_OK;
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("layer_create: ") + e.what());
}

int32_t cbd_layer_free(cbd_layer *l) {
  if (!l) return CBD_OK;
  if (l->w) (void)hipFree(l->w);
  if (l->bias) (void)hipFree(l->bias);
  delete l;
  return CBD_OK;
}

int32_t cbd_layer_apply(const cbd_layer *l, const cbd_layer_io *io, void *hip_stream) try {
  if (!l || !io) return fail(CBD_E_INVALID, "layer_apply: null argument");
  if (io->n_channels < 0 || io->n_frames < 0) return fail(CBD_E_INVALID, "layer_apply: negative size");
  if (io->output_dtype < CBD_F32 || io->output_dtype > CBD_BF16) return fail(CBD_E_INVALID, "layer_apply: output_dtype");
  if (!std::isfinite(io->scale) || (io->residual && !std::isfinite(io->residual_scale)))
    return fail(CBD_E_INVALID, "layer_apply: scales must be finite");
  const int64_t n = io->n_channels, m = io->n_frames, rows = n * m;
  if (rows == 0) return CBD_OK;
  if (rows > (1 << 29) - 256) return fail(CBD_E_INVALID, "layer_apply: too many rows");
  if (!io->input || !io->output) return fail(CBD_E_INVALID, "layer_apply: null input or output");
  if (!aligned(io->input, l->dtype) || !aligned(io->output, io->output_dtype) || !aligned(io->residual, io->output_dtype))
    return fail(CBD_E_INVALID, "layer_apply: a pointer is not aligned to its elements");
  if (!strides_fit(n, m, io->input_channel_stride, io->input_frame_stride) ||
      !strides_fit(n, m, io->output_channel_stride, io->output_frame_stride) ||
      (io->residual && !strides_fit(n, m, io->residual_channel_stride, io->residual_frame_stride)))
    return fail(CBD_E_INVALID, "layer_apply: bad stride");
  if (!rows_apart(n, m, io->output_channel_stride, io->output_frame_stride, l->N))
    return fail(CBD_E_INVALID, "layer_apply: output rows overlap");
  if (io->input == io->output) return fail(CBD_E_INVALID, "layer_apply: the output must not be the input");
  if (io->residual == io->output && ((n > 1 && io->residual_channel_stride != io->output_channel_stride) ||
                                     (m > 1 && io->residual_frame_stride != io->output_frame_stride)))
    return fail(CBD_E_INVALID, "layer_apply: a residual that is the output must have its strides");
  hipStream_t st = (hipStream_t)hip_stream;
  if (!cbd::stream_is_of(st, l->device)) return fail(CBD_E_INVALID, "layer_apply: the stream belongs to another device");
  cbd::DeviceScope on(l->device);
  HIPCHK(on.error);
  LayerParams p{};
  p.x = io->input; p.w = l->w; p.residual = io->residual; p.bias = l->bias; p.out = io->output;
  p.x_cs = io->input_channel_stride; p.x_fs = io->input_frame_stride;
  p.out_cs = io->output_channel_stride; p.out_fs = io->output_frame_stride;
  p.res_cs = io->residual_channel_stride; p.res_fs = io->residual_frame_stride;
  p.rows = (int32_t)rows; p.frames = io->n_frames; p.K = l->K; p.N = l->N;
  {
    int log2 = 0;
    while ((int64_t)1 << log2 < m) ++log2;
    p.frames_shift = 31 + (uint32_t)log2;   // m <= 2^log2: ceil(2^shift / m) < 2^32 is off by less than 2^(shift - 31) / r
    p.frames_mul = (uint32_t)((((uint64_t)1 << p.frames_shift) + (uint64_t)m - 1) / (uint64_t)m);
  }
  p.scale = io->scale; p.residual_scale = io->residual_scale;
  p.w_blocks = l->blocks; p.w_steps = l->steps; p.act = l->act; p.out_dtype = io->output_dtype;
  if (l->dtype == CBD_F32) HIPCHK(launch<float>(p, st));
  else if (l->dtype == CBD_F16) HIPCHK(launch<cbd::f16>(p, st));
  else HIPCHK(launch<cbd::bf16>(p, st));
  return CBD_OK;
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("layer_apply: ") + e.what());
}

}  // extern "C"
