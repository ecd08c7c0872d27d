// Drawing labels from rows of scores: the kernels, the channels' lists of boosted labels, and their part of the C ABI.
// See include/cbd.h for the rule and the contract of each call.
#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>
#include <vector>

#include "cbd_host.hpp"
#include "cbd_score.hpp"

using cbd::dmalloc;
using cbd::fail;

namespace cbd {
namespace {

struct SampleParams {
  const void *scores;
  int64_t row_stride;
  const int32_t *channels;
  const float *random, *temperature, *top_p, *min_p;
  const int32_t *top_k;
  const uint32_t *bits;      // per channel: one bit per label, set = listed
  const float *offsets;      // per channel
  int32_t *labels, *kept;
  float *logprobs;
  int32_t first_row;         // of this launch
  int32_t num_labels, num_channels, words;   // words: 32-bit words of a channel's bits
  int32_t unit_bits;         // weights are summed in units of 2^-unit_bits
  double series[9];          // ln(2)^k / k!, k = 9 .. 1 (arguments: they stay in scalar registers)
};

constexpr int kThreads = 256;   // of the kernels that set lists
constexpr uint32_t kAllTies = 0xFFFFFFFFu;
constexpr int kList = 256;

constexpr float kLargest = 3.402823466e38f;

// Order of scores as unsigned integers: larger score, larger key (-0 does not occur; masked scores are -inf).
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) { return __uint_as_float(k ^ (~(uint32_t)((int32_t)k >> 31) | 0x80000000u)); }
constexpr uint32_t kLowestKey = 0x00800000u;   // of the smallest finite score
constexpr uint32_t kZeroKey = 0x80000000u;     // of 0

// Weights as integers: exp((x - best) / temperature) in units of 2^-unit_bits, with relative error below 2^-36.
struct Weigher {
  double best, inv_t, slope, bits;   // slope = log2(e) / temperature
  const double *series;              // ln(2)^k / k!, k = 9 .. 1
  // x - best, exact; scores of +inf (the best is one then) count as the largest finite number
  __device__ __forceinline__ double distance(float x) const { return (double)fminf(x, kLargest) - best; }
  __device__ __forceinline__ double log_weight(float x) const { return distance(x) * inv_t; }
  // 2^y as 2^n 2^f, |f| <= 1/2, by the exponential series up to f^9 (the next term is below 2^-37).  Adding 1.5 * 2^52
  // leaves the nearest whole number in the low bits: of y (n is added to the exponent of 2^f) and of the weight, which is
  // at most 2^50.  Weights below 2^-4 units are nothing, so y need not be smaller than that.  Some 20 instructions of 64
  // bits per label: they, not the bytes, bound the passes that sum weights.
  __device__ __forceinline__ uint64_t units(float x) const {
    constexpr double kMagic = 6755399441055744.0;
    const double y = fmax(fma(distance(x), slope, bits), -4.0), shifted = y + kMagic, f = y - (shifted - kMagic);
    double e = fma(series[0], f, series[1]);
#pragma unroll
    for (int k = 2; k < 9; ++k) e = fma(e, f, series[k]);
    e = fma(e, f, 1.0);
    const uint32_t n = (uint32_t)__double_as_longlong(shifted);
    e = __hiloint2double(__double2hiint(e) + (int)(n << 20), __double2loint(e));
    return __double_as_longlong(e + kMagic) & 0x0007FFFFFFFFFFFFll;
  }
};

// Sums and maxima over a wave's lanes by data-parallel primitives (lane l of a row of 16 takes from l - 1, - 2, ...; then
// the rows' last lanes are handed on), 64-bit values in two halves.
template <int kCtrl, int kRows, int kBanks> __device__ __forceinline__ uint32_t from_lanes(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRows, kBanks, false);
}
template <int kCtrl, int kRows, int kBanks> __device__ __forceinline__ uint64_t from_lanes(uint64_t v) {
  return (uint64_t)from_lanes<kCtrl, kRows, kBanks>((uint32_t)(v >> 32)) << 32 | from_lanes<kCtrl, kRows, kBanks>((uint32_t)v);
}
template <typename V> __device__ __forceinline__ V wave_scan(V v) {   // sum over this lane and those before
  V s = v;
  s += from_lanes<0x111, 0xf, 0xf>(v);
  s += from_lanes<0x112, 0xf, 0xf>(v);
  s += from_lanes<0x113, 0xf, 0xf>(v);
  s += from_lanes<0x114, 0xf, 0xe>(s);
  s += from_lanes<0x118, 0xf, 0xc>(s);
  s += from_lanes<0x142, 0xa, 0xf>(s);
  s += from_lanes<0x143, 0xc, 0xf>(s);
  return s;
}
// (lane: the same in all lanes)
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane) { return (uint64_t)of_lane((uint32_t)(v >> 32), lane) << 32 | of_lane((uint32_t)v, lane); }
template <typename V> __device__ __forceinline__ V last_lane(V v) { return of_lane(v, 63); }
template <typename V> __device__ __forceinline__ V wave_sum(V v) { return last_lane(wave_scan(v)); }
__device__ __forceinline__ uint32_t max32(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t min32(uint32_t a, uint32_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max32(v, from_lanes<0x111, 0xf, 0xf>(v));
  v = max32(v, from_lanes<0x112, 0xf, 0xf>(v));
  v = max32(v, from_lanes<0x114, 0xf, 0xf>(v));
  v = max32(v, from_lanes<0x118, 0xf, 0xf>(v));
  v = max32(v, from_lanes<0x142, 0xf, 0xf>(v));
  v = max32(v, from_lanes<0x143, 0xf, 0xf>(v));
  return last_lane(v);
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) { return ~wave_max(~v); }

// f(j) for j = 0 .. n - 1
template <int n, typename F> __device__ __forceinline__ void each_of(F f) {
#pragma unroll
  for (int j = 0; j < n; ++j) {
    f(j);
    if (j & 1) __builtin_amdgcn_sched_barrier(0);   // (weights of more labels at once would need too many registers)
  }
}

// One row of scores as a workgroup reads it: kVec neighbouring labels per thread and turn; a wave's turns lie behind one
// another, and the waves' parts too, so that (wave, turn, lane, place) is the labels' order.
template <typename T, int kVec> struct Row {
  static constexpr int kWords = kVec * (int)sizeof(T) / 4;
  typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
  typedef uint32_t Unaligned __attribute__((ext_vector_type(kWords), aligned(sizeof(T))));   // (vector loads need no more)
  const T *scores;
  const uint32_t *bits;   // of the channel's list, or NULL
  float offset;
  int labels;
  struct Piece { Words scores; uint32_t listed; };
  // labels first .. first + kVec - 1; those beyond the last are masked (and not read)
  __device__ __forceinline__ Piece load(int first) const {
    Piece p;
    if (first + kVec <= labels) {
      p.scores = *(const Unaligned *)(scores + first);
    } else {
      T e[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) e[j] = first + j < labels ? scores[first + j] : (T)-__builtin_inff();
      p.scores = __builtin_bit_cast(Words, e);
    }
    p.listed = bits && first < labels ? bits[first >> 5] >> (first & 31) : 0u;
    return p;
  }
  // The same without a branch, for rows of kVec labels at least: near the end the row's last labels are read, and
  // shift_end() puts them in their places.
  __device__ __forceinline__ Piece load_ahead(int first) const {
    Piece p;
    p.scores = *(const Unaligned *)(scores + min(first, labels - kVec));
    p.listed = 0;
    if (bits) p.listed = bits[min(first, labels - 1) >> 5] >> (first & 31);
    return p;
  }
  __device__ __forceinline__ void shift_end(int first, Piece &p) const {
    if (first + kVec <= labels) return;
    struct All { T v[kVec]; };
    All e = __builtin_bit_cast(All, p.scores);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {   // (labels from the last kVec on: one place to the left per round)
#pragma unroll
      for (int i = 0; i + 1 < kVec; ++i) e.v[i] = first - (labels - kVec) > j ? e.v[i + 1] : e.v[i];
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (first + j >= labels) e.v[j] = (T)-__builtin_inff();
    p.scores = __builtin_bit_cast(Words, e);
  }
  // the scores themselves, fp32: NaN is -inf, -0 is 0, listed ones have the offset added
  __device__ __forceinline__ void values(const Piece &p, float (&x)[kVec]) const {
    struct All { T v[kVec]; };
    const All e = __builtin_bit_cast(All, p.scores);
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[j] = (float)e.v[j] + 0.0f;
    if (__ballot((p.listed & ((1u << kVec) - 1u)) != 0)) {   // (few of a row's turns have any)
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] += p.listed >> j & 1 ? offset : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[j] = fmaxf(x[j], -__builtin_inff());
  }
};

// A workgroup of kBlock threads per row.  kHeld: the row is read once and kept as fp32 in LDS (every thread reads its own
// again); otherwise it is read again for each step.
//
// The kept labels are always a beginning of the order, so they are described by a key and a number of labels that have
// just this key ("keys above `cut`, and the first `ties` labels with it").  top_k and top_p find them by histograms over
// the interval of keys in question, one bin a thread: counts or masses per bin, their running sum from the best key
// down, and the bin where it passes the border is the next interval, narrowed to the keys that occur in it, until one
// key is left.  All sums are of integers, so their order does not matter.
//
// Measured: 2048 x 6000 fp32 with min_p and lists 27 us (the copy of its 49 MB takes 10), 64 x 20000 bf16 with top_k 50 and
// top_p 14, 512 x 5003 fp16 with top_p 21, 256 x 200,000 fp32 with top_p and lists 201, without lists 176 (copy 42): there the
// row is read three times (largest score; masses of the bins; sums of what is kept and the labels near the cut), and the last
// two take some 26 vector instructions of four cycles per label for its weight, 71 million in all: 115 us of issue on the
// 1024 SIMDs.  Rows in LDS spend less than half of their time issuing instructions (12 of 25 us with min_p, 9 of 22 with
// top_p, by their counts); the rest is waiting: for the row's first read, a turn at a time, and at the barriers of some fifteen
// steps.
template <typename T, int kBlock, bool kHeld> __global__ __launch_bounds__(kBlock) void sample_kernel(SampleParams p) {
  constexpr int kWaves = kBlock / 64, kVec = kHeld ? 16 / sizeof(T) : 4, kMaxCells = kHeld ? 1 : 16;
  // (512 against 256 labels near the cut: 512 x 5003 in f16 with top_p 0.9 21 us against 28)
  constexpr int kNear = !kHeld ? 8192 : 512;
  extern __shared__ float4 held[];   // kHeld: the row, by label
  __shared__ uint64_t bins[kBlock];   // of a histogram; later weights of listed labels
  // labels near the cut, or all that may be kept: key << 32 | ~label (larger: earlier in the order), in no order
  __shared__ uint64_t near[kNear];
  __shared__ uint64_t cell_mass[kWaves * kMaxCells], wave_mass[kWaves];
  __shared__ uint32_t cell_ties[kWaves * kMaxCells], wave_a[kWaves], wave_b[kWaves], wave_c[kWaves];
  __shared__ uint64_t pick_before;
  __shared__ uint32_t pick_bin, pick_count, n_near;
  const int r = p.first_row + (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, N = p.num_labels;
  const int ch = p.channels ? p.channels[r] : r;
  auto write = [&](int label, float lp, int kept) {   // (by one thread)
    p.labels[r] = label;
    if (p.logprobs) p.logprobs[r] = lp;
    if (p.kept) p.kept[r] = kept;
  };
  if (ch < 0 || ch >= p.num_channels) {
    if (tid == 0) write(-1, -__builtin_inff(), 0);
    return;
  }
  const float temperature = p.temperature ? p.temperature[r] : 1.0f;
  const int k = p.top_k ? p.top_k[r] : 0;
  const float top_p = p.top_p ? p.top_p[r] : 1.0f, min_p = p.min_p ? p.min_p[r] : 0.0f;
  float random = p.random[r];
  typedef Row<T, kVec> RowT;
  RowT row{(const T *)p.scores + (int64_t)r * p.row_stride, nullptr, p.offsets[ch], N};
  if (row.offset != 0.0f) row.bits = p.bits + (int64_t)ch * p.words;
  const int turns = (N + kBlock * kVec - 1) / (kBlock * kVec);
  const int first = (wave * turns * 64 + lane) * kVec;   // of turn 0
  float best = -__builtin_inff();
  if constexpr (kHeld) {
    for (int t = 0; t < turns; ++t) {
      float x[kVec];
      row.values(row.load(first + t * 64 * kVec), x);
      for (int j = 0; j < kVec; ++j) best = fmaxf(best, x[j]);
#pragma unroll
      for (int q = 0; q < kVec / 4; ++q) held[(first + t * 64 * kVec) / 4 + q] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    }
  }
  const int whole_turns = (int)((unsigned)N / (64u * kVec)) - __builtin_amdgcn_readfirstlane(wave) * turns;   // of this wave
  // the thread's scores of turn t
  auto load_turn = [&](int t, float (&x)[kVec]) __attribute__((always_inline)) {
    if constexpr (kHeld) {
#pragma unroll
      for (int q = 0; q < kVec / 4; ++q) {
        const float4 v = held[(first + t * 64 * kVec) / 4 + q];
        x[4 * q] = v.x; x[4 * q + 1] = v.y; x[4 * q + 2] = v.z; x[4 * q + 3] = v.w;
      }
    } else {
      row.values(row.load(first + t * 64 * kVec), x);
    }
  };
  // f(turn, scores) for all of the thread's turns; rows that are read again: two turns on their way
  auto each_turn = [&](auto f) __attribute__((always_inline)) {
    if constexpr (kHeld) {
#pragma unroll 1
      for (int t = 0; t < turns; ++t) {
        float x[kVec];
        load_turn(t, x);
        f(t, x);
      }
    } else {
      typename RowT::Piece even = row.load_ahead(first), odd = row.load_ahead(first + 64 * kVec);
      auto one = [&](int t, typename RowT::Piece &p) __attribute__((always_inline)) {
        float x[kVec];
        if (t >= whole_turns) row.shift_end(first + t * 64 * kVec, p);
        row.values(p, x);
        p = row.load_ahead(first + (t + 2) * 64 * kVec);
        f(t, x);
      };
#pragma unroll 1
      for (int t = 0; t < turns; t += 2) {
        one(t, even);
        if (t + 1 < turns) one(t + 1, odd);
      }
    }
  };
  // the largest and the smallest of what the waves give, to all
  auto block_range = [&](uint32_t hi, uint32_t lo, uint32_t *hi_out, uint32_t *lo_out) __attribute__((always_inline)) {
    hi = wave_max(hi);
    lo = wave_min(lo);
    __syncthreads();
    if (lane == 0) { wave_a[wave] = hi; wave_b[wave] = lo; }
    __syncthreads();
    hi = wave_a[0]; lo = wave_b[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) { hi = max32(hi, wave_a[w]); lo = min32(lo, wave_b[w]); }
    *hi_out = hi; *lo_out = lo;
  };
  // the lowest label of those for which f(score) holds, to all; N if none
  auto lowest_label = [&](auto f) __attribute__((always_inline)) {
    uint32_t at = (uint32_t)N;
    each_turn([&](int t, const float (&x)[kVec]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = kVec - 1; j >= 0; --j)
        if (f(x[j])) at = min32(at, (uint32_t)(first + t * 64 * kVec + j));
    });
    uint32_t hi, lo;
    block_range(0, at, &hi, &lo);
    return (int)lo;
  };
  if constexpr (!kHeld) each_turn([&](int, const float (&x)[kVec]) __attribute__((always_inline)) {
    for (int j = 0; j < kVec; ++j) best = fmaxf(best, x[j]);
  });
  const float thread_best = best;
  uint32_t best_key, unused;
  block_range(score_key(best), 0, &best_key, &unused);
  best = key_score(best_key);
  if (best == -__builtin_inff()) {
    if (tid == 0) write(-1, best, 0);
    return;
  }
  if (!(temperature > 0.0f)) {
    const int label = lowest_label([&](float x) __attribute__((always_inline)) { return x == best; });
    if (tid == 0) write(label, 0.0f, 1);
    return;
  }
  const uint32_t last_key = best == __builtin_inff() ? best_key : kLowestKey;   // (scores of +inf leave the others no mass)
  const Weigher wt{(double)fminf(best, kLargest), 1.0 / (double)temperature, 1.4426950408889634 / (double)temperature, (double)p.unit_bits, p.series};
  uint32_t cut = last_key, ties = kAllTies;

  // f(score) for all of the row's labels, and for the labels in `near`
  auto each_score = [&](auto f) __attribute__((always_inline)) {
    each_turn([&](int, const float (&x)[kVec]) __attribute__((always_inline)) { each_of<kVec>([&](int j) __attribute__((always_inline)) { f(x[j]); }); });
  };
  auto each_near = [&](auto f) __attribute__((always_inline)) {
    for (uint32_t i = tid; i < n_near; i += kBlock) f(key_score((uint32_t)(near[i] >> 32)));
  };
  // Keys from lo to hi, in which the running count or mass, from best_key down, reaches `want`; `before` is the sum over
  // larger keys, `from_lo` (counts only) the number of labels with keys from lo on.
  struct Interval { uint32_t lo, hi; uint64_t before; double want; uint32_t from_lo; };
  // One step: bins over the keys from hi down to `end` (the last bin takes those down to lo as well), and the one in which
  // the sum passes `want` becomes the interval.
  auto narrow = [&](auto by_mass, auto each, Interval &v, uint32_t end, auto want_of) __attribute__((always_inline)) {
    constexpr bool kMass = decltype(by_mass)::value;
    const int width = 32 - __clz((int)((v.hi - max32(end, v.lo)) | 1u)), log2 = kBlock == 1024 ? 10 : kBlock == 512 ? 9 : 8;
    const int shift = width > log2 ? width - log2 : 0;
    __syncthreads();
    bins[tid] = 0;
    __syncthreads();
    const float lo = key_score(v.lo), hi = key_score(v.hi);
    each([&](float x) __attribute__((always_inline)) {
      if (x >= lo && x <= hi) {
        const uint32_t b = min32((v.hi - score_key(x)) >> shift, kBlock - 1);
        if constexpr (kMass) {
          const uint64_t u = wt.units(x);
          if (u) atomicAdd((unsigned long long *)&bins[b], (unsigned long long)u);
        } else {
          atomicAdd((uint32_t *)&bins[b], 1u);
        }
      }
    });
    __syncthreads();
    const uint64_t mine = bins[tid];
    uint64_t upto = wave_scan(mine);
    if (lane == 63) wave_mass[wave] = upto;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) upto += wave_mass[w];
      all += wave_mass[w];
    }
    v.want = want_of(all, v.want);
    const double from = (double)(v.before + upto - mine), to = (double)(v.before + upto);
    if (from < v.want && to >= v.want) {
      pick_bin = (uint32_t)tid;
      pick_before = v.before + upto - mine;
      pick_count = (uint32_t)min((uint64_t)kAllTies, v.before + upto);
    }
    __syncthreads();
    v.before = pick_before;
    v.from_lo = pick_count;
    v.hi -= pick_bin << shift;
    if (pick_bin < kBlock - 1 && (v.hi - v.lo) >> shift) v.lo = v.hi - (1u << shift) + 1u;
    // -0, which no score is, must not be the upper end: as a number it is not below the zeros, whose key is above it.  (The
    // interval has a score, so that lo is below it.)
    if (v.hi == kZeroKey - 1u) v.hi -= 1u;
  };
  auto as_before = [](uint64_t, double want) { return want; };
  auto end_of = [&](double reach) __attribute__((always_inline)) { return score_key((float)fmax((double)fminf(best, kLargest) - reach, -(double)kLargest)); };
  // ... and down to the keys that occur in it
  auto tighten = [&](auto each, Interval &v) __attribute__((always_inline)) {
    uint32_t top = 0, low = 0xFFFFFFFFu;
    const float lo = key_score(v.lo), hi = key_score(v.hi);
    each([&](float x) __attribute__((always_inline)) {
      if (x >= lo && x <= hi) { top = max32(top, score_key(x)); low = min32(low, score_key(x)); }
    });
    block_range(top, low, &v.hi, &v.lo);
  };
  // Mass of the kept labels and labels at the cut per cell: a wave's turns, or a stretch of them.
  const int cell_turns = (turns + kMaxCells - 1) / kMaxCells;
  const int cells = (turns + cell_turns - 1) / cell_turns;   // per wave
  uint64_t mass = 0;
  uint32_t at_cut = 0;
  auto end_cell = [&](int cell) __attribute__((always_inline)) {
    mass = wave_sum(mass);
    at_cut = wave_sum(at_cut);
    if (lane == 0) { cell_mass[wave * cells + cell] = mass; cell_ties[wave * cells + cell] = at_cut; }
    mass = 0; at_cut = 0;
  };
  int cell_left;   // turns until the present cell ends
  auto next_turn = [&](int t) __attribute__((always_inline)) {
    if (cell_left == 0) { end_cell(t / cell_turns - 1); cell_left = cell_turns; }
    --cell_left;
  };
  // One pass that notes the labels with keys from lo to hi in `near` and sums those above per cell (wave_c: their number).
  // False if there are more than fit.
  auto collect = [&](uint32_t lo_key, uint32_t hi_key) __attribute__((always_inline)) {
    const float lo = key_score(lo_key), hi = key_score(hi_key);
    __syncthreads();
    if (tid == 0) n_near = 0;
    __syncthreads();
    uint32_t above = 0;
    cell_left = cell_turns;
    each_turn([&](int t, const float (&x)[kVec]) __attribute__((always_inline)) {
      next_turn(t);
      uint32_t n = 0;
      each_of<kVec>([&](int j) __attribute__((always_inline)) {
        if (x[j] > hi) { mass += wt.units(x[j]); ++above; }
        n += x[j] >= lo && x[j] <= hi;
      });
      if (!__ballot(n != 0)) return;
      const uint32_t upto = wave_scan(n), all = last_lane(upto);
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&n_near, all);
      at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + upto - n;
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (x[j] >= lo && x[j] <= hi) {
          if (at < (uint32_t)kNear) near[at] = (uint64_t)score_key(x[j]) << 32 | (uint32_t)~(first + t * 64 * kVec + j);
          ++at;
        }
    });
    end_cell(cells - 1);
    above = wave_sum(above);
    if (lane == 0) wave_c[wave] = above;
    __syncthreads();
    return n_near <= (uint32_t)kNear;
  };
  // Finds cut and ties: the first `want` labels or the mass `want` (want_of: from the sum of all) of those with keys from
  // v.lo on.  list_all: stops as soon as no more than kList labels have keys from v.lo on (counts only; true then).
  // *listed: labels above this key are in the cells of collect(), those down to cut in `near`; 0: they are not.
  auto search = [&](auto by_mass, Interval &v, auto want_of, bool list_all, uint32_t *listed) __attribute__((always_inline)) {
    constexpr bool kMass = decltype(by_mass)::value;
    // bins reach down to weights of 2^-46 (or, for counts, to scores 40 below the best): beyond, the search begins anew
    uint32_t end = end_of(kMass ? 32.0 * (double)temperature : 40.0);
    *listed = 0;
    for (bool begun = false;; begun = true) {
      narrow(by_mass, each_score, v, end, [&](uint64_t all, double want) __attribute__((always_inline)) { return begun ? want : want_of(all); });
      if (!kMass && list_all && v.from_lo <= (uint32_t)kList) return true;
      if (v.lo == v.hi) break;
      if (!list_all && collect(v.lo, v.hi)) { *listed = v.hi; break; }
      tighten(each_score, v);
      if (v.lo == v.hi) break;
      end = v.lo;
    }
    while (v.lo != v.hi) {
      tighten(each_near, v);
      if (v.lo != v.hi) narrow(by_mass, each_near, v, v.lo, as_before);
    }
    uint32_t t = kAllTies;
    if constexpr (!kMass) {
      t = (uint32_t)(v.want - (double)v.before);
    } else {
      // labels j = 0, 1, ... with this key are kept while before + j * (their weight) < want
      const uint64_t w = wt.units(key_score(v.hi));
      const double j = w > 0 ? ceil((v.want - (double)v.before) / (double)w) : 4e9;
      t = j < 1.0 ? 1u : j < 4e9 ? (uint32_t)j : kAllTies;
    }
    if (v.hi > cut) { cut = v.hi; ties = t; }
    else ties = min32(ties, t);
    return false;
  };
  auto enough = [&](float x, double least) __attribute__((always_inline)) { return exp(wt.log_weight(x)) >= least; };   // min_p's test
  // The rest where all labels that may be kept, n of them, are in `near`: the first `most` of the order, of these those
  // with less than `want` before them (share >= 0: want is this share of the mass of the first `most`), then min_p and the
  // choice.  A thread has one label; its places in the order and by label are found by comparing it with all others.
  auto finish_list = [&](int n, uint32_t most, double share, double want) __attribute__((always_inline)) {
    const bool have = tid < n, in_list = tid < kList;   // (waves beyond the list only keep step)
    const uint64_t me = have ? near[tid] : 0;
    const float score = key_score((uint32_t)(me >> 32));
    uint32_t rank = 0, place = 0;
    uint64_t w = 0, v = 0, upto = 0;
    if (have) {
#pragma unroll 16
      for (int j = 0; j < n; ++j) {
        const uint64_t other = near[j];
        rank += other > me;
        place += (uint32_t)other > (uint32_t)me;   // (~label: larger is lower)
      }
      w = wt.units(score);
      bins[rank] = w;
    }
    // sum up to this thread's entry of bins, over the first n; *all: of all of them
    auto scan_bins = [&](uint64_t *all) __attribute__((always_inline)) {
      __syncthreads();
      v = have ? bins[tid] : 0;
      if (in_list) {
        upto = wave_scan(v);
        if (lane == 63) wave_mass[wave] = upto;
      }
      __syncthreads();
      uint64_t sum = 0;
#pragma unroll
      for (int i = 0; i < kList / 64; ++i) {
        if (i < wave) upto += wave_mass[i];
        sum += wave_mass[i];
      }
      *all = sum;
    };
    uint64_t total;
    scan_bins(&total);
    most = min32(most, (uint32_t)n);
    if (share >= 0.0) {
      if (tid == (int)most - 1) pick_before = upto;
      __syncthreads();
      want = share * (double)pick_before;
    }
    // three beginnings of the order: the shortest counts
    const double least = min_p > 0.0f ? (double)fminf(min_p, 1.0f) : 0.0;
    const uint64_t by_mass = __ballot(have && (tid == 0 || (double)(upto - v) < want));
    const uint64_t by_min = __ballot(have && (least == 0.0 || enough(score, least)));
    if (in_list && lane == 0) { wave_a[wave] = __popcll(by_mass); wave_b[wave] = __popcll(by_min); }
    __syncthreads();
    uint32_t n_mass = 0, n_min = 0;
#pragma unroll
    for (int i = 0; i < kList / 64; ++i) { n_mass += wave_a[i]; n_min += wave_b[i]; }
    const uint32_t kept = min32(most, min32(n_mass, n_min));
    // by label
    const bool mine = have && rank < kept;
    if (have) bins[place] = mine ? w : 0;
    if (tid == 0) pick_bin = kAllTies;
    scan_bins(&total);
    if (!(random > 0.0f)) {
      if (mine && wt.log_weight(score) > -745.13) atomicMin(&pick_bin, place);   // (its weight is not zero in 64 bits)
    } else {
      uint64_t target = (uint64_t)((double)random * (double)total);
      if (random >= 1.0f || target >= total) target = total - 1;
      if (have && upto > target && upto - v <= target) pick_bin = (uint32_t)tid;
    }
    __syncthreads();
    if (mine && place == pick_bin)
      write((int)~(uint32_t)me, (float)(wt.log_weight(score) - log((double)total * ldexp(1.0, -p.unit_bits))), (int)kept);
  };
  const bool by_count = k > 0 && k < N, by_share = top_p < 1.0f;
  uint32_t listed_from = 0;   // not 0: collect()'s sums are of larger keys, and the rest of the kept labels is in `near`
  if (by_count && k <= kList / 2 && N >= 4 * kBlock) {
    // The best scores of the threads are scores of as many labels: what is below the k-th of them is not among the first
    // k.  With labels in no order few others are above it (177 for k = 128 and 256 threads, on average), so that the list
    // is there without bins over the row (with top_k 50: 64 x 20,000 12 against 15 us, 256 x 200,000 63 against 89).
    Interval v{last_key, best_key, 0, 0.0, kAllTies};
    uint64_t threads = 0;
    narrow(std::false_type(), [&](auto f) __attribute__((always_inline)) { f(thread_best); }, v, end_of(40.0),
           [&](uint64_t all, double) __attribute__((always_inline)) { threads = all; return (double)min((uint64_t)k, all); });
    if (threads >= (uint64_t)k && collect(v.lo, best_key) && n_near <= (uint32_t)kList) {
      finish_list((int)n_near, (uint32_t)k, by_share ? (double)max(top_p, 0.0f) : -1.0, __builtin_inf());
      return;
    }
  }
  if (by_count) {
    Interval v{last_key, best_key, 0, 0.0, kAllTies};
    uint64_t valid = 0;   // (no more labels than top_k: nothing is cut)
    if (search(std::false_type(), v, [&](uint64_t all) __attribute__((always_inline)) { valid = all; return (double)min((uint64_t)k, all); }, k <= kList, &listed_from)) {
      collect(v.lo, best_key);
      finish_list((int)v.from_lo, (uint32_t)k, by_share ? (double)max(top_p, 0.0f) : -1.0, __builtin_inf());
      return;
    }
    if (valid <= (uint64_t)k) ties = kAllTies;
  }
  if (top_p <= 0.0f) {
    cut = best_key; ties = 1; listed_from = 0;
  } else if (by_share) {
    // how many labels have the key `cut` matters to the mass only if not all of them are kept
    uint64_t left_out = 0;
    if (ties != kAllTies) {
      uint32_t n = 0;
      const float x_cut = key_score(cut);
      each_score([&](float x) __attribute__((always_inline)) { n += x == x_cut; });
      n = wave_sum(n);
      __syncthreads();
      if (lane == 0) wave_a[wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) n += wave_a[w];
      left_out = (uint64_t)(n - ties) * wt.units(x_cut);
    }
    Interval v{cut, best_key, 0, 0.0, kAllTies};
    search(std::true_type(), v, [&](uint64_t all) __attribute__((always_inline)) { return (double)top_p * (double)(all - left_out); }, false, &listed_from);
  }
  if (min_p > 0.0f) {
    // the smallest key with exp(log_weight) >= min_p: guessed, and found among its neighbours, 64 at a time
    const double least = (double)fminf(min_p, 1.0f);
    const uint32_t guess = score_key((float)fmax(wt.best + (double)temperature * log(least), -(double)kLargest));
    uint32_t from = guess > last_key + 32u ? guess - 32u : last_key;   // lane 0's key
    if (from > best_key) from = best_key;
    uint64_t yes = __ballot(from + lane <= best_key && enough(key_score(min32(from + lane, best_key)), least));
    if (from + 63u >= best_key) yes |= 1ull << (best_key - from);   // (the best always is)
    if (!yes || (yes & 1ull && from > last_key)) {
      // not there (many scores to which the test gives the same result): the whole interval, a 64th of what is left at a
      // time; lo stays a key that is not enough or last_key
      uint32_t lo = last_key, hi = best_key;   // hi is enough
      while (hi > lo) {
        // (64 steps pass hi, but 63 need not: the last lane always has hi, so that one of them is enough)
        const uint32_t step = (hi - lo) / 64u + 1u, key = lane < 63 && lo + (uint64_t)lane * step < hi ? lo + (uint32_t)lane * step : hi;
        const uint64_t ok = __ballot(key == hi || enough(key_score(key), least));
        const int l = __ffsll((unsigned long long)ok) - 1;
        const uint32_t at = __shfl(key, l), under = l > 0 ? __shfl(key, l - 1) + 1u : at;
        hi = at;
        lo = under < hi ? under : hi;
      }
      from = hi;
      yes = 1;
    }
    const uint32_t c = from + (uint32_t)(__ffsll((unsigned long long)yes) - 1);
    if (c > cut) {
      cut = c; ties = kAllTies;
      if (c > listed_from) listed_from = 0;   // (the sums hold labels below the cut)
    }
    if (!by_count && !by_share) {
      // few labels are left, as a rule
      if (collect(cut, best_key)) {
        if (n_near <= (uint32_t)kList) {
          finish_list((int)n_near, kAllTies, -1.0, __builtin_inf());
          return;
        }
        listed_from = best_key;   // (all of them are in `near`)
      }
    }
  }
  const float x_cut = key_score(cut);
  const uint64_t w_cut = wt.units(x_cut);
  if (listed_from) {
    // the cells lack the labels in `near`
    const uint32_t n = n_near;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kBlock) {
      const uint32_t key = (uint32_t)(near[i] >> 32), g = ~(uint32_t)near[i] / (64u * kVec);
      const uint32_t cell = g / (uint32_t)turns * cells + g % (uint32_t)turns / cell_turns;
      if (key > cut) {
        atomicAdd((unsigned long long *)&cell_mass[cell], (unsigned long long)wt.units(key_score(key)));
        atomicAdd(&wave_c[0], 1u);
      } else if (key == cut) {
        atomicAdd(&cell_ties[cell], 1u);
      }
    }
  } else {
    uint32_t above = 0;
    __syncthreads();
    cell_left = cell_turns;
    each_turn([&](int t, const float (&x)[kVec]) __attribute__((always_inline)) {
      next_turn(t);
      each_of<kVec>([&](int j) __attribute__((always_inline)) {
        if (x[j] > x_cut) { mass += wt.units(x[j]); ++above; }
        at_cut += x[j] == x_cut;
      });
    });
    end_cell(cells - 1);
    above = wave_sum(above);
    if (lane == 0) wave_c[wave] = above;
  }
  __syncthreads();
  // (every wave by itself: lane l has cells l * kCells ..; one after the other they would take 256 reads' latency)
  constexpr int kCells = (kWaves * kMaxCells + 63) / 64;
  uint64_t lane_mass = 0, of_cell[kCells];
  uint32_t lane_ties = 0, ties_of_cell[kCells];
#pragma unroll
  for (int i = 0; i < kCells; ++i) {
    const int c = lane * kCells + i;
    of_cell[i] = c < kWaves * cells ? cell_mass[c] : 0;
    ties_of_cell[i] = c < kWaves * cells ? cell_ties[c] : 0;
    lane_mass += of_cell[i];
    lane_ties += ties_of_cell[i];
  }
  const uint32_t ties_upto = wave_scan(lane_ties);
  uint64_t total = wave_sum(lane_mass);
  const uint64_t seen = last_lane(ties_upto), kept_ties = seen < ties ? seen : (uint64_t)ties;
  total += kept_ties * w_cut;
  uint32_t kept = (uint32_t)kept_ties;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) kept += wave_c[w];
  auto answer = [&](int label, float x) __attribute__((always_inline)) {
    write(label, (float)(wt.log_weight(x) - log((double)total * ldexp(1.0, -p.unit_bits))), (int)kept);
  };
  if (!(random > 0.0f)) {
    // the first kept label whose weight is not zero in 64 bits
    const int label = lowest_label([&](float x) __attribute__((always_inline)) { return x >= x_cut && wt.log_weight(x) > -745.13; });
    each_turn([&](int t, const float (&x)[kVec]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (first + t * 64 * kVec + j == label) answer(label, x[j]);
    });
    return;
  }
  uint64_t target = (uint64_t)((double)random * (double)total);
  if (random >= 1.0f || target >= total) target = total - 1;
  // the cell in which the running sum passes the target; its wave goes through its turns
  auto kept_of = [&](uint32_t before, uint32_t n) {   // kept ones of n ties with `before` ahead of them
    return before >= ties ? 0u : min32(n, ties - before);
  };
  uint32_t rank = ties_upto - lane_ties;   // ties before
  const uint64_t lane_kept = lane_mass + (uint64_t)kept_of(rank, lane_ties) * w_cut, lane_upto = wave_scan(lane_kept);
  const int at_lane = __ffsll((unsigned long long)__ballot(lane_upto > target)) - 1;
  uint64_t run = lane_upto - lane_kept;
  int cell = lane * kCells;
#pragma unroll
  for (int i = 0; i < kCells - 1; ++i) {
    const uint64_t m = of_cell[i] + (uint64_t)kept_of(rank, ties_of_cell[i]) * w_cut;
    if (cell == lane * kCells + i && run + m <= target) {
      run += m;
      rank += ties_of_cell[i];
      ++cell;
    }
  }
  run = of_lane(run, at_lane);
  rank = of_lane(rank, at_lane);
  cell = (int)of_lane((uint32_t)cell, at_lane);
  if (wave != cell / cells) return;
  const int t0 = cell % cells * cell_turns, t1 = min(t0 + cell_turns, turns);
  bool found = false;
#pragma unroll 1
  for (int t = t0; t < t1 && !found; ++t) {   // (all lanes of the wave)
    float x[kVec];
    load_turn(t, x);
    uint64_t m = 0;
    uint32_t n = 0;
    each_of<kVec>([&](int j) __attribute__((always_inline)) {
      if (x[j] > x_cut) m += wt.units(x[j]);
      n += x[j] == x_cut;
    });
    const uint64_t m_upto = wave_scan(m);
    const uint32_t n_upto = wave_scan(n);
    const uint64_t upto = run + m_upto + (uint64_t)kept_of(rank, n_upto) * w_cut;
    const uint64_t passed = __ballot(upto > target);
    found = passed != 0;
    if (found && lane == __ffsll((unsigned long long)passed) - 1) {
      uint32_t before = rank + n_upto - n;
      uint64_t sum = run + m_upto - m + (uint64_t)kept_of(rank, n_upto - n) * w_cut;
      bool done = false;
      each_of<kVec>([&](int j) __attribute__((always_inline)) {
        if (done || x[j] < x_cut || (x[j] == x_cut && before++ >= ties)) return;
        sum += wt.units(x[j]);
        if (sum > target) { done = true; answer(first + t * 64 * kVec + j, x[j]); }
      });
    }
    run = last_lane(upto);   // (with the kept ties of this turn)
    rank += last_lane(n_upto);
  }
}

// Clears the bits of the given channels and notes their offsets; one workgroup per channel.
__global__ __launch_bounds__(kThreads) void clear_lists_kernel(const int32_t *channels, const float *offsets, int32_t words,
                                                               uint32_t *bits, float *channel_offset) {
  const int c = channels[blockIdx.x];
  for (int i = threadIdx.x; i < words; i += kThreads) bits[(int64_t)c * words + i] = 0u;
  if (threadIdx.x == 0) channel_offset[c] = offsets[blockIdx.x];
}

// Sets one bit per (channel, label) entry.
__global__ __launch_bounds__(kThreads) void list_labels_kernel(const int2 *entries, int32_t n, int32_t words, uint32_t *bits) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < n) atomicOr(bits + (int64_t)entries[i].x * words + (entries[i].y >> 5), 1u << (entries[i].y & 31));
}

}  // namespace
}  // namespace cbd

struct cbd_sampler {
  int device = 0;
  hipStream_t stream = nullptr;
  int32_t C = 0, N = 0, words = 0, unit_bits = 0;
  uint32_t *bits = nullptr;
  float *offsets = nullptr;
  cbd::StageRing ring;    // list uploads
  std::vector<uint8_t> seen;
};

namespace {
constexpr int32_t kUpload = 1 << 15;   // entries of 8 bytes per upload slot

constexpr size_t kHeldBytes = 144 * 1024;   // of LDS for a row's scores (with the kernel's own 13 KB: within 160 KB)

template <typename T, int kBlock> size_t held_bytes(int num_labels) {   // whole turns
  const size_t turn = (size_t)kBlock * (16 / sizeof(T));
  return ((size_t)num_labels + turn - 1) / turn * turn * sizeof(uint32_t);
}

template <typename T, int kBlock, bool kHeld> void launch_rows(const cbd::SampleParams &p, int n, hipStream_t st) {
  const size_t lds = kHeld ? held_bytes<T, kBlock>(p.num_labels) : 0;
  hipLaunchKernelGGL((cbd::sample_kernel<T, kBlock, kHeld>), dim3((unsigned)n), dim3(kBlock), lds, st, p);
}

// Threads per row: for few labels a step costs as much as its barriers, and two or more workgroups on a compute unit hide
// each other's; a row alone on its compute unit with some thousand labels is faster with more threads.  With top_p 0.9,
// fp32, threads 256 / 512 / 1024: 512 x 1500 12.2 / 12.8 / 24.4 us, 1 x 1500 10.1 / 9.4 / 11.8, 1 x 6000 14.6 / 12.4 / 14.1,
// 256 x 6000 18.5 / 14.7 / 16.2, 512 x 6000 21.3 / 19.2 / 29.7, 512 x 5003 in f16 21.0 / 21.4 / 29.4.
template <typename T> void launch_sample(const cbd::SampleParams &p, int n, hipStream_t st) {
  if (p.num_labels <= 2048 || (p.num_labels <= 8192 && n > 256)) launch_rows<T, 256, true>(p, n, st);
  else if (p.num_labels <= 8192) launch_rows<T, 512, true>(p, n, st);
  else if (held_bytes<T, 1024>(p.num_labels) <= kHeldBytes) launch_rows<T, 1024, true>(p, n, st);
  else launch_rows<T, 1024, false>(p, n, st);
}

template <typename T> hipError_t allow_held() {   // on the current device
  const void *const kernels[] = {(const void *)cbd::sample_kernel<T, 256, true>, (const void *)cbd::sample_kernel<T, 512, true>,
                                 (const void *)cbd::sample_kernel<T, 1024, true>};
  for (const void *k : kernels) {
    const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kHeldBytes);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

extern "C" {

int32_t cbd_sampler_create(int32_t num_channels, int32_t num_labels, void *hip_stream, cbd_sampler **out) try {
  if (!out) return fail(CBD_E_INVALID, "sampler: null argument");
  if (num_channels < 1) return fail(CBD_E_INVALID, "sampler: num_channels < 1");
  if (num_labels < 1 || num_labels > 1048576) return fail(CBD_E_INVALID, "sampler: num_labels must be in [1, 1048576]");
  hipStream_t st = (hipStream_t)hip_stream;
  int device = 0;
  HIPCHK(hipGetDevice(&device));
  if (!cbd::stream_is_of(st, device)) return fail(CBD_E_INVALID, "sampler: the stream belongs to another device");
  if (cbd::is_capturing(st)) return fail(CBD_E_INVALID, "sampler: the stream is being captured");
  cbd_sampler *s = new (std::nothrow) cbd_sampler();
  if (!s) return fail(CBD_E_NOMEM, "sampler: host allocation");
  struct Guard {
    cbd_sampler *s;
    ~Guard() { if (s) cbd_sampler_free(s); }
  } guard{s};
  s->device = device; s->stream = st; s->C = num_channels; s->N = num_labels;
  s->words = (num_labels + 127) / 128 * 4;   // (rows of 16-byte pieces)
  int log2 = 0;
  while ((1 << log2) < num_labels) ++log2;
  s->unit_bits = std::min(50, 62 - log2);   // num_labels weights of at most 1 stay below 2^63; one of them below 2^51
  s->seen.assign((size_t)num_channels, 0);
  const size_t n = (size_t)num_channels * (size_t)s->words;
  HIPCHK(dmalloc(&s->bits, n, nullptr));
  HIPCHK(dmalloc(&s->offsets, (size_t)num_channels, nullptr));
  HIPCHK(allow_held<float>());
  HIPCHK(allow_held<cbd::f16>());
  HIPCHK(allow_held<cbd::bf16>());
  HIPCHK(s->ring.init(sizeof(int2) * kUpload));
  HIPCHK(hipMemsetAsync(s->bits, 0, n * sizeof(uint32_t), st));
  HIPCHK(hipMemsetAsync(s->offsets, 0, (size_t)num_channels * sizeof(float), st));
  *out = s;
  guard.s = nullptr;
  return CBD_OK;
} catch (const std::bad_alloc &) {
  return fail(CBD_E_NOMEM, "sampler_create: host allocation failed");
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("sampler_create: ") + e.what());
}

int32_t cbd_sampler_free(cbd_sampler *s) {
  if (!s) return CBD_OK;
  if (cbd::is_capturing(s->stream)) return fail(CBD_E_INVALID, "sampler_free: the stream is being captured");
  (void)hipStreamSynchronize(s->stream);
  if (s->bits) (void)hipFree(s->bits);
  if (s->offsets) (void)hipFree(s->offsets);
  s->ring.destroy();
  delete s;
  return CBD_OK;
}

int32_t cbd_sampler_set_contexts(cbd_sampler *s, const int32_t *channels, int32_t n_channels, const int32_t *label_idx,
                                 const int32_t *list_offsets, const float *offsets) try {
  if (!s || !channels || !list_offsets || !offsets) return fail(CBD_E_INVALID, "sampler_set_contexts: null argument");
  if (n_channels <= 0 || n_channels > s->C) return fail(CBD_E_INVALID, "sampler_set_contexts: bad channel count");
  // validate everything before anything changes
  std::fill(s->seen.begin(), s->seen.end(), (uint8_t)0);
  if (list_offsets[0] != 0) return fail(CBD_E_INVALID, "sampler_set_contexts: list_offsets[0] != 0");
  for (int32_t i = 0; i < n_channels; ++i) {
    if (channels[i] < 0 || channels[i] >= s->C) return fail(CBD_E_INVALID, "sampler_set_contexts: channel out of range");
    if (s->seen[channels[i]]) return fail(CBD_E_INVALID, "sampler_set_contexts: duplicate channel");
    s->seen[channels[i]] = 1;
    if (list_offsets[i + 1] < list_offsets[i]) return fail(CBD_E_INVALID, "sampler_set_contexts: list_offsets not monotone");
    if (!std::isfinite(offsets[i])) return fail(CBD_E_INVALID, "sampler_set_contexts: non-finite offset");
  }
  const int32_t total = list_offsets[n_channels];
  if (total > 0 && !label_idx) return fail(CBD_E_INVALID, "sampler_set_contexts: null list");
  for (int32_t k = 0; k < total; ++k)
    if (label_idx[k] < 0 || label_idx[k] >= s->N) return fail(CBD_E_INVALID, "sampler_set_contexts: label out of range");
  if (cbd::is_capturing(s->stream)) return fail(CBD_E_INVALID, "sampler_set_contexts: the stream is being captured");
  cbd::DeviceScope on(s->device);
  HIPCHK(on.error);
  // (64 bits: the start of the piece behind the last one may be beyond 32)
  for (int64_t i0 = 0; i0 < n_channels; i0 += kUpload) {
    const int32_t m = (int32_t)std::min<int64_t>(kUpload, n_channels - i0);
    int slot = 0;
    HIPCHK(s->ring.acquire(&slot));
    memcpy(s->ring.host[slot], channels + i0, sizeof(int32_t) * (size_t)m);
    memcpy((int32_t *)s->ring.host[slot] + m, offsets + i0, sizeof(float) * (size_t)m);
    HIPCHK(s->ring.upload(slot, sizeof(int32_t) * 2 * (size_t)m, s->stream));
    const int32_t *dv = (const int32_t *)s->ring.dev[slot];
    hipLaunchKernelGGL(cbd::clear_lists_kernel, dim3((unsigned)m), dim3(cbd::kThreads), 0, s->stream, dv,
                       (const float *)(dv + m), s->words, s->bits, s->offsets);
    HIPCHK(hipGetLastError());
    HIPCHK(s->ring.release(slot, s->stream));
  }
  int32_t channel = 0;   // position whose list entry k belongs to
  for (int64_t k0 = 0; k0 < total; k0 += kUpload) {
    const int32_t m = (int32_t)std::min<int64_t>(kUpload, total - k0);
    int slot = 0;
    HIPCHK(s->ring.acquire(&slot));
    int2 *h = (int2 *)s->ring.host[slot];
    for (int32_t k = 0; k < m; ++k) {
      while (list_offsets[channel + 1] <= k0 + k) ++channel;
      h[k] = make_int2(channels[channel], label_idx[k0 + k]);
    }
    HIPCHK(s->ring.upload(slot, sizeof(int2) * (size_t)m, s->stream));
    hipLaunchKernelGGL(cbd::list_labels_kernel, dim3((unsigned)((m + cbd::kThreads - 1) / cbd::kThreads)), dim3(cbd::kThreads),
                       0, s->stream, (const int2 *)s->ring.dev[slot], m, s->words, s->bits);
    HIPCHK(hipGetLastError());
    HIPCHK(s->ring.release(slot, s->stream));
  }
  return CBD_OK;
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("sampler_set_contexts: ") + e.what());
}

int32_t cbd_sample_labels(cbd_sampler *s, const cbd_sample_desc *d) try {
  if (!s || !d) return fail(CBD_E_INVALID, "sample_labels: null argument");
  if (d->n < 0) return fail(CBD_E_INVALID, "sample_labels: negative row count");
  if (d->dtype < CBD_F32 || d->dtype > CBD_BF16) return fail(CBD_E_INVALID, "sample_labels: dtype");
  if (d->n == 0) return CBD_OK;
  if (!d->channels && d->n > s->C) return fail(CBD_E_INVALID, "sample_labels: more rows than channels");
  if (!d->scores || !d->random || !d->labels) return fail(CBD_E_INVALID, "sample_labels: null scores, random or labels");
  if (d->row_stride < 0 || d->row_stride > ((int64_t)1 << 60) / d->n) return fail(CBD_E_INVALID, "sample_labels: bad row_stride");
  const void *words[] = {d->channels, d->random, d->temperature, d->top_k, d->top_p, d->min_p, d->labels, d->logprobs, d->kept};
  for (const void *w : words)
    if ((uintptr_t)w & 3) return fail(CBD_E_INVALID, "sample_labels: a pointer is not aligned to its elements");
  if ((uintptr_t)d->scores & (cbd::dtype_size(d->dtype) - 1))
    return fail(CBD_E_INVALID, "sample_labels: scores not aligned to their elements");
  cbd::DeviceScope on(s->device);
  HIPCHK(on.error);
  cbd::SampleParams p{};
  p.scores = d->scores; p.row_stride = d->row_stride; p.channels = d->channels;
  p.random = d->random; p.temperature = d->temperature; p.top_p = d->top_p; p.min_p = d->min_p; p.top_k = d->top_k;
  p.bits = s->bits; p.offsets = s->offsets;
  p.labels = d->labels; p.kept = d->kept; p.logprobs = d->logprobs;
  double c = 1.0;
  for (int k = 1; k <= 9; ++k) p.series[9 - k] = c *= 0.69314718055994531 / k;
  p.num_labels = s->N; p.num_channels = s->C; p.words = s->words; p.unit_bits = s->unit_bits;
  constexpr int32_t kRows = 1 << 21;   // (a launch has fewer than 2^32 threads)
  for (int32_t done = 0; done < d->n;) {
    const int32_t m = std::min(kRows, d->n - done);
    p.first_row = done;
    if (d->dtype == CBD_F32) launch_sample<float>(p, m, s->stream);
    else if (d->dtype == CBD_F16) launch_sample<cbd::f16>(p, m, s->stream);
    else launch_sample<cbd::bf16>(p, m, s->stream);
    HIPCHK(hipGetLastError());
    done += m;
  }
  return CBD_OK;
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("sample_labels: ") + e.what());
}

}  // extern "C"
