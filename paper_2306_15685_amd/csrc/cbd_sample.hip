// Drawing labels from rows of scores: the kernels, the channels' lists of boosted labels, and their part of the C ABI.
// See include/cbd.h for the rule and the contract of each call.
#include <cmath>
#include <cstring>
#include <new>
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
  int32_t num_labels, num_channels, words;   // words: 32-bit words of a channel's bits
  int32_t unit_bits;         // weights are summed in units of 2^-unit_bits
};

constexpr int kThreads = 256;

// Order of scores as unsigned integers: larger score, larger key; 0 = masked (-inf or NaN); -0 is +0.
__device__ __forceinline__ uint32_t score_key(float x) {
  if (!(x > -__builtin_inff())) return 0u;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_score(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

template <typename T> struct Row {
  const T *scores;
  const uint32_t *bits;
  float offset;
  __device__ __forceinline__ uint32_t key(int i) const {
    float x = (float)scores[i];
    if (bits[i >> 5] >> (i & 31) & 1u) x += offset;
    return score_key(x);
  }
};

// Weights as integers: exp((x - best) / temperature) in units of 2^-unit_bits.
struct Weigher {
  double best, inv_t, unit;
  __device__ __forceinline__ double log_weight(uint32_t key) const {
    const double x = (double)key_score(key);
    return x == best ? 0.0 : (x - best) * inv_t;
  }
  __device__ __forceinline__ uint64_t units(double w) const { return __double2ull_rn(w * unit); }
};

template <typename V, typename Op> __device__ V block_reduce(V v, V *lds, Op op) {
  __syncthreads();
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int s = kThreads / 2; s > 0; s >>= 1) {
    if ((int)threadIdx.x < s) lds[threadIdx.x] = op(lds[threadIdx.x], lds[threadIdx.x + s]);
    __syncthreads();
  }
  v = lds[0];
  __syncthreads();
  return v;
}

template <typename T> __global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p) {
  __shared__ uint64_t red[kThreads];
  __shared__ uint64_t hist_mass[256];
  __shared__ uint32_t hist_count[256];
  __shared__ uint64_t pick[4];
  const int r = blockIdx.x, tid = threadIdx.x, N = p.num_labels;
  const int ch = p.channels ? p.channels[r] : r;
  auto write = [&](int label, float lp, int kept) {
    if (tid == 0) {
      p.labels[r] = label;
      if (p.logprobs) p.logprobs[r] = lp;
      if (p.kept) p.kept[r] = kept;
    }
  };
  if (ch < 0 || ch >= p.num_channels) { write(-1, -__builtin_inff(), 0); return; }
  const Row<T> row{(const T *)p.scores + (int64_t)r * p.row_stride, p.bits + (int64_t)ch * p.words, p.offsets[ch]};
  auto max64 = [](uint64_t a, uint64_t b) { return a > b ? a : b; };
  auto add64 = [](uint64_t a, uint64_t b) { return a + b; };
  // the first of the order: largest key, then lowest label
  uint64_t top = 0;
  for (int i = tid; i < N; i += kThreads) top = max64(top, (uint64_t)row.key(i) << 32 | (uint32_t)~i);
  top = block_reduce(top, red, max64);
  const uint32_t key_best = (uint32_t)(top >> 32);
  if (key_best == 0) { write(-1, -__builtin_inff(), 0); return; }
  const float temperature = p.temperature ? p.temperature[r] : 1.0f;
  if (!(temperature > 0.0f)) { write((int)~(uint32_t)top, 0.0f, 1); return; }
  const float best = key_score(key_best);
  const Weigher wt{(double)best, 1.0 / (double)temperature, ldexp(1.0, p.unit_bits)};
  const uint32_t lowest = best == __builtin_inff() ? key_best : 1u;   // smaller keys are masked
  // kept so far: keys above `cut`, and the first `ties` labels (by label) with key `cut`
  uint32_t cut = lowest, ties = 0xFFFFFFFFu;
  // finds the key at which the running count (by_mass false) or mass, from the best downwards, reaches `want`
  auto descend = [&](bool by_mass, double want, uint64_t *above) {
    uint32_t prefix = 0;
    uint64_t before = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist_mass[tid] = 0; hist_count[tid] = 0;
      __syncthreads();
      for (int i = tid; i < N; i += kThreads) {
        const uint32_t k = row.key(i);
        if (k < lowest || (shift < 24 && (k >> (shift + 8)) != (prefix >> (shift + 8)))) continue;
        const uint32_t b = k >> shift & 255u;
        atomicAdd(&hist_count[b], 1u);
        if (by_mass) atomicAdd((unsigned long long *)&hist_mass[b], (unsigned long long)wt.units(exp(wt.log_weight(k))));
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t run = before;
        int b = 255, last = -1;
        for (; b >= 0; --b) {
          if (hist_count[b] == 0) continue;
          last = b;
          const uint64_t next = run + (by_mass ? hist_mass[b] : (uint64_t)hist_count[b]);
          if ((double)next >= want) break;
          run = next;
        }
        if (b < 0) { b = last; run -= by_mass ? hist_mass[b] : (uint64_t)hist_count[b]; }
        pick[0] = (uint64_t)b; pick[1] = run;
      }
      __syncthreads();
      prefix |= (uint32_t)pick[0] << shift;
      before = pick[1];
      __syncthreads();
    }
    *above = before;
    return prefix;
  };
  const int k = p.top_k ? p.top_k[r] : 0;
  if (k > 0 && k < N) {
    uint64_t above = 0;
    uint64_t valid = 0;
    for (int i = tid; i < N; i += kThreads) valid += row.key(i) >= lowest;
    valid = block_reduce(valid, red, add64);
    if ((uint64_t)k < valid) {
      cut = descend(false, (double)k, &above);
      ties = (uint32_t)((uint64_t)k - above);
    }
  }
  // mass and number of what is kept: keys above `cut`, and ties
  auto kept_mass = [&](double min_weight, uint64_t *mass, uint64_t *count, uint64_t *n_ties) {
    uint64_t m = 0, c = 0, t = 0;
    for (int i = tid; i < N; i += kThreads) {
      const uint32_t key = row.key(i);
      if (key < cut) continue;
      const double w = exp(wt.log_weight(key));
      if (w < min_weight) continue;
      if (key == cut) { ++t; continue; }
      m += wt.units(w); ++c;
    }
    *mass = block_reduce(m, red, add64);
    *count = block_reduce(c, red, add64);
    *n_ties = block_reduce(t, red, add64);
  };
  uint64_t mass, count, n_ties;
  const float top_p = p.top_p ? p.top_p[r] : 1.0f;
  if (top_p <= 0.0f) {
    cut = key_best; ties = 1;
  } else if (top_p < 1.0f) {
    kept_mass(0.0, &mass, &count, &n_ties);
    const uint64_t w_cut = wt.units(exp(wt.log_weight(cut)));
    const uint64_t all = mass + (n_ties < ties ? n_ties : (uint64_t)ties) * w_cut;
    const double want = (double)top_p * (double)all;
    uint64_t above = 0;
    const uint32_t c2 = descend(true, want, &above);
    const uint64_t w2 = wt.units(exp(wt.log_weight(c2)));
    // ties j = 0, 1, ... are kept while above + j * w2 < want
    uint32_t t2 = 0xFFFFFFFFu;
    if (w2 > 0) {
      const double j = ceil((want - (double)above) / (double)w2);
      t2 = j < 1.0 ? 1u : j < 4e9 ? (uint32_t)j : 0xFFFFFFFFu;
    }
    if (c2 > cut) { cut = c2; ties = t2; }
    else if (c2 == cut && t2 < ties) ties = t2;
  }
  const float min_p = p.min_p ? p.min_p[r] : 0.0f;
  const double min_weight = min_p > 0.0f ? (double)fminf(min_p, 1.0f) : 0.0;
  kept_mass(min_weight, &mass, &count, &n_ties);
  const uint64_t w_cut = wt.units(exp(wt.log_weight(cut)));
  const uint64_t kept_ties = n_ties < ties ? n_ties : (uint64_t)ties;
  const uint64_t total = mass + kept_ties * w_cut;
  float u = p.random[r];
  if (!(u > 0.0f)) u = 0.0f;
  uint64_t target = (uint64_t)((double)u * (double)total);
  if (target >= total) target = total - 1;
  // the label, found by one thread going through the row
  if (tid == 0) {
    uint64_t run = 0, seen = 0;
    int label = -1;
    uint32_t at = 0;
    for (int i = 0; i < N; ++i) {
      const uint32_t key = row.key(i);
      if (key < cut) continue;
      if (key == cut && seen++ >= ties) continue;
      const double w = exp(wt.log_weight(key));
      if (w < min_weight) continue;
      run += wt.units(w);
      if (run > target || (u == 0.0f && w > 0.0)) { label = i; at = key; break; }
    }
    p.labels[r] = label;
    if (p.logprobs) p.logprobs[r] = (float)(wt.log_weight(at) - log((double)total / wt.unit));
    if (p.kept) p.kept[r] = (int32_t)(count + kept_ties);
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
}

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
  s->unit_bits = 62 - log2;   // num_labels weights of at most 1 stay below 2^63
  s->seen.assign((size_t)num_channels, 0);
  const size_t n = (size_t)num_channels * (size_t)s->words;
  HIPCHK(dmalloc(&s->bits, n, nullptr));
  HIPCHK(dmalloc(&s->offsets, (size_t)num_channels, nullptr));
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
  for (int32_t i0 = 0; i0 < n_channels; i0 += kUpload) {
    const int32_t m = std::min(kUpload, n_channels - i0);
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
  for (int32_t k0 = 0; k0 < total; k0 += kUpload) {
    const int32_t m = std::min(kUpload, total - k0);
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
  p.num_labels = s->N; p.num_channels = s->C; p.words = s->words; p.unit_bits = s->unit_bits;
  const dim3 grid((unsigned)d->n), block(cbd::kThreads);
  if (d->dtype == CBD_F32) hipLaunchKernelGGL(cbd::sample_kernel<float>, grid, block, 0, s->stream, p);
  else if (d->dtype == CBD_F16) hipLaunchKernelGGL(cbd::sample_kernel<cbd::f16>, grid, block, 0, s->stream, p);
  else hipLaunchKernelGGL(cbd::sample_kernel<cbd::bf16>, grid, block, 0, s->stream, p);
  HIPCHK(hipGetLastError());
  return CBD_OK;
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("sample_labels: ") + e.what());
}

}  // extern "C"
