// Affine layers: the weights' layout, the product kernels and their epilogue, and their part of the C ABI.  See
// include/cbd.h for the contract of each call.
#include <cmath>
#include <new>

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
  float scale, residual_scale;
};

template <int kAct> __device__ __forceinline__ float activate(float y) {
  if (kAct == CBD_ACT_RELU) return y < 0.0f ? 0.0f : y;   // (NaN stays)
  if (kAct == CBD_ACT_SIGMOID) return 1.0f / (1.0f + expf(-y));
  if (kAct == CBD_ACT_TANH) return tanhf(y);
  if (kAct == CBD_ACT_GELU) return 0.5f * y * (1.0f + erff(y * 0.70710678118654752f));
  if (kAct == CBD_ACT_SILU) return y / (1.0f + expf(-y));
  return y;
}

template <typename T> __global__ void pack_weight_kernel(const T *src, int64_t stride, T *dst, int32_t K, int32_t N) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < (int64_t)N * K) dst[i] = src[i / K * stride + i % K];
}

// The plain kernel: 16 x 16 outputs a workgroup, one each thread, operands through LDS.
template <typename T, typename O, int kAct> __global__ __launch_bounds__(256) void layer_kernel(LayerParams p) {
  __shared__ float xs[16][17], ws[16][17];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t r = (int64_t)blockIdx.y * 16 + ty;
  const int n = blockIdx.x * 16 + tx, nw = blockIdx.x * 16 + ty;
  const T *x = (const T *)p.x + (r < p.rows ? r / p.frames * p.x_cs + r % p.frames * p.x_fs : 0);
  const T *w = (const T *)p.w + (int64_t)nw * p.K;
  float acc = 0.0f;
  for (int k0 = 0; k0 < p.K; k0 += 16) {
    const int k = k0 + tx;
    xs[ty][tx] = r < p.rows && k < p.K ? (float)x[k] : 0.0f;
    ws[ty][tx] = nw < p.N && k < p.K ? (float)w[k] : 0.0f;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 16; ++j) acc = fmaf(xs[ty][j], ws[tx][j], acc);
    __syncthreads();
  }
  if (r >= p.rows || n >= p.N) return;
  const int64_t c = r / p.frames, f = r % p.frames;
  float y = p.scale * activate<kAct>(acc + (p.bias ? p.bias[n] : 0.0f));
  if (p.residual) y += p.residual_scale * (float)((const O *)p.residual)[c * p.res_cs + f * p.res_fs + n];
  ((O *)p.out)[c * p.out_cs + f * p.out_fs + n] = (O)y;
}

}  // namespace
}  // namespace cbd

struct cbd_layer {
  int device = 0;
  int32_t K = 0, N = 0, dtype = 0, act = 0;
  void *w = nullptr;
  float *bias = nullptr;
};

namespace {

using cbd::LayerParams;

template <typename T, typename O, int kAct> hipError_t launch(const LayerParams &p, hipStream_t st) {
  hipLaunchKernelGGL((cbd::layer_kernel<T, O, kAct>), dim3((p.N + 15) / 16, (p.rows + 15) / 16), dim3(256), 0, st, p);
  return hipGetLastError();
}

template <typename T, typename O> hipError_t launch_act(int act, const LayerParams &p, hipStream_t st) {
  switch (act) {
    case CBD_ACT_RELU: return launch<T, O, CBD_ACT_RELU>(p, st);
    case CBD_ACT_SIGMOID: return launch<T, O, CBD_ACT_SIGMOID>(p, st);
    case CBD_ACT_TANH: return launch<T, O, CBD_ACT_TANH>(p, st);
    case CBD_ACT_GELU: return launch<T, O, CBD_ACT_GELU>(p, st);
    case CBD_ACT_SILU: return launch<T, O, CBD_ACT_SILU>(p, st);
    default: return launch<T, O, CBD_ACT_NONE>(p, st);
  }
}

template <typename T> hipError_t launch_out(int out, int act, const LayerParams &p, hipStream_t st) {
  if (out == CBD_F32) return launch_act<T, float>(act, p, st);
  if (out == CBD_F16) return launch_act<T, cbd::f16>(act, p, st);
  return launch_act<T, cbd::bf16>(act, p, st);
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
  const int64_t total = (int64_t)l->K * l->N;
  HIPCHK(dmalloc((char **)&l->w, (size_t)total * cbd::dtype_size(l->dtype), nullptr));
  const dim3 grid((unsigned)((total + 255) / 256));
  if (l->dtype == CBD_F32)
    hipLaunchKernelGGL(cbd::pack_weight_kernel<uint32_t>, grid, dim3(256), 0, st, (const uint32_t *)desc->weight, stride,
                       (uint32_t *)l->w, l->K, l->N);
  else
    hipLaunchKernelGGL(cbd::pack_weight_kernel<uint16_t>, grid, dim3(256), 0, st, (const uint16_t *)desc->weight, stride,
                       (uint16_t *)l->w, l->K, l->N);
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
  if (rows > 0x7FFFFF00) return fail(CBD_E_INVALID, "layer_apply: too many rows");
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
  p.scale = io->scale; p.residual_scale = io->residual_scale;
  if (l->dtype == CBD_F32) HIPCHK(launch_out<float>(io->output_dtype, l->act, p, st));
  else if (l->dtype == CBD_F16) HIPCHK(launch_out<cbd::f16>(io->output_dtype, l->act, p, st));
  else HIPCHK(launch_out<cbd::bf16>(io->output_dtype, l->act, p, st));
  return CBD_OK;
} catch (const std::exception &e) {
  return fail(CBD_E_HIP, std::string("layer_apply: ") + e.what());
}

}  // extern "C"
