// Norm of many gradients as one vector, and clipping by it (et_grad_norm, et_grad_clip).
//
// Every tensor is cut into chunks, a workgroup per chunk adds its squares in float64, a wave per tensor adds its chunks, one workgroup adds the
// tensors and derives the coefficient; clipping then goes over the chunks once more.  The table of tensors travels as kernel
// arguments: nothing is copied from the host.  No atomics: the order of every sum is fixed.
#include <cmath>

#include "context.h"
#include "op_args.h"

namespace et {
namespace {

constexpr int BATCH = 120;   // tensors per launch (kernel arguments: 32 bytes each)
struct Tensors {
  int n, first;              // tensors of this launch, and the index of the first
  uint32_t chunk;            // elements of a chunk
  uint32_t begin[BATCH + 1]; // first chunk of each, counted over all launches
  const void* g[BATCH];
  void* out[BATCH];
  uint64_t numel[BATCH];
};

// the tensor that a chunk belongs to: the last that begins at or in front of it and is not empty
__device__ __forceinline__ int tensor_of(const Tensors& t, uint32_t chunk) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.begin[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ double block_sum_d(double v, double* red) {
  v = wave_sum_d(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void squares_kernel(Tensors t, double* __restrict__ part) {
  __shared__ double red[4];
  const uint32_t c = t.begin[0] + blockIdx.x;
  const int k = tensor_of(t, c);
  const uint64_t off = (uint64_t)(c - t.begin[k]) * t.chunk;
  const T* g = (const T*)t.g[k] + off;
  const uint32_t n = (uint32_t)min((uint64_t)t.chunk, t.numel[k] - off);
  double s = 0;
  for (uint32_t i = threadIdx.x; i < n; i += 256) {
    const double v = (double)(float)g[i];
    s += v * v;
  }
  s = block_sum_d(s, red);
  if (threadIdx.x == 0) part[c] = s;
}

__global__ __launch_bounds__(64) void tensor_kernel(Tensors t, const double* __restrict__ part, double* __restrict__ squares, float* __restrict__ norm) {
  const int k = blockIdx.x;
  double s = 0;
  for (uint32_t c = t.begin[k] + threadIdx.x; c < t.begin[k + 1]; c += 64) s += part[c];
  s = wave_sum_d(s);
  if (threadIdx.x == 0) {
    squares[t.first + k] = s;
    if (norm) norm[t.first + k] = (float)sqrt(s);
  }
}

__global__ __launch_bounds__(256) void norm_kernel(const double* __restrict__ squares, int n, float* __restrict__ norm) {
  __shared__ double red[4];
  double s = 0;
  for (int i = threadIdx.x; i < n; i += 256) s += squares[i];
  s = block_sum_d(s, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

__device__ __forceinline__ float clip_scale(float norm, float max_norm) {
  return isfinite(norm) && norm > max_norm ? (float)((double)max_norm / (double)norm) : 1.f;
}

template <typename T>
__global__ __launch_bounds__(256) void scale_kernel(Tensors t, const float* __restrict__ norm, float max_norm) {
  const uint32_t c = t.begin[0] + blockIdx.x;
  const int k = tensor_of(t, c);
  const float f = clip_scale(*norm, max_norm);
  if (f == 1.f && t.out[k] == t.g[k]) return;
  const uint64_t off = (uint64_t)(c - t.begin[k]) * t.chunk;
  const T* g = (const T*)t.g[k] + off;
  T* o = (T*)t.out[k] + off;
  const uint32_t n = (uint32_t)min((uint64_t)t.chunk, t.numel[k] - off);
  for (uint32_t i = threadIdx.x; i < n; i += 256) o[i] = f == 1.f ? g[i] : (T)((float)g[i] * f);
}

}  // namespace
}  // namespace et

namespace {

using namespace et_op;

struct Plan {
  uint64_t total = 0, chunks = 0;
  uint32_t chunk = 16384;
};

// false: a size that no memory holds
bool make_plan(int32_t n, const uint64_t* numel, Plan* p) {
  for (int32_t i = 0; i < n; i++) {
    if (numel[i] > (1ull << 48) || (p->total += numel[i]) > (1ull << 48)) return false;
  }
  while (p->chunk < (1u << 30) && p->total / p->chunk > 65536) p->chunk *= 2;
  for (int32_t i = 0; i < n; i++) p->chunks += (numel[i] + p->chunk - 1) / p->chunk;
  return p->chunks < (1ull << 31);
}
size_t ws_bytes(int32_t n, const Plan& p) { return 64 + sizeof(double) * ((size_t)n + p.chunks); }

int check_tensors(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, int32_t dtype, const float* norm) {
  if (n < 0 || (n > 0 && (!grad || !numel)) || !type_ok(dtype) || !norm || !aligned(norm, 4)) return ET_EINVAL;
  const size_t size = type_size(dtype);
  for (int32_t i = 0; i < n; i++) {
    if (numel[i] == 0) continue;
    const void* o = out ? out[i] : grad[i];
    if (!grad[i] || !o || !aligned(grad[i], size) || !aligned(o, size) || numel[i] > (1ull << 48)) return ET_EINVAL;
    if (o != grad[i] && Span(grad[i], 1, (int64_t)numel[i], 0, size).meets(Span(o, 1, (int64_t)numel[i], 0, size))) return ET_EINVAL;
  }
  return ET_OK;
}

// calls f(table, workgroups) for every launch over the chunks
template <typename F>
void each_batch(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, const Plan& p, F f) {
  uint32_t next = 0;
  for (int32_t i0 = 0; i0 < n; i0 += et::BATCH) {
    et::Tensors t;
    t.n = std::min<int32_t>(et::BATCH, n - i0);
    t.first = i0;
    t.chunk = p.chunk;
    for (int k = 0; k < t.n; k++) {
      t.begin[k] = next;
      t.g[k] = grad[i0 + k];
      t.out[k] = out ? out[i0 + k] : const_cast<void*>(grad[i0 + k]);
      t.numel[k] = numel[i0 + k];
      next += (uint32_t)((numel[i0 + k] + p.chunk - 1) / p.chunk);
    }
    t.begin[t.n] = next;
    f(t, next - t.begin[0]);
  }
}

void norm_launch(int32_t n, const void* const* grad, const uint64_t* numel, int32_t dtype, const Plan& p, void* ws, hipStream_t s, float* norm,
                 float* tensor_norm) {
  double* squares = (double*)ws;
  double* part = squares + n;
  each_batch(n, grad, nullptr, numel, p, [&](const et::Tensors& t, uint32_t grid) {
    if (grid) {
      if (dtype == ET_BF16) hipLaunchKernelGGL(et::squares_kernel<bf16>, dim3(grid), dim3(256), 0, s, t, part);
      else hipLaunchKernelGGL(et::squares_kernel<float>, dim3(grid), dim3(256), 0, s, t, part);
    }
    hipLaunchKernelGGL(et::tensor_kernel, dim3(t.n), dim3(64), 0, s, t, part, squares, tensor_norm);
  });
  hipLaunchKernelGGL(et::norm_kernel, dim3(1), dim3(256), 0, s, squares, n, norm);
}

void scale_launch(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, int32_t dtype, const Plan& p, const float* norm, float max_norm,
                  hipStream_t s) {
  each_batch(n, grad, out, numel, p, [&](const et::Tensors& t, uint32_t grid) {
    if (!grid) return;
    if (dtype == ET_BF16) hipLaunchKernelGGL(et::scale_kernel<bf16>, dim3(grid), dim3(256), 0, s, t, norm, max_norm);
    else hipLaunchKernelGGL(et::scale_kernel<float>, dim3(grid), dim3(256), 0, s, t, norm, max_norm);
  });
}

// max_norm < 0: the norm only
int norm_and_clip(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, int32_t dtype, float max_norm, void* ws, size_t bytes,
                  void* hip_stream, float* norm, float* tensor_norm) {
  const int rc = check_tensors(n, grad, out, numel, dtype, norm);
  if (rc != ET_OK) return rc;
  if (!ws || !aligned(ws, 16) || !aligned(tensor_norm, 4)) return ET_EINVAL;
  Plan p;
  if (!make_plan(n, numel, &p)) return ET_EINVAL;
  if (bytes < ws_bytes(n, p)) return ET_ENOMEM;
  const hipStream_t s = (hipStream_t)hip_stream;
  const OnDeviceOf on(s);
  if (!on.ok) return ET_EHIP;
  norm_launch(n, grad, numel, dtype, p, ws, s, norm, tensor_norm);
  if (max_norm >= 0) scale_launch(n, grad, out, numel, dtype, p, norm, max_norm, s);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

}  // namespace

extern "C" {

size_t et_grad_norm_ws_bytes(int32_t n, const uint64_t* numel) {
  Plan p;
  return n < 0 || (n > 0 && !numel) || !make_plan(n, numel, &p) ? 0 : ws_bytes(n, p);
}

int et_grad_norm(int32_t n, const void* const* grad_dev, const uint64_t* numel, int32_t dtype, void* workspace_dev, size_t workspace_bytes,
                 void* hip_stream, float* norm_dev, float* tensor_norm_dev) {
  return norm_and_clip(n, grad_dev, nullptr, numel, dtype, -1.f, workspace_dev, workspace_bytes, hip_stream, norm_dev, tensor_norm_dev);
}

int et_grad_clip(int32_t n, const void* const* grad_dev, void* const* out_dev, const uint64_t* numel, int32_t dtype, float max_norm,
                 void* workspace_dev, size_t workspace_bytes, void* hip_stream, float* norm_dev, float* tensor_norm_dev) {
  if (!(max_norm >= 0)) return ET_EINVAL;
  return norm_and_clip(n, grad_dev, out_dev, numel, dtype, max_norm, workspace_dev, workspace_bytes, hip_stream, norm_dev, tensor_norm_dev);
}

int et_grad_scale(int32_t n, const void* const* grad_dev, void* const* out_dev, const uint64_t* numel, int32_t dtype, const float* norm_dev, float max_norm,
                  void* hip_stream) {
  if (!(max_norm >= 0)) return ET_EINVAL;
  const int rc = check_tensors(n, grad_dev, out_dev, numel, dtype, norm_dev);
  if (rc != ET_OK) return rc;
  Plan p;
  if (!make_plan(n, numel, &p)) return ET_EINVAL;
  const hipStream_t s = (hipStream_t)hip_stream;
  const OnDeviceOf on(s);
  if (!on.ok) return ET_EHIP;
  scale_launch(n, grad_dev, out_dev, numel, dtype, p, norm_dev, max_norm, s);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

}  // extern "C"
