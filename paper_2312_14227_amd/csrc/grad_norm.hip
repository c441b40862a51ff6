// Norm of many gradients as one vector, and clipping by it (et_grad_norm, et_grad_clip, et_grad_scale).
//
// Every tensor is cut into chunks, a workgroup adds the squares of each in float64 (a conversion and a fused multiply-add, a quarter of what the vector
// units do in the time that memory takes), one launch adds the chunks: a workgroup all of them, and one for each tensor its own.  Clipping goes over the chunks once more,
// from the last to the first, so that what the norm has read last is found in the caches.  The table of tensors travels as kernel arguments: nothing is
// copied from the host.  No atomics: the order of every sum is fixed.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "context.h"
#include "op_args.h"

namespace et {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Tensors of one launch (kernel arguments: at most 4096 bytes)
constexpr int NORM_BATCH = 196, SCALE_BATCH = 140;
template <int BATCH>
struct Tensors {
  int n, first;               // how many, and the index of the first
  uint32_t chunk;             // elements of a chunk, a multiple of 16
  uint32_t begin[BATCH + 1];  // first chunk of each, counted over all launches
  const void* g[BATCH];
  uint64_t numel[BATCH];
};
struct ScaleTensors : Tensors<SCALE_BATCH> {
  void* out[SCALE_BATCH];
};

// the tensor that a chunk belongs to: as many as begin at or in front of it, less one (every wave asks for the whole table at once)
template <int BATCH>
__device__ __forceinline__ int tensor_of(const Tensors<BATCH>& t, uint32_t chunk) {
  int k = -1;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < BATCH; i += 64) k += __popcll(__ballot(i + lane < t.n && i + lane < BATCH && t.begin[i + lane < BATCH ? i + lane : 0] <= chunk));
  return __builtin_amdgcn_readfirstlane(k);
}

// A chunk as vectors that begin at multiples of 16 bytes, and single elements in front of and behind them
template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  const T* g;
  int n, head, vecs, edge;
  __device__ __forceinline__ Piece(const T* at, int count) : g(at), n(count) {
    head = min(n, (int)(-(uintptr_t)at & 15) / (int)sizeof(T));
    vecs = (n - head) / N;
    edge = n - vecs * N;
  }
  __device__ __forceinline__ int edge_at(int i) const { return i < head ? i : vecs * N + i; }
  __device__ __forceinline__ const u32x4* vec() const { return (const u32x4*)(g + head); }
};
template <typename T, int BATCH>
__device__ __forceinline__ Piece<T> piece_of(const Tensors<BATCH>& t, int k, uint32_t chunk) {
  const uint64_t off = (uint64_t)(chunk - t.begin[k]) * t.chunk;
  return Piece<T>((const T*)t.g[k] + off, (int)min((uint64_t)t.chunk, t.numel[k] - off));
}
template <typename T>
__device__ __forceinline__ float value(u32x4 v, int k) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v[k]);
  else return __uint_as_float(k & 1 ? v[k >> 1] & 0xffff0000u : v[k >> 1] << 16);
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <int WAVES>
__device__ __forceinline__ double block_sum_d(double v, double* red) {
  v = wave_sum_d(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < WAVES; w++) v += red[w];
  return v;
}

constexpr int VECS = 8;   // of a thread, on the way at once

// a thread's part of a chunk's squares
template <typename T, typename LOAD>
__device__ __forceinline__ double squares_of(const Piece<T>& p, LOAD load) {
  double s0 = 0, s1 = 0;
  for (int v0 = threadIdx.x; v0 < p.vecs; v0 += 256 * VECS) {
    u32x4 v[VECS];
#pragma unroll
    for (int i = 0; i < VECS; i++) v[i] = v0 + 256 * i < p.vecs ? load(p.vec() + v0 + 256 * i) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < VECS; i++)
#pragma unroll
      for (int e = 0; e < Piece<T>::N; e += 2) {
        const double a = (double)value<T>(v[i], e), b = (double)value<T>(v[i], e + 1);
        s0 = fma(a, a, s0);
        s1 = fma(b, b, s1);
      }
  }
  if ((int)threadIdx.x < p.edge) {
    const double a = (double)(float)p.g[p.edge_at(threadIdx.x)];
    s0 = fma(a, a, s0);
  }
  return s0 + s1;
}

template <typename T>
__global__ __launch_bounds__(256) void squares_kernel(Tensors<NORM_BATCH> t, uint32_t cached_from, double* __restrict__ part, uint32_t* __restrict__ begin) {
  __shared__ double red[4];
  const uint32_t c = t.begin[0] + blockIdx.x;
  const int k = tensor_of(t, c);
  const Piece<T> p = piece_of<T>(t, k, c);
  const double mine = c < cached_from ? squares_of(p, [](const u32x4* at) { return __builtin_nontemporal_load(at); }) : squares_of(p, [](const u32x4* at) { return *at; });
  const double s = block_sum_d<4>(mine, red);
  if (threadIdx.x == 0 && p.n > 0) part[c] = s;   // (a launch of empty tensors has a workgroup, but no chunk)
  // what the next launch needs of the table
  for (int i = blockIdx.x * 256 + threadIdx.x; i < t.n; i += gridDim.x * 256) begin[t.first + i] = t.begin[i];
}

// the same over chunks of a context's table (16-byte aligned, float32)
__global__ __launch_bounds__(256) void selected_squares_kernel(const UpdateSeg* __restrict__ segs, const uint32_t* __restrict__ selected, double* __restrict__ part) {
  __shared__ double red[4];
  const UpdateSeg sg = segs[selected[blockIdx.x]];
  const Piece<float> p(sg.g, (int)sg.n);
  const double s = block_sum_d<4>(squares_of(p, [](const u32x4* at) { return *at; }), red);   // (the update reads them again)
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// workgroup 0: the norm of all; k + 1: of tensor k
__global__ __launch_bounds__(1024) void norms_kernel(const double* __restrict__ part, const uint32_t* __restrict__ begin, int n, uint32_t chunks, float* __restrict__ norm,
                                                     float* __restrict__ tensor_norm) {
  __shared__ double red[16];
  const int k = (int)blockIdx.x - 1;
  const uint32_t from = k < 0 ? 0 : begin[k], to = k < 0 || k + 1 == n ? chunks : begin[k + 1];
  double s = 0;
#pragma unroll 4
  for (uint32_t c = from + threadIdx.x; c < to; c += 1024) s += part[c];
  s = block_sum_d<16>(s, red);
  if (threadIdx.x == 0) (k < 0 ? norm[0] : tensor_norm[k]) = (float)sqrt(s);
}

template <typename T>
__global__ __launch_bounds__(256) void scale_kernel(ScaleTensors t, const float* __restrict__ norm, float max_norm) {
  const uint32_t c = t.begin[t.n] - 1 - blockIdx.x;
  const int k = tensor_of(t, c);
  const float f = clip_scale(*norm, max_norm);
  if (f == 1.f && t.out[k] == t.g[k]) return;
  const Piece<T> p = piece_of<T>(t, k, c);
  T* const o = (T*)t.out[k] + (p.g - (const T*)t.g[k]);
  for (int v0 = threadIdx.x; v0 < p.vecs; v0 += 256 * VECS) {
    u32x4 v[VECS];
#pragma unroll
    for (int i = 0; i < VECS; i++)
      if (v0 + 256 * i < p.vecs) v[i] = p.vec()[v0 + 256 * i];
#pragma unroll
    for (int i = 0; i < VECS; i++) {
      if (v0 + 256 * i >= p.vecs) break;
      u32x4 w;
#pragma unroll
      for (int d = 0; d < 4; d++) {
        if constexpr (sizeof(T) == 4) {
          w[d] = __float_as_uint(value<T>(v[i], d) * f);
        } else {
          bf16x2 b;
          b[0] = (bf16)(value<T>(v[i], 2 * d) * f);
          b[1] = (bf16)(value<T>(v[i], 2 * d + 1) * f);
          w[d] = __builtin_bit_cast(uint32_t, b);
        }
      }
      __builtin_nontemporal_store(w, (u32x4_any*)(o + p.head) + v0 + 256 * i);
    }
  }
  if ((int)threadIdx.x < p.edge) {
    const int j = p.edge_at(threadIdx.x);
    o[j] = (T)((float)p.g[j] * f);
  }
}

}  // namespace

hipError_t selected_norm(const UpdateSeg* segs_dev, const uint32_t* selected_dev, int n_selected, double* part_dev, float* norm_dev, hipStream_t s) {
  if (n_selected < 0 || !part_dev || !norm_dev) return hipErrorInvalidValue;
  if (n_selected > 0) hipLaunchKernelGGL(selected_squares_kernel, dim3(n_selected), dim3(256), 0, s, segs_dev, selected_dev, part_dev);
  hipLaunchKernelGGL(norms_kernel, dim3(1), dim3(1024), 0, s, part_dev, nullptr, 0, (uint32_t)n_selected, norm_dev, nullptr);
  return hipGetLastError();
}

}  // namespace et

namespace {

using namespace et_op;

struct Plan {
  uint64_t total = 0, chunks = 0;
  uint32_t chunk = 4096;
};

// The chunk from which on the norm reads through the caches: what follows a norm, clipping or an update, reads the same gradients, and finds the last 192 MB in the last-level
// cache (256 MB).  86 million float32 gradients: norm and scaling 169 us, past the caches 185.  Up to 128 MB are read past the caches all the same (60 million bf16:
// 24 us, through them 26), as is what lies in front of the last 192 MB of more (303 million float32: 188 and 208).  That is the norm's side of it.  With the scaling that follows, calls of
// up to 128 MB would gain through the caches (float32 into other outputs: 10 million 24.5 us instead of 29.5, 30 million 65.6 instead of 72.2; 30 million in place 77.7 instead of 80.3), and calls
// that find nothing to scale would lose (2.5 million 10.5 instead of 9.7, 30 million 28.8 instead of 25.8).
uint32_t cached_from(const Plan& p, size_t size) {
  const double bytes = (double)p.total * size;
  if (bytes <= 128e6) return UINT32_MAX;
  const uint64_t kept = (uint64_t)(192e6 / ((double)p.chunk * size));
  return p.chunks > kept ? (uint32_t)(p.chunks - kept) : 0;
}

// False: a size that no memory holds.  Chunks of 64 KB where there are enough of them, so that a workgroup's beginning and end are a small part of it;
// smaller ones spread few elements over the chip (200 000 float32: 49 workgroups of 4096, 5.1 us, or 13 of 16384, 5.6); larger ones keep the sums of chunks few.
bool make_plan(int32_t n, const uint64_t* numel, Plan* p) {
  for (int32_t i = 0; i < n; i++) {
    if (numel[i] > (1ull << 48) || (p->total += numel[i]) > (1ull << 48)) return false;
  }
  while (p->chunk < 16384 && p->total / p->chunk > 1024) p->chunk *= 2;
  while (p->chunk < (1u << 30) && p->total / p->chunk > 65536) p->chunk *= 2;
  for (int32_t i = 0; i < n; i++) p->chunks += (numel[i] + p->chunk - 1) / p->chunk;
  return p->chunks < (1ull << 31);
}
size_t ws_bytes(int32_t n, const Plan& p) { return 64 + sizeof(double) * (size_t)p.chunks + sizeof(uint32_t) * (size_t)n; }

// Whether what is written (out, or in place: grad) meets anything that another tensor reads or writes.  Tensors of an arena, in its order, are seen to be apart in one pass.
bool apart(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, size_t size) {
  struct Piece {
    uintptr_t begin, end;
    bool written;
  };
  uintptr_t last = 0;
  bool ascending = true;
  for (int32_t i = 0; i < n && ascending; i++) {
    if (numel[i] == 0) continue;
    const uintptr_t at = reinterpret_cast<uintptr_t>(grad[i]);
    ascending = (!out || out[i] == grad[i]) && at >= last;
    last = at + numel[i] * size;
  }
  if (ascending) return true;
  std::vector<Piece> all;
  all.reserve(2 * (size_t)n);
  for (int32_t i = 0; i < n; i++) {
    if (numel[i] == 0) continue;
    const uintptr_t g = reinterpret_cast<uintptr_t>(grad[i]), o = out ? reinterpret_cast<uintptr_t>(out[i]) : g;
    all.push_back({o, o + numel[i] * size, true});
    if (o != g) all.push_back({g, g + numel[i] * size, false});
  }
  std::sort(all.begin(), all.end(), [](const Piece& a, const Piece& b) { return a.begin < b.begin; });
  uintptr_t read = 0, written = 0;   // where what begins at or in front of a piece ends
  for (const Piece& p : all) {
    if (p.begin < written || (p.written && p.begin < read)) return false;
    uintptr_t& end = p.written ? written : read;
    end = std::max(end, p.end);
  }
  return true;
}

// writes: whether tensors are scaled (in place, if out is null)
int check_tensors(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, int32_t dtype, const float* norm, bool writes) {
  if (n < 0 || n > 1 << 21 || (n > 0 && (!grad || !numel)) || !type_ok(dtype) || !norm || !aligned(norm, 4)) return ET_EINVAL;
  const size_t size = type_size(dtype);
  for (int32_t i = 0; i < n; i++) {
    if (numel[i] == 0) continue;
    const void* o = out ? out[i] : grad[i];
    if (!grad[i] || !o || !aligned(grad[i], size) || !aligned(o, size) || numel[i] > (1ull << 48)) return ET_EINVAL;
  }
  try {
    return !writes || apart(n, grad, out, numel, size) ? ET_OK : ET_EINVAL;
  } catch (const std::bad_alloc&) {
    return ET_ENOMEM;
  }
}

// fills the table of the launch that begins with tensor `first`; next: its first chunk, and what follows its last
template <int BATCH>
void fill(et::Tensors<BATCH>* t, int32_t n, int32_t first, const void* const* grad, const uint64_t* numel, const Plan& p, uint32_t* next) {
  t->n = std::min<int32_t>(BATCH, n - first);
  t->first = first;
  t->chunk = p.chunk;
  for (int k = 0; k < t->n; k++) {
    t->begin[k] = *next;
    t->g[k] = grad[first + k];
    t->numel[k] = numel[first + k];
    *next += (uint32_t)((numel[first + k] + p.chunk - 1) / p.chunk);
  }
  t->begin[t->n] = *next;
}

void norm_launch(int32_t n, const void* const* grad, const uint64_t* numel, int32_t dtype, const Plan& p, void* ws, hipStream_t s, float* norm,
                 float* tensor_norm) {
  double* part = (double*)ws;
  uint32_t* begin = (uint32_t*)(part + p.chunks);
  uint32_t next = 0;
  const uint32_t cached = cached_from(p, type_size(dtype));
  for (int32_t first = 0; first < n; first += et::NORM_BATCH) {
    et::Tensors<et::NORM_BATCH> t;
    fill(&t, n, first, grad, numel, p, &next);
    const uint32_t grid = std::max(1u, next - t.begin[0]);
    if (dtype == ET_BF16) hipLaunchKernelGGL(et::squares_kernel<bf16>, dim3(grid), dim3(256), 0, s, t, cached, part, begin);
    else hipLaunchKernelGGL(et::squares_kernel<float>, dim3(grid), dim3(256), 0, s, t, cached, part, begin);
  }
  hipLaunchKernelGGL(et::norms_kernel, dim3(tensor_norm ? n + 1 : 1), dim3(1024), 0, s, part, begin, n, (uint32_t)p.chunks, norm, tensor_norm);
}

void scale_launch(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, int32_t dtype, const Plan& p, const float* norm, float max_norm,
                  hipStream_t s) {
  for (int32_t i = (n - 1) / et::SCALE_BATCH; n > 0 && i >= 0; i--) {
    et::ScaleTensors t;
    uint32_t next = 0;
    const int32_t first = i * et::SCALE_BATCH;
    fill(&t, n, first, grad, numel, p, &next);
    for (int k = 0; k < t.n; k++) t.out[k] = out ? out[first + k] : const_cast<void*>(grad[first + k]);
    if (!next) continue;
    if (dtype == ET_BF16) hipLaunchKernelGGL(et::scale_kernel<bf16>, dim3(next), dim3(256), 0, s, t, norm, max_norm);
    else hipLaunchKernelGGL(et::scale_kernel<float>, dim3(next), dim3(256), 0, s, t, norm, max_norm);
  }
}

// max_norm < 0: the norm only
int norm_and_clip(int32_t n, const void* const* grad, void* const* out, const uint64_t* numel, int32_t dtype, float max_norm, void* ws, size_t bytes,
                  void* hip_stream, float* norm, float* tensor_norm) {
  const int rc = check_tensors(n, grad, out, numel, dtype, norm, max_norm >= 0);
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
  return n < 0 || n > 1 << 21 || (n > 0 && !numel) || !make_plan(n, numel, &p) ? 0 : ws_bytes(n, p);
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
  const int rc = check_tensors(n, grad_dev, out_dev, numel, dtype, norm_dev, true);
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
