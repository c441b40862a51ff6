// Losses of log probabilities over rows of logits, with their gradients: the clipped policy loss with a divergence term, and the
// preference loss of pairs of sequences (et_policy_loss, et_preference_loss).
//
// Both need of a row the softmax statistics m = max x and S = sum exp(x - m), from which log p[a] = x[a] - m - log S, and give
// it a gradient that is a multiple of [j = a] - p[j] (the exact divergence adds p[j] times a log ratio).  What multiple it is follows
// from the row alone (policy) or from the sums over both sequences of its pair (preference).
// The label's own term is left out of the sum, S = rest + exp(x[a] - m): 1 - p[a] = rest / S, its gradient, and log p[a] = -log1p(rest / exp(x[a] - m)) are
// exact to rounding also where p[a] is close to 1.
#include <cmath>

#include "context.h"
#include "op_args.h"

namespace et {
namespace {

constexpr int MAX_GRID = 2048;   // workgroups of the row kernels; each leaves one line of partial sums

template <typename T>
__device__ __forceinline__ float as_float(T v) { return (float)v; }

__device__ __forceinline__ void put(void* row, bool bf16_out, long long j, float v) {
  if (bf16_out) ((bf16*)row)[j] = (bf16)v;
  else ((float*)row)[j] = v;
}

// ---- sums over a workgroup of 256 threads, the same in every thread
template <typename F>
__device__ __forceinline__ float block_reduce(float v, float* red, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return f(f(red[0], red[1]), f(red[2], red[3]));
}
__device__ __forceinline__ float block_max(float v, float* red) {
  return block_reduce(v, red, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float block_sum(float v, float* red) {
  return block_reduce(v, red, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ double block_sum_d(double v, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

struct Stat {
  float m, s, rest;   // max x, sum exp(x - m), and that sum without the label's term; s = 0: every x is minus infinity
};
// exp(x - m): m = -inf stands for a row of minus infinities
__device__ __forceinline__ float exp_of(float x, float m) { return __expf(x - (m == -INFINITY ? 0.f : m)); }

template <typename T>
__device__ Stat row_stat(const T* x, int C, int at, float* red) {
  float m = -INFINITY;
  for (int j = threadIdx.x; j < C; j += 256) m = fmaxf(m, as_float(x[j]));
  m = block_max(m, red);
  float s = 0.f;
  for (int j = threadIdx.x; j < C; j += 256)
    if (j != at) s += exp_of(as_float(x[j]), m);
  s = block_sum(s, red);
  return {m, s + (at < 0 ? 0.f : exp_of(as_float(x[at]), m)), s};
}

__device__ __forceinline__ double log_prob(const Stat& s, float xa) {
  const float e = exp_of(xa, s.m);
  return e > s.rest ? -log1p((double)s.rest / (double)e) : ((double)xa - (double)s.m) - log((double)s.s);
}

struct RowArgs {
  const void* logits;
  long long ld;
  const int32_t* label;
  void* grad;
  long long gld;
  int rows, classes, grad_bf16;
};

struct PolicyArgs {
  const float *old_logp, *advantage, *ref_logp, *weight;
  const void* ref;
  long long ref_ld;
  double low, high, kl_coef;   // borders of the ratio
  float* logp;
};

// what a row's scalars come to: gradient = g ([j = a] - p[j])
struct PolicyRow {
  double surrogate, kl, clipped, g;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& p, int r, double lp, double kl) {
  const double A = (double)p.advantage[r], ratio = exp(lp - (double)p.old_logp[r]);
  const bool over = (A > 0 && ratio > p.high) || (A < 0 && ratio < p.low);
  PolicyRow o;
  o.clipped = over ? 1.0 : 0.0;
  o.surrogate = A * (over ? (A > 0 ? p.high : p.low) : ratio);
  o.g = over ? 0.0 : -ratio * A;
  o.kl = kl;
  if (p.ref_logp) {
    const double d = (double)p.ref_logp[r] - lp, e = expm1(d);
    o.kl = e == INFINITY ? INFINITY : e - d;
    if (p.kl_coef != 0) o.g -= p.kl_coef * e;
  }
  return o;
}

__global__ __launch_bounds__(256) void count_kernel(const int32_t* __restrict__ label, int rows, int classes, double* __restrict__ count) {
  __shared__ double red[4];
  double n = 0;
  for (int r = threadIdx.x; r < rows; r += 256) n += (unsigned)label[r] < (unsigned)classes ? 1.0 : 0.0;
  n = block_sum_d(n, red);
  if (threadIdx.x == 0) *count = n;
}

template <typename T, bool FULL>
__global__ __launch_bounds__(256) void policy_kernel(RowArgs a, PolicyArgs p, const double* __restrict__ count, double* __restrict__ parts) {
  __shared__ float red[4];
  double sum[4] = {0, 0, 0, 0};
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.logits + (long long)r * a.ld;
    unsigned char* out = a.grad ? (unsigned char*)a.grad + (long long)r * a.gld * (a.grad_bf16 ? 2 : 4) : nullptr;
    const int at = a.label[r];
    if ((unsigned)at >= (unsigned)a.classes) {
      if (p.logp && threadIdx.x == 0) p.logp[r] = 0.f;
      if (out)
        for (int j = threadIdx.x; j < a.classes; j += 256) put(out, a.grad_bf16, j, 0.f);
      continue;
    }
    const float xa = as_float(x[at]);
    const Stat s = row_stat(x, a.classes, at, red);
    const bool none = s.s == 0.f;
    const double lp = none ? -INFINITY : log_prob(s, xa);
    if (p.logp && threadIdx.x == 0) p.logp[r] = (float)lp;
    if (none) {
      if (out)
        for (int j = threadIdx.x; j < a.classes; j += 256) put(out, a.grad_bf16, j, 0.f);
      continue;
    }
    const T* y = nullptr;
    float apart = 0.f;   // log sum exp x - log sum exp y
    double kl = 0;
    if (FULL) {
      y = (const T*)p.ref + (long long)r * p.ref_ld;
      const Stat q = row_stat(y, a.classes, -1, red);
      apart = (float)(((double)s.m - (double)q.m) + (log((double)s.s) - log((double)q.s)));
      float t = 0.f;
      for (int j = threadIdx.x; j < a.classes; j += 256) {
        const float e = exp_of(as_float(x[j]), s.m);
        t += e == 0.f ? 0.f : e * (as_float(x[j]) - as_float(y[j]) - apart);
      }
      kl = (double)block_sum(t, red) / (double)s.s;
    }
    const PolicyRow row = policy_row(p, r, lp, kl);
    const double w = p.weight ? (double)p.weight[r] : 1.0 / *count;
    sum[0] += w * ((p.kl_coef != 0 ? p.kl_coef * row.kl : 0.0) - row.surrogate);
    sum[1] += w * row.surrogate;
    sum[2] += w * row.kl;
    sum[3] += w * row.clipped;
    if (!out) continue;
    const float cf = (float)(-w * row.g / (double)s.s), ck = (float)(w * p.kl_coef / (double)s.s), k = (float)kl;
    const float own = (float)(w * row.g * ((double)s.rest / (double)s.s));
    __syncthreads();   // (in place: every thread has read the label's logit)
    for (int j = threadIdx.x; j < a.classes; j += 256) {
      const float xj = as_float(x[j]), e = exp_of(xj, s.m);
      float v = j == at ? own : cf * e;
      if (FULL && ck != 0.f && e != 0.f) v += ck * e * (xj - as_float(y[j]) - apart - k);
      put(out, a.grad_bf16, j, v);
    }
  }
  if (threadIdx.x == 0)
#pragma unroll
    for (int i = 0; i < 4; i++) parts[4 * blockIdx.x + i] = sum[i];
}

// adds the lines of partial sums: out[0] = scale * column 0, more[i - 1] = scale * column i
template <int COLS>
__global__ __launch_bounds__(256) void finish_kernel(const double* __restrict__ parts, int lines, double scale, float* __restrict__ out,
                                                     float* __restrict__ more) {
  __shared__ double red[4];
#pragma unroll
  for (int i = 0; i < COLS; i++) {
    double v = 0;
    for (int l = threadIdx.x; l < lines; l += 256) v += parts[COLS * l + i];
    v = block_sum_d(v, red) * scale;
    if (threadIdx.x == 0) {
      if (i == 0) *out = (float)v;
      else if (more) more[i - 1] = (float)v;
    }
  }
}

// ---- preference
struct Sequences {
  const int32_t* offsets;   // or null: every row is one
  int rows, n;
  __device__ __forceinline__ int at(int i) const { return offsets ? min(max(offsets[i], 0), rows) : i; }
};
struct SeqRows {   // per row, in the workspace
  float *m, *s, *rest;
  double* lp;
  float* g;        // the gradient is g ([j = a] - p[j])
};

template <typename T>
__global__ __launch_bounds__(256) void row_stats_kernel(RowArgs a, Sequences seq, SeqRows o) {
  __shared__ float red[4];
  const int begin = seq.at(0), end = seq.at(seq.n);
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int at = a.label[r];
    Stat s = {0.f, 0.f, 0.f};
    double lp = 0;
    if (r >= begin && r < end && (unsigned)at < (unsigned)a.classes) {
      const T* x = (const T*)a.logits + (long long)r * a.ld;
      s = row_stat(x, a.classes, at, red);
      if (s.s != 0.f) lp = log_prob(s, as_float(x[at]));
    }
    if (threadIdx.x == 0) {
      o.m[r] = s.m;
      o.s[r] = s.s;
      o.rest[r] = s.rest;
      o.lp[r] = lp;
      o.g[r] = 0.f;
    }
  }
}

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

__global__ __launch_bounds__(256) void pair_kernel(Sequences seq, SeqRows o, const float* __restrict__ ref, double beta, double eps, double per_pair,
                                                   float* __restrict__ logp, double* __restrict__ parts) {
  __shared__ double red[4];
  const int pair = blockIdx.x;
  double L[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int begin = seq.at(2 * pair + i), end = seq.at(2 * pair + i + 1);
    double v = 0;
    for (int r = begin + (int)threadIdx.x; r < end; r += 256) v += o.lp[r];
    L[i] = block_sum_d(v, red);
    if (logp && threadIdx.x == 0) logp[2 * pair + i] = (float)L[i];
  }
  const double z = beta * ((L[0] - (ref ? (double)ref[2 * pair] : 0.0)) - (L[1] - (ref ? (double)ref[2 * pair + 1] : 0.0)));
  const double up = 1.0 / (1.0 + exp(-z)), down = 1.0 / (1.0 + exp(z));
  const double dz = (eps != 0 ? eps * up : 0.0) - (eps != 1 ? (1 - eps) * down : 0.0);
  const float g = (float)(dz * beta * per_pair);
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int begin = seq.at(2 * pair + i), end = seq.at(2 * pair + i + 1);
    for (int r = begin + (int)threadIdx.x; r < end; r += 256) o.g[r] = i == 0 ? g : -g;
  }
  if (threadIdx.x == 0) {
    parts[3 * pair] = (eps != 1 ? (1 - eps) * softplus(-z) : 0.0) + (eps != 0 ? eps * softplus(z) : 0.0);
    parts[3 * pair + 1] = z;
    parts[3 * pair + 2] = z > 0 ? 1.0 : 0.0;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void pair_grad_kernel(RowArgs a, Sequences seq, SeqRows o) {
  const int begin = seq.at(0), end = seq.at(seq.n);
  for (int r = begin + (int)blockIdx.x; r < end; r += gridDim.x) {
    unsigned char* out = (unsigned char*)a.grad + (long long)r * a.gld * (a.grad_bf16 ? 2 : 4);
    const T* x = (const T*)a.logits + (long long)r * a.ld;
    const int at = a.label[r];
    const float s = o.s[r], m = o.m[r], g = o.g[r];
    if (s == 0.f) {   // (masked, or without a distribution)
      for (int j = threadIdx.x; j < a.classes; j += 256) put(out, a.grad_bf16, j, 0.f);
      continue;
    }
    const float cf = -g / s, own = g * (o.rest[r] / s);
    for (int j = threadIdx.x; j < a.classes; j += 256) put(out, a.grad_bf16, j, j == at ? own : cf * exp_of(as_float(x[j]), m));
  }
}

int row_grid(int rows) { return rows < MAX_GRID ? rows : MAX_GRID; }

}  // namespace
}  // namespace et

namespace {

using namespace et_op;

constexpr size_t POLICY_WS = 256 + sizeof(double) * 4 * et::MAX_GRID;

size_t preference_ws(int64_t rows, int64_t pairs) { return (size_t)(rows * 24 + 64 + pairs * 24 + 256); }

// the arguments that both losses have in common
int check_rows(int32_t rows, int32_t classes, const void* logits, int32_t dtype, int64_t stride, const int32_t* label, const void* grad,
               int32_t grad_dtype, int64_t grad_stride, const void* ws, const float* loss) {
  if (rows < 1 || classes < 1 || !logits || !label || !ws || !loss || !type_ok(dtype) || (grad && !type_ok(grad_dtype))) return ET_EINVAL;
  const int64_t most = (INT64_MAX >> 4) / rows;   // (offsets in bytes stay below 2^62)
  if (stride < classes || stride > most || (grad && (grad_stride < classes || grad_stride > most))) return ET_EINVAL;
  if (!aligned(logits, type_size(dtype)) || !aligned(label, 4) || !aligned(loss, 4) || !aligned(ws, 16)) return ET_EINVAL;
  if (!grad) return ET_OK;
  if (!aligned(grad, type_size(grad_dtype))) return ET_EINVAL;
  const Span in(logits, rows, classes, stride, type_size(dtype)), out(grad, rows, classes, grad_stride, type_size(grad_dtype));
  if (out.meets(in) && !(grad == logits && grad_dtype == dtype && grad_stride == stride)) return ET_EINVAL;
  return ET_OK;
}

}  // namespace

extern "C" {

size_t et_policy_loss_ws_bytes(int32_t rows) { return rows < 1 ? 0 : POLICY_WS; }

int et_policy_loss(int32_t rows, int32_t classes, const void* logits_dev, int32_t dtype, int64_t row_stride, const int32_t* label_dev,
                   const et_policy* p, void* grad_dev, int32_t grad_dtype, int64_t grad_stride, void* workspace_dev, size_t workspace_bytes,
                   void* hip_stream, float* loss_dev) {
  const int rc = check_rows(rows, classes, logits_dev, dtype, row_stride, label_dev, grad_dev, grad_dtype, grad_stride, workspace_dev, loss_dev);
  if (rc != ET_OK) return rc;
  if (!p || !p->old_logp_dev || !p->advantage_dev || (p->ref_logp_dev && p->ref_logits_dev)) return ET_EINVAL;
  for (const float* v : {p->old_logp_dev, p->advantage_dev, p->ref_logp_dev, p->weight_dev, (const float*)p->logp_dev, (const float*)p->stats_dev})
    if (!aligned(v, 4)) return ET_EINVAL;
  if (!(p->clip_low >= 0 && p->clip_low <= 1 && p->clip_high >= 0 && std::isfinite(p->clip_high) && std::isfinite(p->kl_coef))) return ET_EINVAL;
  if (p->ref_logits_dev) {
    if (p->ref_stride < classes || p->ref_stride > (INT64_MAX >> 4) / rows || !aligned(p->ref_logits_dev, type_size(dtype))) return ET_EINVAL;
    if (grad_dev && Span(grad_dev, rows, classes, grad_stride, type_size(grad_dtype)).meets(Span(p->ref_logits_dev, rows, classes, p->ref_stride, type_size(dtype))))
      return ET_EINVAL;
  }
  if (workspace_bytes < POLICY_WS) return ET_ENOMEM;
  const hipStream_t s = (hipStream_t)hip_stream;
  const OnDeviceOf on(s);
  if (!on.ok) return ET_EHIP;
  et::RowArgs a = {logits_dev, row_stride, label_dev, grad_dev, grad_stride, rows, classes, grad_dtype == ET_BF16};
  et::PolicyArgs q = {p->old_logp_dev, p->advantage_dev, p->ref_logp_dev, p->weight_dev, p->ref_logits_dev, p->ref_stride,
                      1.0 - (double)p->clip_low, 1.0 + (double)p->clip_high, (double)p->kl_coef, p->logp_dev};
  double* count = (double*)workspace_dev;
  double* parts = count + 32;
  if (!p->weight_dev) hipLaunchKernelGGL(et::count_kernel, dim3(1), dim3(256), 0, s, label_dev, rows, classes, count);
  const int grid = et::row_grid(rows);
#define ET_POLICY(T, FULL) hipLaunchKernelGGL((et::policy_kernel<T, FULL>), dim3(grid), dim3(256), 0, s, a, q, count, parts)
  if (dtype == ET_BF16) {
    if (p->ref_logits_dev) ET_POLICY(bf16, true); else ET_POLICY(bf16, false);
  } else {
    if (p->ref_logits_dev) ET_POLICY(float, true); else ET_POLICY(float, false);
  }
#undef ET_POLICY
  hipLaunchKernelGGL(et::finish_kernel<4>, dim3(1), dim3(256), 0, s, parts, grid, 1.0, loss_dev, p->stats_dev);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

size_t et_preference_loss_ws_bytes(int32_t rows, int32_t pairs) { return rows < 1 || pairs < 1 ? 0 : preference_ws(rows, pairs); }

int et_preference_loss(int32_t rows, int32_t pairs, int32_t classes, const void* logits_dev, int32_t dtype, int64_t row_stride,
                       const int32_t* label_dev, const et_preference* p, void* grad_dev, int32_t grad_dtype, int64_t grad_stride,
                       void* workspace_dev, size_t workspace_bytes, void* hip_stream, float* loss_dev) {
  const int rc = check_rows(rows, classes, logits_dev, dtype, row_stride, label_dev, grad_dev, grad_dtype, grad_stride, workspace_dev, loss_dev);
  if (rc != ET_OK) return rc;
  if (!p || pairs < 1 || pairs > (INT32_MAX - 1) / 2 || (!p->offsets_dev && rows != 2 * pairs)) return ET_EINVAL;
  if (!aligned(p->offsets_dev, 4) || !aligned(p->ref_logp_dev, 4) || !aligned(p->logp_dev, 4) || !aligned(p->stats_dev, 4)) return ET_EINVAL;
  if (!(p->beta > 0 && std::isfinite(p->beta) && p->label_smoothing >= 0 && p->label_smoothing <= 1)) return ET_EINVAL;
  if (workspace_bytes < preference_ws(rows, pairs)) return ET_ENOMEM;
  const hipStream_t s = (hipStream_t)hip_stream;
  const OnDeviceOf on(s);
  if (!on.ok) return ET_EHIP;
  const et::RowArgs a = {logits_dev, row_stride, label_dev, grad_dev, grad_stride, rows, classes, grad_dtype == ET_BF16};
  const et::Sequences seq = {p->offsets_dev, rows, 2 * pairs};
  et::SeqRows o;
  o.lp = (double*)workspace_dev;
  double* parts = o.lp + rows;
  o.m = (float*)(parts + 3 * (size_t)pairs);
  o.s = o.m + rows;
  o.rest = o.s + rows;
  o.g = o.rest + rows;
  const int grid = et::row_grid(rows);
  if (dtype == ET_BF16) hipLaunchKernelGGL(et::row_stats_kernel<bf16>, dim3(grid), dim3(256), 0, s, a, seq, o);
  else hipLaunchKernelGGL(et::row_stats_kernel<float>, dim3(grid), dim3(256), 0, s, a, seq, o);
  hipLaunchKernelGGL(et::pair_kernel, dim3(pairs), dim3(256), 0, s, seq, o, p->ref_logp_dev, (double)p->beta, (double)p->label_smoothing, 1.0 / pairs,
                     p->logp_dev, parts);
  if (grad_dev) {
    if (dtype == ET_BF16) hipLaunchKernelGGL(et::pair_grad_kernel<bf16>, dim3(grid), dim3(256), 0, s, a, seq, o);
    else hipLaunchKernelGGL(et::pair_grad_kernel<float>, dim3(grid), dim3(256), 0, s, a, seq, o);
  }
  hipLaunchKernelGGL(et::finish_kernel<3>, dim3(1), dim3(256), 0, s, parts, pairs, 1.0 / pairs, loss_dev, p->stats_dev);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

}  // extern "C"
