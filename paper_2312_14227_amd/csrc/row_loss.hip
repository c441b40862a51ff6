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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Rows start at any element: vectors are loaded and stored at the alignment of an element, which global memory takes on this hardware
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float LOWEST = -3.4028234663852886e38f;   // in place of the maximum of nothing: x - LOWEST of x = -inf is -inf, and its exponential 0
constexpr float LOG2E = 1.44269502162933349609375f, LOG2E_LO = 1.925963033500979e-8f;   // log2 e = LOG2E + LOG2E_LO

// exp(d), d <= 0
__device__ __forceinline__ float exp_fast(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }
// The same where many are added: with LOG2E alone all are off the same way, 1.3e-8 |d| of their value, and sums of the logarithms over the rows of a sequence
// add that up (the mean margin of 16 sequences of 500 rows was 3e-6 off, three times its own roundings)
__device__ __forceinline__ float exp_true(float d) { return __builtin_amdgcn_exp2f(fmaf(d, LOG2E, d * LOG2E_LO)); }

// exp(d) for a row's scalars: the argument is reduced in float64, so that what is off is the hardware's exponential on [-1/2, 1/2], 2^-23 of the value
__device__ __forceinline__ double exp_d(double d) {
  double u = d * 1.4426950408889634;
  u = u < -1200 ? -1200 : u;
  u = u > 1200 ? 1200 : u;
  const double n = rint(u);
  return ldexp((double)__builtin_amdgcn_exp2f((float)(u - n)), n == n ? (int)n : 0);
}
// exp(d) - 1 - d, to rounding also where it is small: its series up to 1
__device__ __forceinline__ double exp_rest(double d) {
  if (!(fabs(d) <= 1.0)) {
    const double e = exp_d(d);
    return e == INFINITY ? INFINITY : e - 1 - d;
  }
  const float f = (float)d;
  float s = 1.f / 479001600;
  const float c[10] = {1.f / 39916800, 1.f / 3628800, 1.f / 362880, 1.f / 40320, 1.f / 5040, 1.f / 720, 1.f / 120, 1.f / 24, 1.f / 6, 1.f / 2};
#pragma unroll
  for (int i = 0; i < 10; i++) s = fmaf(s, f, c[i]);
  return d * d * (double)s;
}

template <typename T>
struct Vec {   // 16 bytes of a row
  static constexpr int N = 16 / sizeof(T);
};
template <typename T>
__device__ __forceinline__ u32x4 load_vec(const T* p) { return *(const u32x4_any*)p; }
template <typename T>
__device__ __forceinline__ void unpack(u32x4 v, float (&f)[Vec<T>::N]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 4; k++) f[k] = __uint_as_float(v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++) {
      f[2 * k] = __uint_as_float(v[k] << 16);
      f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
    }
  }
}
// element k becomes minus infinity
template <typename T>
__device__ __forceinline__ void take_out(u32x4& v, int k) {
#pragma unroll
  for (int d = 0; d < 4; d++) {
    if constexpr (sizeof(T) == 4) {
      if (d == k) v[d] = 0xff800000u;
    } else {
      if (d == k >> 1) v[d] = k & 1 ? (v[d] & 0xffffu) | 0xff800000u : (v[d] & 0xffff0000u) | 0xff80u;
    }
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  bf16x2 o;
  o[0] = (bf16)a;
  o[1] = (bf16)b;
  return __builtin_bit_cast(uint32_t, o);
}
// N values at element j of a gradient row
template <int N>
__device__ __forceinline__ void store_vec(void* row, bool as_bf16, unsigned j, const float (&f)[N]) {
  if (as_bf16) {
    bf16* o = (bf16*)row + j;
    if constexpr (N == 8) {
      u32x4 v;
#pragma unroll
      for (int k = 0; k < 4; k++) v[k] = pack2(f[2 * k], f[2 * k + 1]);
      *(u32x4_any*)o = v;
    } else {
      u32x2 v;
      v[0] = pack2(f[0], f[1]);
      v[1] = pack2(f[2], f[3]);
      *(u32x2_any*)o = v;
    }
  } else {
    float* o = (float*)row + j;
#pragma unroll
    for (int h = 0; h < N / 4; h++) {
      u32x4 v;
#pragma unroll
      for (int k = 0; k < 4; k++) v[k] = __float_as_uint(f[4 * h + k]);
      *(u32x4_any*)(o + 4 * h) = v;
    }
  }
}
__device__ __forceinline__ void put(void* row, bool as_bf16, int j, float v) {
  if (as_bf16) ((bf16*)row)[j] = (bf16)v;
  else ((float*)row)[j] = v;
}

template <typename F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ double block_sum_d(double v, double* red) {   // 256 threads
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---- softmax statistics as they run along a row: the maximum m so far and the sum s of exp(x - m).  The maximum passes over NaN, the sum does not.
struct Run {
  float m, s;   // {LOWEST, 0} at the start
  __device__ __forceinline__ void raise(float to) {   // to >= m
    s *= exp_true(m - to);
    m = to;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&f)[N]) {
    float top = f[0];
#pragma unroll
    for (int k = 1; k < N; k++) top = fmaxf(top, f[k]);
    raise(fmaxf(m, top));
    float e[N];
#pragma unroll
    for (int k = 0; k < N; k++) e[k] = exp_true(f[k] - m);
#pragma unroll
    for (int w = N / 2; w > 0; w /= 2)
#pragma unroll
      for (int k = 0; k < w; k++) e[k] += e[k + w];
    s += e[0];
  }
  __device__ __forceinline__ void over_wave() {
    raise(wave_max(m));
    s = wave_sum(s);
  }
};
// Two rows at once, and t = sum exp(x - mx) ((x - mx) - (y - my)), from which their divergence follows without the rows' offsets
struct RunPair {
  Run x, y;
  float t;
  __device__ __forceinline__ void raise(float mx, float my) {
    const float f = exp_true(x.m - mx), shift = (x.m - mx) - (y.m - my);
    t = f * x.s == 0.f ? 0.f : f * (t + x.s * shift);   // (a lane that has met nothing but minus infinities has no offset to speak of)
    x.s *= f;
    x.m = mx;
    y.raise(my);
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&f)[N], const float (&g)[N]) {
    float tx = f[0], ty = g[0];
#pragma unroll
    for (int k = 1; k < N; k++) {
      tx = fmaxf(tx, f[k]);
      ty = fmaxf(ty, g[k]);
    }
    raise(fmaxf(x.m, tx), fmaxf(y.m, ty));
#pragma unroll
    for (int k = 0; k < N; k++) {
      const float dx = f[k] - x.m, dy = g[k] - y.m, e = exp_true(dx);
      x.s += e;
      y.s += exp_true(dy);
      t += e == 0.f ? 0.f : e * (dx - dy);
    }
  }
  __device__ __forceinline__ void over_wave() {
    raise(wave_max(x.m), wave_max(y.m));
    x.s = wave_sum(x.s);
    y.s = wave_sum(y.s);
    t = wave_sum(t);
  }
};

struct RowArgs {
  const void* logits;
  long long ld;
  const int32_t* label;
  void* grad;
  long long gld;
  int rows, classes, grad_bf16;
  __device__ __forceinline__ void* grad_row(int r) const { return (unsigned char*)grad + (long long)r * gld * (grad_bf16 ? 2 : 4); }
  __device__ __forceinline__ bool masked(int at) const { return (unsigned)at >= (unsigned)classes; }
};

struct PolicyArgs {
  const float *old_logp, *advantage, *ref_logp, *weight;
  const void* ref;
  long long ref_ld;
  double low, high, kl_coef;   // borders of the ratio
  float* logp;
};

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

// what a row's statistics come to: m and s = sum exp(x - m) over all classes, rest = the sum without the label's term
struct RowStat {
  double s, ea, rest, lp;
  float m;
  bool none;       // no distribution
};
__device__ __forceinline__ RowStat row_stat(const Run& others, float xa) {
  RowStat o;
  o.m = fmaxf(others.m, xa);
  o.ea = exp_d((double)xa - (double)o.m);
  o.rest = (double)others.s * exp_d((double)others.m - (double)o.m);
  o.s = o.rest + o.ea;
  o.none = o.s == 0.0;
  const bool likely = o.ea > o.rest;
  const double q = o.rest / o.ea, l = log(likely ? 1.0 + q : o.s);
  o.lp = o.none ? -INFINITY : !likely ? ((double)xa - (double)o.m) - l : -(q < 1e-6 ? q - 0.5 * q * q : l);
  return o;
}

// what the waves of a row's workgroup need for its gradient: cf exp(x - m), with the exact divergence (cf + ck ((x - m) - (y - my) - kk)) exp(x - m), and
// `own` for the label
struct RowGrad {
  float m, my, cf, ck, kk, own;
  int zero;
};

// Adds a row to the sums (loss, surrogate, divergence, clipped) and says what its gradient is made of
__device__ __forceinline__ RowGrad policy_row(const PolicyArgs& p, const RowStat& s, double* sum, float old, float adv, float ref, double w) {
  RowGrad o = {s.m, 0.f, 0.f, 0.f, 0.f, 0.f, 1};
  if (s.none) return o;
  const double A = (double)adv, ratio = exp_d(s.lp - (double)old);
  const bool over = (A > 0 && ratio > p.high) || (A < 0 && ratio < p.low);
  const double surrogate = A * (over ? (A > 0 ? p.high : p.low) : ratio);
  double g = over ? 0.0 : -ratio * A, kl = 0;
  if (p.ref_logp) {
    const double d = (double)ref - s.lp;
    kl = exp_rest(d);
    if (p.kl_coef != 0) g -= p.kl_coef * (kl + d);
  }
  sum[0] += w * ((p.kl_coef != 0 ? p.kl_coef * kl : 0.0) - surrogate);
  sum[1] += w * surrogate;
  sum[2] += w * kl;
  if (over) sum[3] += w;
  o.cf = (float)(-w * g / s.s);
  o.own = (float)(w * g * (s.rest / s.s));
  o.zero = 0;
  return o;
}
// the exact divergence on top; pair: over the classes other than the label for x, all for y
__device__ __forceinline__ void full_kl(const PolicyArgs& p, const RowStat& s, RunPair& pair, double* sum, float xa, float ya, double w, RowGrad& o) {
  if (s.none) return;
  pair.raise(s.m, pair.y.m);
  const double ea = s.ea, apart = ((double)xa - (double)s.m) - ((double)ya - (double)pair.y.m);
  const double kk = ((double)pair.t + (ea == 0 ? 0.0 : ea * apart)) / s.s, kl = kk + log((double)pair.y.s / s.s);
  if (p.kl_coef != 0) sum[0] += w * p.kl_coef * kl;
  sum[2] += w * kl;
  o.my = pair.y.m;
  o.kk = (float)kk;
  o.ck = (float)(w * p.kl_coef / s.s);
  if (p.kl_coef != 0 && ea != 0) o.own = (float)((double)o.own + w * p.kl_coef * (ea / s.s) * (apart - kk));
}

enum Mode { POLICY, POLICY_FULL, STATS };

constexpr int MAX_GRID = 2048;    // workgroups of the row kernels
constexpr int COUNT_ROWS = 8192;  // rows that a workgroup counts by itself

// unmasked rows among [begin, end), by all threads of a workgroup; red: one entry for each wave
__device__ __forceinline__ int count_rows(const RowArgs& a, int begin, int end, int* red) {
  int n = 0;
  for (int r = begin + (int)threadIdx.x; r < end; r += blockDim.x) n += a.masked(a.label[r]) ? 0 : 1;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
  for (int i = 0; i < (int)blockDim.x / 64; i++) n += red[i];
  return n;
}
__global__ __launch_bounds__(256) void count_kernel(RowArgs a, int* __restrict__ counts) {
  __shared__ int red[4];
  const long long per = ((long long)a.rows + gridDim.x - 1) / gridDim.x;
  const int n = count_rows(a, (int)min((long long)a.rows, per * blockIdx.x), (int)min((long long)a.rows, per * (blockIdx.x + 1)), red);
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// ---- rows.  Both kernels below go over the rows r = first, first + step, ...; the threads of a row ("team") are t = 0 .. TPR - 1, and vector v of a row, 16 bytes, is
// that at element (v * TPR + t) * N of thread t.  A last piece shorter than a vector is one element each of the first threads.
template <typename T, int W>
struct RowShape {
  static constexpr int N = Vec<T>::N, TPR = 64 * W;
  int C, Cv, rem, nv, mine;   // classes, those in vectors, those behind; vectors of the team, of this thread
  __device__ __forceinline__ RowShape(int classes, int t) : C(classes), Cv(classes - classes % N), rem(classes % N) {
    nv = (Cv / N + TPR - 1) / TPR;
    mine = (Cv / N - t + TPR - 1) / TPR;
  }
};
struct LabelAt {
  int v, t, k;   // vector, thread and element of a label (v = -1: in the last piece)
  template <typename T, int W>
  __device__ __forceinline__ LabelAt(const RowShape<T, W>& s, int at) {
    constexpr int N = RowShape<T, W>::N, TPR = RowShape<T, W>::TPR;
    const bool in_vec = at < s.Cv;
    v = in_vec ? at / N / TPR : -1;
    t = in_vec ? at / N % TPR : at - s.Cv;
    k = at % N;
  }
};

__device__ __forceinline__ double unit_weight(const RowArgs& a, const int* counts, int n_counts, int* red) {
  int n = 0;
  if (n_counts)
    for (int i = 0; i < n_counts; i++) n += counts[i];
  else
    n = count_rows(a, 0, a.rows, red);
  return 1.0 / n;
}

// Adds up a row's statistics over its waves and says what follows from them, in every thread; sums: this team's.  b.zero stays for a row without a distribution.
template <int W, Mode MODE>
__device__ __forceinline__ RowGrad row_scalars(const PolicyArgs& p, const SeqRows& o, int r, RunPair run, float xa, float ya, float old, float adv, float ref, double w,
                                               RunPair* red, RowGrad* said, double* sums) {
  constexpr bool FULL = MODE == POLICY_FULL;
  if (FULL) run.over_wave();
  else run.x.over_wave();
  RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1};
  if (W > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = run;
    __syncthreads();
  }
  if (W == 1 || threadIdx.x < 64) {
    if (W > 1) {
      run = red[0];
#pragma unroll 1
      for (int i = 1; i < W; i++) {
        RunPair one = red[i];
        const float mx = fmaxf(run.x.m, one.x.m);
        if (FULL) {
          const float my = fmaxf(run.y.m, one.y.m);
          run.raise(mx, my);
          one.raise(mx, my);
          run.y.s += one.y.s;
          run.t += one.t;
        } else {
          run.x.raise(mx);
          one.x.raise(mx);
        }
        run.x.s += one.x.s;
      }
    }
    const RowStat s = row_stat(run.x, xa);
    const bool first = (threadIdx.x & 63) == 0;
    if (MODE == STATS) {
      if (first) {
        o.m[r] = s.m;
        o.s[r] = (float)s.s;
        o.rest[r] = (float)s.rest;
        o.lp[r] = s.none ? 0.0 : s.lp;
        o.g[r] = 0.f;
      }
    } else {
      double sum[4] = {0, 0, 0, 0};
      b = policy_row(p, s, sum, old, adv, ref, w);
      if (FULL) full_kl(p, s, run, sum, xa, ya, w, b);
      if (first) {
        if (p.logp) p.logp[r] = (float)s.lp;
#pragma unroll
        for (int i = 0; i < 4; i++) sums[i] += sum[i];
        if (W > 1) *said = b;
      }
    }
  }
  if (W > 1) {
    __syncthreads();
    if (MODE != STATS) b = *said;
  }
  return b;
}
// a masked row, of which nothing is looked at
template <Mode MODE>
__device__ __forceinline__ void masked_row(const PolicyArgs& p, const SeqRows& o, int r) {
  if (MODE == STATS) {
    o.m[r] = o.s[r] = o.rest[r] = o.g[r] = 0.f;
    o.lp[r] = 0;
  } else if (p.logp) {
    p.logp[r] = 0.f;
  }
}

template <bool FULL, int N>
__device__ __forceinline__ void gradient(const RowGrad& b, const float (&f)[N], const float (&g)[N], float (&out)[N]) {
#pragma unroll
  for (int k = 0; k < N; k++) {
    const float d = f[k] - b.m, e = exp_fast(d);
    if (FULL) out[k] = e == 0.f ? 0.f : e * fmaf(b.ck, d - (g[k] - b.my) - b.kk, b.cf);
    else out[k] = b.cf * e;
  }
}

// One row of W waves (W = 1: four rows in a workgroup, a wave each) that stays in registers, at most NV vectors a thread: the logits are read once, and as each
// vector has become a piece of the gradient the same vector of the next row is loaded in its place, so that loads are on the way all the time, though a row is read and
// written by turns.  Loads go through buffer descriptors: lanes beyond the row and rows that are not looked at ask for nothing, without a branch around the load (with
// one the vectors were copied from register to register, which waits for them).
template <typename T, int W, int NV, Mode MODE, bool GRAD>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, 4) void kept_kernel(RowArgs a, PolicyArgs p, Sequences seq, SeqRows o, const int* __restrict__ counts, int n_counts,
                                                                        double* __restrict__ parts) {
  constexpr int N = Vec<T>::N, TPR = 64 * W, TEAMS = W == 1 ? 4 : 1;
  constexpr bool FULL = MODE == POLICY_FULL;
  __shared__ RunPair red[W];
  __shared__ RowGrad said;
  __shared__ double sums[TEAMS][4];
  __shared__ int red_n[16];
  const int t = threadIdx.x % TPR, team = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const RowShape<T, W> shape(a.classes, t);
  const int step = gridDim.x * TEAMS;
  double unit = 0;   // weight of an unmasked row
  if (MODE != STATS) {
    if (threadIdx.x < TEAMS * 4) sums[threadIdx.x / 4][threadIdx.x % 4] = 0;
    if (!p.weight) unit = unit_weight(a, counts, n_counts, red_n);
    __syncthreads();
  }
  const int begin = MODE == STATS ? seq.at(0) : 0, end = MODE == STATS ? seq.at(seq.n) : a.rows;
  auto label_of = [&](int r) { return __builtin_amdgcn_readfirstlane(r >= begin && r < end ? a.label[r] : -1); };
  u32x4 x[NV], y[FULL ? NV : 1];
  float x_tail, y_tail = 0.f;
  struct Source {
    __amdgpu_buffer_rsrc_t rows, all;
  };
  auto source = [&](const void* base, long long ld, int r, bool there) {
    void* at = (void*)((const T*)base + (there ? (long long)r * ld : 0));
    return Source{__builtin_amdgcn_make_buffer_rsrc(at, 0, there ? shape.Cv * (int)sizeof(T) : 0, 0x00027000),
                  __builtin_amdgcn_make_buffer_rsrc(at, 0, there ? shape.C * (int)sizeof(T) : 0, 0x00027000)};
  };
  auto vec_of = [&](const Source& s, int v) { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(s.rows, t * 16, v * TPR * 16, 0)); };
  auto tail_of = [&](const Source& s) {
    const int at = (shape.Cv + t) * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(s.all, at, 0, 0));
    else return __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b16(s.all, at, 0, 0) << 16);
  };
  int r = blockIdx.x * TEAMS + team, at = r < a.rows ? label_of(r) : -1;
  {
    const Source sx = source(a.logits, a.ld, r, !a.masked(at)), sy = source(p.ref, p.ref_ld, r, FULL && !a.masked(at));
#pragma unroll
    for (int v = 0; v < NV; v++) {
      x[v] = vec_of(sx, v);
      if (FULL) y[v] = vec_of(sy, v);
    }
    x_tail = tail_of(sx);
    if (FULL) y_tail = tail_of(sy);
  }
  const u32x4 nothing = sizeof(T) == 4 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
  while (r < a.rows) {
    const int next = (int)min((long long)r + step, (long long)a.rows), next_at = next < a.rows ? label_of(next) : -1;
    const bool look = !a.masked(at), more = !a.masked(next_at);
    const Source sx = source(a.logits, a.ld, next, more), sy = source(p.ref, p.ref_ld, next, FULL && more);
    float xa = 0, ya = 0, old = 0, adv = 0, ref = 0;
    double w = unit;
    RunPair run = {{LOWEST, 0.f}, {LOWEST, 0.f}, 0.f};
    const LabelAt place(shape, at);
    if (look) {
      xa = (float)((const T*)a.logits + (long long)r * a.ld)[at];
      if (FULL) ya = (float)((const T*)p.ref + (long long)r * p.ref_ld)[at];
      if (MODE != STATS) {
        old = p.old_logp[r];
        adv = p.advantage[r];
        if (p.ref_logp) ref = p.ref_logp[r];
        if (p.weight) w = (double)p.weight[r];
      }
#pragma unroll
      for (int v = 0; v < NV; v++)
        if (v < shape.nv) {
          u32x4 u = x[v], uy = FULL ? y[v] : x[v];
          if (v == place.v && t == place.t) take_out<T>(u, place.k);
          if (v == shape.nv - 1 && v >= shape.mine) u = uy = nothing;
          float f[N], g[N];
          unpack<T>(u, f);
          if (FULL) {
            unpack<T>(uy, g);
            run.add(f, g);
          } else {
            run.x.add(f);
          }
        }
      if (shape.rem) {
        const float f[1] = {t < shape.rem && !(place.v < 0 && t == place.t) ? x_tail : -INFINITY}, g[1] = {t < shape.rem ? y_tail : -INFINITY};
        if (FULL) run.add(f, g);
        else run.x.add(f);
      }
    }
    if (!GRAD) {
#pragma unroll
      for (int v = 0; v < NV; v++) {
        x[v] = vec_of(sx, v);
        if (FULL) y[v] = vec_of(sy, v);
      }
      x_tail = tail_of(sx);
      if (FULL) y_tail = tail_of(sy);
    }
    RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1};
    if (look) b = row_scalars<W, MODE>(p, o, r, run, xa, ya, old, adv, ref, w, red, &said, sums[team]);
    else if (t == 0) masked_row<MODE>(p, o, r);
    if (GRAD) {
      unsigned char* const out = (unsigned char*)a.grad_row(r);
      const int size = a.grad_bf16 ? 2 : 4;
#pragma unroll
      for (int v = 0; v < NV; v++) {
        if (v < shape.nv) {
          float f[N], g[N], d[N];
          asm volatile("" : "+v"(x[v]));   // (unpacked again: kept from the first pass it would take twice the registers)
          unpack<T>(x[v], f);
          if (FULL) {
            asm volatile("" : "+v"(y[v]));
            unpack<T>(y[v], g);
          }
          gradient<FULL>(b, f, g, d);
          if (b.zero)
#pragma unroll
            for (int k = 0; k < N; k++) d[k] = 0.f;
          if (v == place.v && t == place.t)
#pragma unroll
            for (int k = 0; k < N; k++) d[k] = k == place.k ? b.own : d[k];
          if (v < shape.mine) store_vec(out + v * TPR * N * size, a.grad_bf16, t * N, d);
        }
        x[v] = vec_of(sx, v);
        if (FULL) y[v] = vec_of(sy, v);
      }
      if (shape.rem) {
        const float f[1] = {x_tail}, g[1] = {y_tail};
        float d[1];
        gradient<FULL>(b, f, g, d);
        if (t < shape.rem) put(out, a.grad_bf16, shape.Cv + t, b.zero ? 0.f : place.v < 0 && t == place.t ? b.own : d[0]);
      }
      x_tail = tail_of(sx);
      if (FULL) y_tail = tail_of(sy);
    }
    r = next;
    at = next_at;
  }
  if (MODE != STATS) {
    __syncthreads();
    if (threadIdx.x < TEAMS * 4) parts[blockIdx.x * TEAMS * 4 + threadIdx.x] = sums[threadIdx.x / 4][threadIdx.x % 4];
  }
}

// Rows of any length, U vectors of a thread at a time; read again for the gradient
template <typename T, int W, int U, Mode MODE>
__global__ __launch_bounds__(64 * W) void streamed_kernel(RowArgs a, PolicyArgs p, Sequences seq, SeqRows o, const int* __restrict__ counts, int n_counts,
                                                          double* __restrict__ parts) {
  constexpr int N = Vec<T>::N, TPR = 64 * W;
  constexpr bool FULL = MODE == POLICY_FULL;
  __shared__ RunPair red[W];
  __shared__ RowGrad said;
  __shared__ double sums[4];
  __shared__ int red_n[16];
  const int t = threadIdx.x;
  const RowShape<T, W> shape(a.classes, t);
  double unit = 0;
  if (MODE != STATS) {
    if (threadIdx.x < 4) sums[threadIdx.x] = 0;
    if (!p.weight) unit = unit_weight(a, counts, n_counts, red_n);
    __syncthreads();
  }
  const int begin = MODE == STATS ? seq.at(0) : 0, end = MODE == STATS ? seq.at(seq.n) : a.rows;
  const u32x4 nothing = sizeof(T) == 4 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
  for (int r = blockIdx.x; r < a.rows; r = (int)min((long long)r + gridDim.x, (long long)a.rows)) {
    const int at = __builtin_amdgcn_readfirstlane(r >= begin && r < end ? a.label[r] : -1);
    const bool look = !a.masked(at), grad = MODE != STATS && a.grad;
    const T *x = (const T*)a.logits + (long long)r * a.ld, *y = FULL ? (const T*)p.ref + (long long)r * p.ref_ld : x;
    const LabelAt place(shape, at);
    RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1};
    float x_tail = -INFINITY, y_tail = -INFINITY;
    if (look) {
      float old = 0, adv = 0, ref = 0;
      double w = unit;
      const float xa = (float)x[at], ya = FULL ? (float)y[at] : 0.f;
      if (MODE != STATS) {
        old = p.old_logp[r];
        adv = p.advantage[r];
        if (p.ref_logp) ref = p.ref_logp[r];
        if (p.weight) w = (double)p.weight[r];
      }
      if (t < shape.rem) {
        x_tail = (float)x[shape.Cv + t];
        if (FULL) y_tail = (float)y[shape.Cv + t];
      }
      RunPair run = {{LOWEST, 0.f}, {LOWEST, 0.f}, 0.f};
      for (int v = 0; v < shape.nv; v += U) {
        u32x4 ux[U], uy[FULL ? U : 1];
#pragma unroll
        for (int i = 0; i < U; i++) {
          const bool in = v + i < shape.mine;
          ux[i] = in ? load_vec(x + ((size_t)(v + i) * TPR + t) * N) : nothing;
          if (FULL) uy[i] = in ? load_vec(y + ((size_t)(v + i) * TPR + t) * N) : nothing;
        }
#pragma unroll
        for (int i = 0; i < U; i++) {
          if (v + i == place.v && t == place.t) take_out<T>(ux[i], place.k);
          float f[N], g[N];
          unpack<T>(ux[i], f);
          if (FULL) {
            unpack<T>(uy[i], g);
            run.add(f, g);
          } else {
            run.x.add(f);
          }
        }
      }
      if (shape.rem) {
        const float f[1] = {place.v < 0 && t == place.t ? -INFINITY : x_tail}, g[1] = {y_tail};
        if (FULL) run.add(f, g);
        else run.x.add(f);
      }
      b = row_scalars<W, MODE>(p, o, r, run, xa, ya, old, adv, ref, w, red, &said, sums);
    } else if (t == 0) {
      masked_row<MODE>(p, o, r);
    }
    if (!grad) continue;
    void* const out = a.grad_row(r);
    for (int v = 0; v < shape.nv; v += U) {
      u32x4 ux[U], uy[FULL ? U : 1];
#pragma unroll
      for (int i = 0; i < U; i++)
        if (look && v + i < shape.mine) {
          ux[i] = load_vec(x + ((size_t)(v + i) * TPR + t) * N);
          if (FULL) uy[i] = load_vec(y + ((size_t)(v + i) * TPR + t) * N);
        }
#pragma unroll
      for (int i = 0; i < U; i++) {
        if (v + i >= shape.mine) break;
        float f[N], g[N], d[N];
        unpack<T>(ux[i], f);
        if (FULL) unpack<T>(uy[i], g);
        gradient<FULL>(b, f, g, d);
#pragma unroll
        for (int k = 0; k < N; k++) d[k] = b.zero ? 0.f : v + i == place.v && t == place.t && k == place.k ? b.own : d[k];
        store_vec(out, a.grad_bf16, ((unsigned)(v + i) * TPR + t) * N, d);
      }
    }
    if (t < shape.rem) {
      const float f[1] = {x_tail}, g[1] = {y_tail};
      float d[1];
      gradient<FULL>(b, f, g, d);
      put(out, a.grad_bf16, shape.Cv + t, b.zero ? 0.f : place.v < 0 && t == place.t ? b.own : d[0]);
    }
  }
  if (MODE != STATS) {
    __syncthreads();
    if (threadIdx.x < 4) parts[blockIdx.x * 4 + threadIdx.x] = sums[threadIdx.x];
  }
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

// The gradient once the factors are known: nothing but a map of the logits.  A wave takes GRAD_VECS vectors a lane of a row at a time.
constexpr int GRAD_VECS = 8;
template <typename T>
__global__ __launch_bounds__(256) void pair_grad_kernel(RowArgs a, Sequences seq, SeqRows o) {
  constexpr int N = Vec<T>::N, PIECE = 64 * N * GRAD_VECS;
  const int begin = seq.at(0), end = seq.at(seq.n), lane = threadIdx.x & 63;
  const int C = a.classes, Cv = C - C % N, pieces = (C + PIECE - 1) / PIECE;
  const long long tasks = (long long)(end - begin) * pieces;
  for (long long task = blockIdx.x * 4ll + (threadIdx.x >> 6); task < tasks; task += gridDim.x * 4ll) {
    const int r = begin + (int)(task / pieces), j0 = (int)(task % pieces) * PIECE;
    void* const out = a.grad_row(r);
    const T* x = (const T*)a.logits + (long long)r * a.ld;
    const int at = a.label[r];
    const float s = o.s[r], m = o.m[r], g = o.g[r];
    const bool zero = s == 0.f;   // masked, or without a distribution
    const float cf = -g / s, own = g * (o.rest[r] / s);
    u32x4 v[GRAD_VECS];
#pragma unroll
    for (int i = 0; i < GRAD_VECS; i++) {
      const int j = j0 + (i * 64 + lane) * N;
      if (j < Cv && !zero) v[i] = load_vec(x + j);
    }
#pragma unroll
    for (int i = 0; i < GRAD_VECS; i++) {
      const int j = j0 + (i * 64 + lane) * N;
      if (j >= Cv) break;
      float f[N];
      unpack<T>(v[i], f);
#pragma unroll
      for (int k = 0; k < N; k++) f[k] = zero ? 0.f : at == j + k ? own : cf * exp_fast(f[k] - m);
      store_vec(out, a.grad_bf16, j, f);
    }
    const int j = Cv + lane;
    if (j < C && Cv >= j0 && Cv < j0 + PIECE) put(out, a.grad_bf16, j, zero ? 0.f : at == j ? own : cf * exp_fast((float)x[j] - m));
  }
}

// How a row is taken apart: waves, and whether it stays in registers.  16 vectors a thread and 16 waves on a compute unit are what its registers hold
struct RowPlan {
  int waves;
  bool keep;
};
RowPlan row_plan(int classes, size_t size, bool full) {
  const int64_t vecs = ((int64_t)classes * (int64_t)size + 15) / 16, most = full ? 8 : 16;
  if (vecs <= 64 * (full ? 4 : 8)) return {1, true};
  if (vecs <= 256 * most) return {4, true};
  if (vecs <= 512 * most) return {8, true};
  if (vecs <= 1024 * most) return {16, true};
  return {8, false};
}
int row_grid(int rows, const RowPlan& plan, int cus) {
  const int per_group = plan.waves == 1 ? 4 : 1, most = std::min(MAX_GRID, cus * (plan.waves == 1 ? 8 : 16 / plan.waves));
  return std::min(most, (rows - 1) / per_group + 1);
}

template <typename T, Mode MODE>
void row_launch(const RowPlan& plan, int grid, hipStream_t s, const RowArgs& a, const PolicyArgs& p, const Sequences& seq, const SeqRows& o, const int* counts,
                int n_counts, double* parts) {
  constexpr int F = MODE == POLICY_FULL ? 2 : 1;
#define ET_KEPT(W, NV) \
  do { \
    if constexpr (MODE != STATS) { \
      if (a.grad) { hipLaunchKernelGGL((kept_kernel<T, W, NV, MODE, true>), dim3(grid), dim3(W == 1 ? 256 : 64 * W), 0, s, a, p, seq, o, counts, n_counts, parts); break; } \
    } \
    hipLaunchKernelGGL((kept_kernel<T, W, NV, MODE, false>), dim3(grid), dim3(W == 1 ? 256 : 64 * W), 0, s, a, p, seq, o, counts, n_counts, parts); \
  } while (0)
  if (!plan.keep) hipLaunchKernelGGL((streamed_kernel<T, 8, 8 / F, MODE>), dim3(grid), dim3(512), 0, s, a, p, seq, o, counts, n_counts, parts);
  else if (plan.waves == 1) ET_KEPT(1, 8 / F);
  else if (plan.waves == 4) ET_KEPT(4, 16 / F);
  else if (plan.waves == 8) ET_KEPT(8, 16 / F);
  else ET_KEPT(16, 16 / F);
#undef ET_KEPT
}

}  // namespace
}  // namespace et

namespace {

using namespace et_op;

constexpr int MAX_COUNTS = 256;
constexpr size_t POLICY_WS = sizeof(int) * MAX_COUNTS + sizeof(double) * 4 * 4 * et::MAX_GRID;

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
  int* counts = (int*)workspace_dev;
  double* parts = (double*)(counts + MAX_COUNTS);
  const et::RowPlan plan = et::row_plan(classes, type_size(dtype), q.ref != nullptr);
  const int grid = et::row_grid(rows, plan, device_cus(on.dev)), n_counts = q.weight || rows <= et::COUNT_ROWS ? 0 : std::min(MAX_COUNTS, rows / 4096);
  if (n_counts) hipLaunchKernelGGL(et::count_kernel, dim3(n_counts), dim3(256), 0, s, a, counts);
  const et::Sequences seq = {};
  const et::SeqRows none = {};
  if (dtype == ET_BF16) {
    if (q.ref) et::row_launch<bf16, et::POLICY_FULL>(plan, grid, s, a, q, seq, none, counts, n_counts, parts);
    else et::row_launch<bf16, et::POLICY>(plan, grid, s, a, q, seq, none, counts, n_counts, parts);
  } else {
    if (q.ref) et::row_launch<float, et::POLICY_FULL>(plan, grid, s, a, q, seq, none, counts, n_counts, parts);
    else et::row_launch<float, et::POLICY>(plan, grid, s, a, q, seq, none, counts, n_counts, parts);
  }
  hipLaunchKernelGGL(et::finish_kernel<4>, dim3(1), dim3(256), 0, s, parts, grid * (plan.waves == 1 ? 4 : 1), 1.0, loss_dev, p->stats_dev);
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
  const int cus = device_cus(on.dev);
  const et::RowPlan plan = et::row_plan(classes, type_size(dtype), false);
  const int grid = et::row_grid(rows, plan, cus);
  const et::PolicyArgs none = {};
  if (dtype == ET_BF16) et::row_launch<bf16, et::STATS>(plan, grid, s, a, none, seq, o, nullptr, 0, nullptr);
  else et::row_launch<float, et::STATS>(plan, grid, s, a, none, seq, o, nullptr, 0, nullptr);
  hipLaunchKernelGGL(et::pair_kernel, dim3(pairs), dim3(256), 0, s, seq, o, p->ref_logp_dev, (double)p->beta, (double)p->label_smoothing, 1.0 / pairs,
                     p->logp_dev, parts);
  if (grad_dev) {
    const int64_t piece = 64 * et::GRAD_VECS * (16 / (int64_t)type_size(dtype)), tasks = rows * ((classes + piece - 1) / piece);
    const int groups = (int)std::min<int64_t>((tasks + 3) / 4, 1 << 20);
    if (dtype == ET_BF16) hipLaunchKernelGGL(et::pair_grad_kernel<bf16>, dim3(groups), dim3(256), 0, s, a, seq, o);
    else hipLaunchKernelGGL(et::pair_grad_kernel<float>, dim3(groups), dim3(256), 0, s, a, seq, o);
  }
  hipLaunchKernelGGL(et::finish_kernel<3>, dim3(1), dim3(256), 0, s, parts, pairs, 1.0 / pairs, loss_dev, p->stats_dev);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

}  // extern "C"
