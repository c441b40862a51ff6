// Kernels over rows of logits: softmax statistics, and the gradients of losses that depend on a row through the log probability of its label.
//
// Of a row they need a reference m near its maximum and S = sum exp(x - m), from which log p[a] = x[a] - m - log S.
// The label's own term is left out of the sum, S = rest + its term: 1 - p[a] = rest / S, its gradient, and log p[a] = -log1p(rest / term) are exact to rounding also where
// p[a] is close to 1.
//
// What bounds them: memory, with the vector units close behind.  An element costs a row's statistics some 8 issue slots, four of them the exponential, and the
// gradient 8 more: by count, a row of 128000 bf16 classes takes a compute unit 18 us of those and 24 us of its share of the memory.  Policy loss with gradient of 8192 such rows:
// 813 us, 5.2 TB/s; its value alone of 2048 rows of 32000, one in five masked: 25.4 us, 4.1 TB/s; exact divergence of 4096 rows of 50257, one in ten masked: 263 us, 4.4 TB/s (calls that
// go on; the first thirty of a process take up to 306).
#pragma once
#include <cmath>
#include <type_traits>

#include "context.h"
#include "op_args.h"

namespace et {
namespace rows {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Vectors are loaded and stored at the alignment of an element, which global memory takes on this hardware
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

// log2 e in float32 is LOG2E = (1 + SKEW) log2 e.  Exponentials taken with it are those of (1 + SKEW) (x - m), which moves log S by SKEW E[x - m]: of one sign, it adds up over the
// rows of a sequence, so it is taken off again, E from the first element of every vector.  (log p of 4096 rows of 100003 classes: -2e-8 to -4e-8 in the mean without that, 1e-8
// with it, 2e-7 in the root mean square; the mean margin of 16 sequences of 500 such rows: 1.3e-6 and 3e-7 of its value.)
constexpr float LOG2E = 1.44269502162933349609375f;
constexpr double SKEW = -1.3349817e-8;
constexpr float LOWEST = -3.4028234663852886e38f;   // the reference of nothing: x - LOWEST of x = -inf is -inf, and its exponential 0

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
// 2^u for a row's scalars: reduced in float64, so that what is off is the hardware's exponential on [-1/2, 1/2], 2^-23 of the value
__device__ __forceinline__ double exp2_d(double u) {
  u = u < -1200 ? -1200 : u;
  u = u > 1200 ? 1200 : u;
  const double n = rint(u);
  return ldexp((double)exp2_of((float)(u - n)), n == n ? (int)n : 0);
}
__device__ __forceinline__ float exp_of(float d) { return exp2_of(d * LOG2E); }
__device__ __forceinline__ double exp_d(double d) { return exp2_d(d * 1.4426950408889634); }
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

// log x, x > 0: the hardware's logarithm is taken of the mantissa, so that it is off by 2^-24 and not by that of the whole
__device__ __forceinline__ double log_d(double x) {
  const int e = __builtin_amdgcn_frexp_exp(x);
  return ((double)e + (double)__builtin_amdgcn_logf((float)__builtin_amdgcn_frexp_mant(x))) * 0.69314718055994530942;
}
// log(1 + q), 0 <= q <= 1, to rounding also where it is small: 2 artanh z, z = q / (2 + q)
__device__ __forceinline__ double log1p_d(double q) {
  const double z = q / (2.0 + q);
  const float y = (float)(z * z), c[6] = {1.f / 13, 1.f / 11, 1.f / 9, 1.f / 7, 1.f / 5, 1.f / 3};
  float s = 1.f / 15;
#pragma unroll
  for (int i = 0; i < 6; i++) s = fmaf(s, y, c[i]);
  return 2.0 * (z + z * (double)(y * s));
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
template <bool NT, typename V, typename P>
__device__ __forceinline__ void put(V v, P* at) {
  if (NT) __builtin_nontemporal_store(v, at);
  else *at = v;
}
// N values of a gradient
template <typename G, bool NT = false, int N>
__device__ __forceinline__ void store_vec(G* o, const float (&f)[N]) {
  if constexpr (sizeof(G) == 2 && N == 8) {
    u32x4 v;
#pragma unroll
    for (int k = 0; k < 4; k++) v[k] = pack2(f[2 * k], f[2 * k + 1]);
    put<NT>(v, (u32x4_any*)o);
  } else if constexpr (sizeof(G) == 2) {
    u32x2 v;
    v[0] = pack2(f[0], f[1]);
    v[1] = pack2(f[2], f[3]);
    put<NT>(v, (u32x2_any*)o);
  } else {
#pragma unroll
    for (int h = 0; h < N / 4; h++) {
      u32x4 v;
#pragma unroll
      for (int k = 0; k < 4; k++) v[k] = __float_as_uint(f[4 * h + k]);
      put<NT>(v, (u32x4_any*)(o + 4 * h));
    }
  }
}

// ---- over the lanes of a wave (LANES = 64), or the first LANES of it, without the LDS: within rows of 16 lanes, then from row to row; the result in every lane
template <int LANES, typename F>
__device__ __forceinline__ float lanes_reduce(float v, float none, F f) {
#define ET_DPP(CTRL, ROWS) \
  v = f(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xf, false)))
  ET_DPP(0x111, 0xf);
  if (LANES > 2) ET_DPP(0x112, 0xf);
  if (LANES > 4) ET_DPP(0x114, 0xf);
  if (LANES > 8) ET_DPP(0x118, 0xf);
  if (LANES > 16) {
    ET_DPP(0x142, 0xa);
    ET_DPP(0x143, 0xc);
  }
#undef ET_DPP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), LANES - 1));
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_reduce<LANES>(v, LOWEST, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_reduce<LANES>(v, 0.f, [](float a, float b) { return a + b; });
}

// ---- softmax statistics as they run along a row.  m: the reference, at first the maximum of what came first and raised only to what lies far above it (sums of
// numbers up to 2^16 are as exact as those of numbers up to 1); s = sum exp(x - m).
struct Sum {
  float m, s;
  __device__ __forceinline__ void start() { m = LOWEST, s = 0.f; }
  __device__ __forceinline__ bool above(float top) const { return top > m + 11.f; }
  __device__ __forceinline__ float raise(float to) {   // returns the factor
    const float f = exp_of(m - to);
    m = to;
    s *= f;
    return f;
  }
};
// and of the first element of each vector, s0 = sum exp(x - m) and t = sum exp(x - m) (x - m)
struct Run : Sum {
  float s0, t;
  __device__ __forceinline__ void start() { Sum::start(), s0 = t = 0.f; }
  __device__ __forceinline__ float raise(float to) {
    const float by = fmaxf(m - to, -1e4f), f = Sum::raise(to);   // (beyond 1e4 nothing is left of the terms)
    t = f * fmaf(s0, by, t);
    s0 *= f;
    return f;
  }
  __device__ __forceinline__ void first(float d, float e) {
    t = fmaf(e, fmaxf(d, -1e4f), t);
    s0 += e;
  }
};
// (the builtin maximum would first quiet every operand, an instruction each)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int N>
__device__ __forceinline__ float max_of(const float (&f)[N]) {
  float top = f[0];
#pragma unroll
  for (int k = 1; k < N; k += 2) top = max3(top, f[k], f[k + 1 < N ? k + 1 : k]);
  return top;
}
// dx - dy of two logits' distances to their row's reference.  What is further apart than 1e30 counts as that far, an infinite difference too; minus infinity less itself, of a class that both
// give probability zero, counts for nothing, as its term does
constexpr float FARTHEST = 1e30f;
__device__ __forceinline__ float apart(float dx, float dy) { return __builtin_amdgcn_fmed3f(dx - dy, -FARTHEST, FARTHEST); }
// Two rows at once, and kl = sum over x's terms of term * (dx - dy): of distances, so that what a whole row has in common, be it the type's lowest value, does not count
struct RunPair {
  Run x;
  Sum y;
  float kl;
  __device__ __forceinline__ void start() { x.start(), y.start(), kl = 0.f; }
  template <bool FULL>
  __device__ __forceinline__ void raise_x(float to) {
    const float by = fmaxf(x.m - to, -1e4f), s = x.s, f = x.raise(to);
    if (FULL) kl = f * fmaf(s, by, kl);
  }
  __device__ __forceinline__ void raise_y(float to) {
    if (y.s != 0.f) kl = fmaf(x.s, fminf(to - y.m, FARTHEST), kl);   // (y.s = 0: all infinitely far, to any reference)
    y.raise(to);
  }
  template <bool FULL, int N>
  __device__ __forceinline__ void add(const float (&f)[N], const float (&g)[N]) {
    const float top = max_of(f);
    if (x.above(top)) raise_x<FULL>(top);
    if (FULL) {
      const float top_y = max_of(g);
      if (y.above(top_y)) raise_y(top_y);
    }
    float sx = 0.f, sy = 0.f;
#pragma unroll
    for (int k = 0; k < N; k++) {
      const float dx = f[k] - x.m, ex = exp_of(dx);
      if (k == 0) x.first(dx, ex);
      sx = k == 0 ? ex : sx + ex;
      if (FULL) {
        const float dy = g[k] - y.m, ey = exp_of(dy);
        kl = fmaf(ex, apart(dx, dy), kl);
        sy = k == 0 ? ey : sy + ey;
      }
    }
    x.s += sx;
    if (FULL) y.s += sy;
  }
  template <bool FULL, int LANES>
  __device__ __forceinline__ void over_lanes() {
    raise_x<FULL>(lanes_max<LANES>(x.m));
    if (FULL) raise_y(lanes_max<LANES>(y.m));
    x.s = lanes_sum<LANES>(x.s);
    x.s0 = lanes_sum<LANES>(x.s0);
    x.t = lanes_sum<LANES>(x.t);
    if (FULL) {
      y.s = lanes_sum<LANES>(y.s);
      kl = lanes_sum<LANES>(kl);
    }
  }
};

struct RowArgs {
  const void* logits;
  long long ld;
  const int32_t* label;
  void* grad;
  long long gld;
  int rows, classes;
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
  double* lp;
  float *m, *s, *rest;   // (s = 0: masked, or without a distribution)
  float* g;              // the gradient is g ([j = a] - p[j])
  int* descend;          // of all: whether offsets descend, so that a row may be in several sequences
  // (the statistics' launch clears it for that of the pairs)
  __device__ __forceinline__ void clear() const {
    if (blockIdx.x == 0 && threadIdx.x == 0) *descend = 0;
  }
};

// what a row's statistics come to: s = sum of the terms against m, ea the label's, rest the others', by: what others' terms were multiplied with
struct RowStat {
  double s, inv_s, ea, rest, lp, by;
  float m;
  bool none;       // no distribution
};
__device__ __forceinline__ RowStat row_stat(const Run& others, float xa) {
  RowStat o;
  const double u = (double)xa - (double)others.m, e = exp_d(-fabs(u));
  const bool above = u > 0;   // (the label becomes the reference)
  o.m = above ? xa : others.m;
  o.by = above ? e : 1.0;
  o.ea = above ? 1.0 : e;
  o.rest = u == INFINITY ? NAN : (double)others.s * o.by;   // (an infinite logit has no log probability: infinity less infinity)
  o.s = o.rest + o.ea;
  o.inv_s = 1.0 / o.s;
  o.none = o.s == 0.0;
  o.lp = o.none ? -INFINITY : o.ea > o.rest ? -log1p_d(o.rest / o.ea) : fmin(u, 0.0) - log_d(o.s);
  if (others.s0 > 0.f) o.lp += SKEW * (double)(others.t / others.s0) * (o.rest * o.inv_s);
  return o;
}

// what the threads of a row need for its gradient: cf exp(x - m), with the exact divergence (cf + ck ((x - m) - (y - my))) times that, and `own` for the label.  All zeros: a
// gradient of zeros.
struct RowGrad {
  float m, cf, ck, my, own;
};

// Adds a row to the sums (loss, surrogate, divergence, clipped) and says what its gradient is made of
__device__ __forceinline__ void policy_row(const PolicyArgs& p, const RowStat& s, double* sum, float old, float adv, float ref, double w, RowGrad& o) {
  if (s.none) return;
  const double A = (double)adv, ratio = exp_d(s.lp - (double)old);
  const bool over = (A > 0 && ratio > p.high) || (A < 0 && ratio < p.low);
  const double surrogate = A * (over ? (A > 0 ? p.high : p.low) : ratio);
  double g = over ? 0.0 : -ratio * A, kl = 0;
  if (p.ref_logp) {
    const double d = (double)ref - s.lp;
    kl = exp_rest(d);
    if (p.kl_coef != 0) g -= p.kl_coef * (d == -INFINITY ? -1.0 : kl + d);   // exp(d) - 1
  }
  sum[0] += w * ((p.kl_coef != 0 ? p.kl_coef * kl : 0.0) - surrogate);
  sum[1] += w * surrogate;
  sum[2] += w * kl;
  if (over) sum[3] += w;
  o.cf = (float)(-w * g * s.inv_s);
  o.own = (float)(w * g * (s.rest * s.inv_s));
}
// The exact divergence on top: the mean distance between the rows less the difference of their logarithms of sums.  NaN where the reference has no distribution, and with it every element
// of the gradient (the distances alone do not show it: what is not a number among them counts for something finite).
__device__ __forceinline__ void full_kl(const PolicyArgs& p, const RowStat& s, const RunPair& run, double* sum, float xa, float ya, double w, RowGrad& o) {
  if (s.none) return;
  const double sum_apart = s.by * (double)fmaf(run.x.s, fmaxf(run.x.m - s.m, -1e4f), run.kl);   // (the label may have become the reference)
  const double mine = (double)apart(xa - s.m, ya - run.y.m);
  const double kk = (sum_apart + (s.ea == 0 ? 0.0 : s.ea * mine)) * s.inv_s;
  const double kl = run.y.s == 0.f ? NAN : kk - (log_d(s.s) - log_d((double)run.y.s)), nan = kl - kl;   // (0 otherwise)
  sum[2] += w * kl;
  if (p.kl_coef == 0) return;
  sum[0] += w * p.kl_coef * kl;
  const double ck = w * p.kl_coef * s.inv_s;
  o.my = run.y.m;
  o.ck = (float)ck;
  o.cf = (float)((double)o.cf - ck * kk + nan);
  o.own = (float)((double)o.own + nan + (s.ea != 0 ? ck * s.ea * (mine - kk) : 0.0));
}

constexpr int AUX_NT = 2;   // cache policy of a buffer load: non-temporal

enum Mode { POLICY, POLICY_FULL, STATS };

constexpr int MAX_GRID = 4096;    // workgroups of the row kernels
constexpr int COLUMNS = 5;        // sums over rows: loss, surrogate, divergence, clipped; unmasked rows
constexpr int COUNT_ROWS = 8192;  // rows that a workgroup counts by itself

// the sum over a workgroup of each thread's n; red: one entry for each wave
__device__ __forceinline__ int block_count(int n, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
  for (int i = 0; i < (int)blockDim.x / 64; i++) n += red[i];
  return n;
}
// unmasked rows among [begin, end), by all threads of a workgroup: their labels come sixteen a thread at once
__device__ __forceinline__ int count_rows(const RowArgs& a, int begin, int end, int* red) {
  constexpr int AT_ONCE = 16;
  int n = 0;
  for (int r0 = begin + (int)threadIdx.x; r0 < end; r0 += AT_ONCE * blockDim.x) {
    int label[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; k++) label[k] = a.label[min(r0 + k * (int)blockDim.x, end - 1)];
#pragma unroll
    for (int k = 0; k < AT_ONCE; k++) n += r0 + k * (int)blockDim.x < end && !a.masked(label[k]) ? 1 : 0;
  }
  return block_count(n, red);
}
// ---- rows.  The kernels below go over the rows r = first, first + step, ...; the threads of a row ("team") are t = 0 .. TPR - 1.  Vectors of a row are those that
// begin at multiples of 16 bytes: vector v of thread t at element head + (v * TPR + t) * N.  What lies in front of the first and behind the last is one element each of the
// first threads (loads and stores of vectors at any element are right too, and cost 8192 rows of 100003 bf16 classes 10 per cent, and 24 where they are only read; the second pass of a
// preference loss makes them).  Of the reference's rows the same elements are loaded as vectors, wherever its rows begin.
template <typename T, int W>
struct RowShape {
  static constexpr int N = Vec<T>::N, TPR = 64 * W;
  int head, Cv, edge, nv, mine;   // elements in front, in vectors, outside of them; vectors of the team, of this thread
  __device__ __forceinline__ RowShape(int C, const T* row, int t) {
    head = min(C, (int)(-(uintptr_t)row & 15) / (int)sizeof(T));
    Cv = (C - head) / N * N;
    edge = C - Cv;
    nv = (Cv / N + TPR - 1) / TPR;
    mine = (Cv / N - t + TPR - 1) / TPR;
  }
  __device__ __forceinline__ int edge_at(int t) const { return t < head ? t : Cv + t; }
};
struct LabelAt {
  int v, t, k;   // vector, thread and element of a label (v = -1: outside of the vectors)
  template <typename T, int W>
  __device__ __forceinline__ LabelAt(const RowShape<T, W>& s, int at) {
    constexpr int N = RowShape<T, W>::N, TPR = RowShape<T, W>::TPR;
    const int i = at - s.head;
    const bool in_vec = i >= 0 && i < s.Cv;
    v = in_vec ? i / N / TPR : -1;
    t = in_vec ? i / N % TPR : i < 0 ? at : at - s.Cv;
    k = i & (N - 1);
  }
};

// the weight of an unmasked row
__device__ __forceinline__ double unit_weight(const RowArgs& a, const int* counts, int n_counts, int* red) {
  if (n_counts == 0) return 1.0 / count_rows(a, 0, a.rows, red);
  int n = 0;
  for (int i = threadIdx.x; i < n_counts; i += blockDim.x) n += counts[i];
  return 1.0 / block_count(n, red);
}

// a row's other inputs
struct RowInputs {
  float xa, ya, old, adv, ref;
  double w;
};
template <typename T, Mode MODE>
__device__ __forceinline__ RowInputs row_inputs(const RowArgs& a, const PolicyArgs& p, int r, int at, double unit) {
  RowInputs o = {0, 0, 0, 0, 0, unit};
  o.xa = (float)((const T*)a.logits + (long long)r * a.ld)[at];
  if (MODE == POLICY_FULL) o.ya = (float)((const T*)p.ref + (long long)r * p.ref_ld)[at];
  if (MODE != STATS) {
    o.old = p.old_logp[r];
    o.adv = p.advantage[r];
    if (p.ref_logp) o.ref = p.ref_logp[r];
    if (p.weight) o.w = (double)p.weight[r];
  }
  return o;
}

__device__ __forceinline__ void stat_row(const SeqRows& o, int r, const RowStat& s) {
  o.m[r] = s.m;
  o.s[r] = (float)s.s;
  o.rest[r] = (float)s.rest;
  o.lp[r] = s.none ? 0.0 : s.lp;
  o.g[r] = 0.f;
}
// a masked row, of which nothing is looked at
template <Mode MODE>
__device__ __forceinline__ void masked_row(const PolicyArgs& p, const SeqRows& o, int r) {
  const RowStat none = {0, 0, 0, 0, 0, 0, 0.f, true};
  if (MODE == STATS) stat_row(o, r, none);
  else if (p.logp) p.logp[r] = 0.f;
}

// what follows from a row's statistics: added to the sums, and what its gradient is made of (zeros before)
template <Mode MODE>
__device__ __forceinline__ RowStat row_result(const PolicyArgs& p, const RunPair& run, const RowInputs& in, double* sum, RowGrad& b) {
  const RowStat s = row_stat(run.x, in.xa);
  b.m = s.m;
  if (MODE != STATS) policy_row(p, s, sum, in.old, in.adv, in.ref, in.w, b);
  if (MODE == POLICY_FULL) full_kl(p, s, run, sum, in.xa, in.ya, in.w, b);
  return s;
}
template <Mode MODE>
__device__ __forceinline__ void row_out(const PolicyArgs& p, const SeqRows& o, int r, const RowStat& s) {
  if (MODE == STATS) stat_row(o, r, s);
  else if (p.logp) p.logp[r] = (float)s.lp;
}

// Adds up a row's statistics over its waves and says what follows from them, in every thread; sums: this team's
template <int W, Mode MODE>
__device__ __forceinline__ RowGrad row_scalars(const PolicyArgs& p, const SeqRows& o, int r, RunPair run, const RowInputs& in, RunPair* red, RowGrad* said,
                                               double* sums) {
  constexpr bool FULL = MODE == POLICY_FULL;
  run.over_lanes<FULL, 64>();
  RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f};
  if (W > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = run;
    __syncthreads();
  }
  if (W == 1 || threadIdx.x < 64) {
    const bool first = (threadIdx.x & 63) == 0;
    if (W > 1) {
      run.start();
      if (threadIdx.x < W) run = red[threadIdx.x];
      run.over_lanes<FULL, W>();
    }
    double sum[4] = {0, 0, 0, 0};
    const RowStat s = row_result<MODE>(p, run, in, sum, b);
    if (first) {
      row_out<MODE>(p, o, r, s);
      if (MODE != STATS) {
#pragma unroll
        for (int i = 0; i < 4; i++) sums[i] += sum[i];
        sums[4] += 1;
      }
    }
    if (W > 1 && first) *said = b;
  }
  if (W > 1) {
    __syncthreads();
    b = *said;
  }
  return b;
}

// ck = 0 without the exact divergence
template <bool FULL, int N>
__device__ __forceinline__ void gradient(const RowGrad& b, const float (&f)[N], const float (&g)[N], float (&out)[N]) {
#pragma unroll
  for (int k = 0; k < N; k++) {
    const float d = f[k] - b.m, e = exp_of(d);
    out[k] = e * (FULL ? fmaf(b.ck, apart(d, g[k] - b.my), b.cf) : b.cf);
  }
}

// One row of W waves (W = 1: four rows in a workgroup, a wave each) that stays in registers, at most NV vectors a thread: the logits are read once, and as each
// vector has become a piece of the gradient the same vector of the next row is loaded in its place, so that loads are on the way all the time, though a row is read and
// written by turns.  Loads go through buffer descriptors: lanes beyond the row and rows that are not looked at ask for nothing, without a branch around the load (with
// one the vectors were copied from register to register, which waits for them).
// NT: past the caches, both ways.
template <typename T, typename G, int W, int NV, Mode MODE, bool GRAD, bool NT>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, 4) void kept_kernel(RowArgs a, PolicyArgs p, Sequences seq, SeqRows o, const int* __restrict__ counts, int n_counts,
                                                                        double* __restrict__ parts) {
  constexpr int N = Vec<T>::N, TPR = 64 * W, TEAMS = W == 1 ? 4 : 1;
  constexpr bool FULL = MODE == POLICY_FULL;
  __shared__ RunPair red[W];
  __shared__ RowGrad said;
  __shared__ double sums[TEAMS][COLUMNS];
  __shared__ int red_n[16];
  const int t = threadIdx.x % TPR, team = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const int step = gridDim.x * TEAMS;
  if (MODE == STATS) o.clear();
  const int begin = MODE == STATS ? seq.at(0) : 0, end = MODE == STATS ? seq.at(seq.n) : a.rows;
  auto label_of = [&](int r) {
    const int label = a.label[r];
    return __builtin_amdgcn_readfirstlane(r >= begin && r < end ? label : -1);
  };
  u32x4 x[NV], y[FULL ? NV : 1];
  auto row_x = [&](int r) { return (const T*)a.logits + (long long)r * a.ld; };
  auto row_y = [&](int r) { return (const T*)p.ref + (long long)r * p.ref_ld; };
  auto source = [&](const T* row, const RowShape<T, W>& s, bool there) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(row + s.head), 0, there ? s.Cv * (int)sizeof(T) : 0, 0x00027000);
  };
  auto vec_of = [&](__amdgpu_buffer_rsrc_t s, int v) { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(s, t * 16, v * TPR * 16, NT ? AUX_NT : 0)); };
  int r = blockIdx.x * TEAMS + team, at = r < a.rows ? label_of(r) : -1;
  RowShape<T, W> shape(a.classes, row_x(min(r, a.rows - 1)), t);
  {
    const auto sx = source(row_x(min(r, a.rows - 1)), shape, !a.masked(at)), sy = source(row_y(min(r, a.rows - 1)), shape, FULL && !a.masked(at));
#pragma unroll
    for (int v = 0; v < NV; v++) {
      x[v] = vec_of(sx, v);
      if (FULL) y[v] = vec_of(sy, v);
    }
  }
  double unit = 0;   // weight of an unmasked row
  if (MODE != STATS) {
    if (threadIdx.x < TEAMS * COLUMNS) sums[threadIdx.x / COLUMNS][threadIdx.x % COLUMNS] = 0;
    if (!p.weight) unit = GRAD ? unit_weight(a, counts, n_counts, red_n) : 1.0;
    __syncthreads();
  }
  while (r < a.rows) {
    const int next = (int)min((long long)r + step, (long long)a.rows), next_at = next < a.rows ? label_of(next) : -1;
    const bool look = !a.masked(at), more = !a.masked(next_at);
    const int then = min(next, a.rows - 1);
    const RowShape<T, W> shape_then(a.classes, row_x(then), t);
    const auto sx = source(row_x(then), shape_then, more), sy = source(row_y(then), shape_then, FULL && more);
    RowInputs in = {0, 0, 0, 0, 0, 0};
    float x_edge = -INFINITY, y_edge = -INFINITY;
    RunPair run;
    run.start();
    LabelAt place(shape, at);
    if (!look) place.v = place.t = -2;
    asm volatile("" : "+v"(shape.mine));   // (or what is compared with it is kept, in registers that spill)
    if (look) {
      in = row_inputs<T, MODE>(a, p, r, at, unit);
      if (t < shape.edge) {
        if (!(place.v < 0 && t == place.t)) x_edge = (float)row_x(r)[shape.edge_at(t)];
        if (FULL) y_edge = (float)row_y(r)[shape.edge_at(t)];
      }
#pragma unroll
      for (int v = 0; v < NV; v++)
        if (v < shape.mine) {
          if (v == place.v) {
            if (t == place.t) take_out<T>(x[v], place.k);
          }
          float f[N], g[N];
          unpack<T>(x[v], f);
          if (FULL) unpack<T>(y[v], g);
          run.add<FULL>(f, g);
        }
      if (t < shape.edge) {
        const float f[1] = {x_edge}, g[1] = {y_edge};
        run.add<FULL>(f, g);
      }
    }
    if (!GRAD) {
#pragma unroll
      for (int v = 0; v < NV; v++) {
        x[v] = vec_of(sx, v);
        if (FULL) y[v] = vec_of(sy, v);
      }
    }
    RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f};
    if (look) {
      b = row_scalars<W, MODE>(p, o, r, run, in, red, &said, sums[team]);
    } else if (t == 0) {
      masked_row<MODE>(p, o, r);
    }
    if (GRAD) {
      G* const out = (G*)a.grad + (long long)r * a.gld;
#pragma unroll
      for (int v = 0; v < NV; v++) {
        if (v < shape.mine) {
          float f[N], g[N], d[N];
          asm volatile("" : "+v"(x[v]));   // (unpacked again: kept from the first pass it would take twice the registers)
          unpack<T>(x[v], f);
          if (FULL) {
            asm volatile("" : "+v"(y[v]));
            unpack<T>(y[v], g);
          }
          gradient<FULL>(b, f, g, d);
          if (v == place.v) {
            if (t == place.t)
#pragma unroll
              for (int k = 0; k < N; k++) d[k] = k == place.k ? b.own : d[k];
          }
          store_vec<G, NT>(out + shape.head + v * TPR * N + (unsigned)(t * N), d);
        }
        x[v] = vec_of(sx, v);
        if (FULL) y[v] = vec_of(sy, v);
      }
      if (t < shape.edge) {
        const float f[1] = {look ? x_edge : 0.f}, g[1] = {look ? y_edge : 0.f};
        float d[1];
        gradient<FULL>(b, f, g, d);
        out[shape.edge_at(t)] = (G)(place.v == -1 && t == place.t ? b.own : d[0]);
      }
    }
    r = next;
    at = next_at;
    shape = shape_then;
  }
  if (MODE != STATS) {
    __syncthreads();
    if (threadIdx.x < COLUMNS) {
      double sum = sums[0][threadIdx.x];
#pragma unroll
      for (int i = 1; i < TEAMS; i++) sum += sums[i][threadIdx.x];
      parts[blockIdx.x * COLUMNS + threadIdx.x] = sum;
    }
  }
}

// Short rows: a wave takes ROWS of them at a time, which stay in registers, and the scalars of all of them are worked out at once, a row in each of its first lanes (in the
// kernel above they are most of such a row's instructions).
constexpr int GROUP_ROWS = 4, GROUP_VECS = 2;
template <typename T, typename G, int ROWS, int NV, Mode MODE, bool GRAD>
__global__ __launch_bounds__(256, 4) void group_kernel(RowArgs a, PolicyArgs p, Sequences seq, SeqRows o, const int* __restrict__ counts, int n_counts,
                                                       double* __restrict__ parts) {
  constexpr int N = Vec<T>::N;
  constexpr bool FULL = MODE == POLICY_FULL;
  __shared__ int red_n[4];
  __shared__ double sums[4][COLUMNS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  double unit = 0, sum[4] = {0, 0, 0, 0}, seen = 0;
  if (MODE == STATS) o.clear();
  if (MODE != STATS && !p.weight) unit = GRAD ? unit_weight(a, counts, n_counts, red_n) : 1.0;
  const int begin = MODE == STATS ? seq.at(0) : 0, end = MODE == STATS ? seq.at(seq.n) : a.rows;
  for (long long first = (long long)wave * ROWS; first < a.rows; first += (long long)gridDim.x * 4 * ROWS) {
    const int r0 = (int)first, mine = min(r0 + lane, a.rows - 1);
    const bool there = lane < ROWS && r0 + lane < a.rows;
    int label = there && mine >= begin && mine < end ? a.label[mine] : -1;
    const bool look = !a.masked(label);
    if (!look) label = -1;
    RowInputs in = {0, 0, 0, 0, 0, 0};
    if (look) in = row_inputs<T, MODE>(a, p, mine, label, unit);
    u32x4 x[ROWS][NV], y[FULL ? ROWS : 1][NV];
    float xe[ROWS], ye[ROWS];
    int at[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; i++) {
      at[i] = __builtin_amdgcn_readlane(label, i);
      const int r = min(r0 + i, a.rows - 1);
      const T *rx = (const T*)a.logits + (long long)r * a.ld, *ry = FULL ? (const T*)p.ref + (long long)r * p.ref_ld : rx;
      const RowShape<T, 1> s(a.classes, rx, lane);
      const int bytes = a.masked(at[i]) ? 0 : s.Cv * (int)sizeof(T);   // (beyond the row, and of a masked one, nothing is asked for)
      const auto sx = __builtin_amdgcn_make_buffer_rsrc((void*)(rx + s.head), 0, bytes, 0x00027000), sy = __builtin_amdgcn_make_buffer_rsrc((void*)(ry + s.head), 0, bytes, 0x00027000);
#pragma unroll
      for (int v = 0; v < NV; v++) {
        x[i][v] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(sx, lane * 16, v * 64 * 16, 0));
        if (FULL) y[i][v] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(sy, lane * 16, v * 64 * 16, 0));
      }
      xe[i] = ye[i] = 0.f;
      if (!a.masked(at[i]) && lane < s.edge) {
        xe[i] = (float)rx[s.edge_at(lane)];
        if (FULL) ye[i] = (float)ry[s.edge_at(lane)];
      }
    }
    RunPair of_mine;
    of_mine.start();
#pragma unroll
    for (int i = 0; i < ROWS; i++) {
      const RowShape<T, 1> s(a.classes, (const T*)a.logits + (long long)min(r0 + i, a.rows - 1) * a.ld, lane);
      const LabelAt place(s, at[i]);
      RunPair run;
      run.start();
#pragma unroll
      for (int v = 0; v < NV; v++)
        if (v < s.mine) {
          if (v == place.v && lane == place.t) take_out<T>(x[i][v], place.k);
          float f[N], g[N];
          unpack<T>(x[i][v], f);
          if (FULL) unpack<T>(y[i][v], g);
          run.add<FULL>(f, g);
        }
      if (place.v < 0 && lane == place.t) xe[i] = -INFINITY;
      if (lane < s.edge) {
        const float f[1] = {xe[i]}, g[1] = {ye[i]};
        run.add<FULL>(f, g);
      }
      run.over_lanes<FULL, 64>();
      if (lane == i) of_mine = run;
    }
    RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f};
    if (look) {
      row_out<MODE>(p, o, mine, row_result<MODE>(p, of_mine, in, sum, b));
      seen += 1;
    } else if (there) {
      masked_row<MODE>(p, o, mine);
    }
    if (!GRAD) continue;
#pragma unroll
    for (int i = 0; i < ROWS; i++) {
      if (r0 + i >= a.rows) break;
      auto of = [&](float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), i)); };
      const RowGrad c = {of(b.m), of(b.cf), of(b.ck), of(b.my), of(b.own)};
      const RowShape<T, 1> s(a.classes, (const T*)a.logits + (long long)(r0 + i) * a.ld, lane);
      const LabelAt place(s, at[i]);
      G* const out = (G*)a.grad + (long long)(r0 + i) * a.gld;
#pragma unroll
      for (int v = 0; v < NV; v++)
        if (v < s.mine) {
          float f[N], g[N], d[N];
          unpack<T>(x[i][v], f);
          if (FULL) unpack<T>(y[i][v], g);
          gradient<FULL>(c, f, g, d);
#pragma unroll
          for (int k = 0; k < N; k++) d[k] = v == place.v && lane == place.t && k == place.k ? c.own : d[k];
          store_vec(out + s.head + (v * 64 + lane) * N, d);
        }
      if (lane < s.edge) {
        const float f[1] = {xe[i]}, g[1] = {ye[i]};
        float d[1];
        gradient<FULL>(c, f, g, d);
        out[s.edge_at(lane)] = (G)(place.v == -1 && lane == place.t ? c.own : d[0]);
      }
    }
  }
  if (MODE != STATS) {
    double line[COLUMNS] = {sum[0], sum[1], sum[2], sum[3], seen};
#pragma unroll
    for (int i = 0; i < COLUMNS; i++) {
#pragma unroll
      for (int d = 1; d < ROWS; d *= 2) line[i] += __shfl_xor(line[i], d, 64);
      if (lane == 0) sums[threadIdx.x >> 6][i] = line[i];
    }
    __syncthreads();
    if (threadIdx.x < COLUMNS) parts[blockIdx.x * COLUMNS + threadIdx.x] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
  }
}

// Rows of any length, streamed through a window of U vectors a thread: as each has been used the vector U further on is loaded in its place.  Where there is a gradient
// the row passes twice, and the beginning of the second pass is on the way before the first has ended.  That second pass finds the row in the last-level cache: sixteen waves a row leave
// one on a compute unit at a time, and the gradient goes past the cache (2197 rows of 96785 float32 classes: 385 us, 4.4 TB/s counting logits and gradient once; with stores through the
// cache 411, with rows of four waves, four on a compute unit, 525).
template <typename T, typename G, int W, int U, Mode MODE, bool GRAD, bool NT>
__global__ __launch_bounds__(64 * W, 4) void streamed_kernel(RowArgs a, PolicyArgs p, Sequences seq, SeqRows o, const int* __restrict__ counts, int n_counts,
                                                             double* __restrict__ parts) {
  constexpr int N = Vec<T>::N, TPR = 64 * W;
  constexpr bool FULL = MODE == POLICY_FULL;
  __shared__ RunPair red[W];
  __shared__ RowGrad said;
  __shared__ double sums[COLUMNS];
  __shared__ int red_n[16];
  const int t = threadIdx.x;
  double unit = 0;
  if (MODE == STATS) o.clear();
  if (MODE != STATS) {
    if (threadIdx.x < COLUMNS) sums[threadIdx.x] = 0;
    if (!p.weight) unit = GRAD ? unit_weight(a, counts, n_counts, red_n) : 1.0;
    __syncthreads();
  }
  const int begin = MODE == STATS ? seq.at(0) : 0, end = MODE == STATS ? seq.at(seq.n) : a.rows;
  for (int r = blockIdx.x; r < a.rows; r = (int)min((long long)r + gridDim.x, (long long)a.rows)) {
    const int label = a.label[r], at = __builtin_amdgcn_readfirstlane(r >= begin && r < end ? label : -1);
    const bool look = !a.masked(at);
    const T *x = (const T*)a.logits + (long long)r * a.ld, *y = FULL ? (const T*)p.ref + (long long)r * p.ref_ld : x;
    const RowShape<T, W> shape(a.classes, x, t);
    const int turn = (shape.nv + U - 1) / U * U;   // where the second pass begins
    const int bytes = look ? shape.Cv * (int)sizeof(T) : 0;
    const auto sx = __builtin_amdgcn_make_buffer_rsrc((void*)(x + shape.head), 0, bytes, 0x00027000),
               sy = __builtin_amdgcn_make_buffer_rsrc((void*)(y + shape.head), 0, bytes, 0x00027000);
    u32x4 ux[U], uy[FULL ? U : 1];
    auto fetch = [&](int v, int i) {
      const int at = ((v + i) * TPR + t) * 16;   // (beyond the row: nothing is asked for)
      ux[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(sx, at, 0, NT ? AUX_NT : 0));
      if (FULL) uy[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(sy, at, 0, NT ? AUX_NT : 0));
    };
#pragma unroll
    for (int i = 0; i < U; i++) fetch(0, i);
    LabelAt place(shape, at);
    if (!look) place.v = place.t = -2;
    RowGrad b = {0.f, 0.f, 0.f, 0.f, 0.f};
    float x_edge = -INFINITY, y_edge = -INFINITY;
    if (look) {
      const RowInputs in = row_inputs<T, MODE>(a, p, r, at, unit);
      if (t < shape.edge) {
        if (!(place.v < 0 && t == place.t)) x_edge = (float)x[shape.edge_at(t)];
        if (FULL) y_edge = (float)y[shape.edge_at(t)];
      }
      RunPair run;
      run.start();
      for (int v = 0; v < turn; v += U) {
        const int then = GRAD && v + U == turn ? 0 : v + U;
#pragma unroll
        for (int i = 0; i < U; i++) {
          if (v + i < shape.mine) {
            if (v + i == place.v) {
              if (t == place.t) take_out<T>(ux[i], place.k);
            }
            float f[N], g[N];
            unpack<T>(ux[i], f);
            if (FULL) unpack<T>(uy[i], g);
            run.add<FULL>(f, g);
          }
          fetch(then, i);
        }
      }
      if (t < shape.edge) {
        const float f[1] = {x_edge}, g[1] = {y_edge};
        run.add<FULL>(f, g);
      }
      b = row_scalars<W, MODE>(p, o, r, run, in, red, &said, sums);
    } else if (t == 0) {
      masked_row<MODE>(p, o, r);
    }
    if (!GRAD) continue;
    G* const out = (G*)a.grad + (long long)r * a.gld;
    for (int v = 0; v < turn; v += U)
#pragma unroll
      for (int i = 0; i < U; i++) {
        if (v + i < shape.mine) {
          float f[N], g[N], d[N];
          unpack<T>(ux[i], f);
          if (FULL) unpack<T>(uy[i], g);
          gradient<FULL>(b, f, g, d);
          if (v + i == place.v) {
            if (t == place.t)
#pragma unroll
              for (int k = 0; k < N; k++) d[k] = k == place.k ? b.own : d[k];
          }
          store_vec<G, true>(out + shape.head + (size_t)(v + i) * (TPR * N) + t * N, d);
        }
        fetch(v + U, i);
      }
    if (t < shape.edge) {
      const float f[1] = {look ? x_edge : 0.f}, g[1] = {look ? y_edge : 0.f};
      float d[1];
      gradient<FULL>(b, f, g, d);
      out[shape.edge_at(t)] = (G)(place.v == -1 && t == place.t ? b.own : d[0]);
    }
  }
  if (MODE != STATS) {
    __syncthreads();
    if (threadIdx.x < COLUMNS) parts[blockIdx.x * COLUMNS + threadIdx.x] = sums[threadIdx.x];
  }
}

// How rows are taken apart: waves of a row, whether it stays in registers, workgroups at most, whether past the caches
struct RowPlan {
  int waves;
  bool keep;
  int groups;
  bool nt;
  int rows = 1;   // of a wave at a time
  int teams() const { return waves == 1 ? 4 : 1; }
};
// Sixteen vectors a thread (of both rows together) and sixteen waves on a compute unit are what its registers hold.  Where nothing is written rows need not stay: they are
// streamed, a workgroup each, more of them at once than run, so that none has much more of them than another (2048 rows of 32000 classes of which one in five is
// masked take 25.4 us, over the workgroups that run at once 27.8).
// Short rows are taken four at a time where there are more than run at once (16384 rows of 200 bf16 classes 20.3 us, one at a time 24.2; 4096 of 1000 14.1 and 13.1; exact divergence of
// 16384 rows of 200 float32 24.3 and 26.8, but of 1000 bf16, twice the vectors, 38.9 and 37.3).
// A row that a wave's registers hold takes one (16384 rows of 4000 bf16 classes 59 us, with four waves 88).
// Rows no more than compute units leave them idle, so such a row takes more waves: four from a half of a wave's registers on (64 rows of 4000 8.5 us instead of 9.9); with a
// gradient eight from 1024 vectors on (256 rows of 32000 13.9 us instead of 15.4; below, 64 rows of 8000 take 9.1 with four and 9.4 with eight); without one sixteen from 2048 on
// (64 rows of 128000 14.5 us instead of 22.4; one row of 16400 takes 7.8 with four and 8.1 with sixteen).
// Past the caches goes what is read once: preference loss of 7148 rows of 100003 classes 624 us instead of 654, values of 2048 rows of 32000 25.4 instead of 26.4.  What the last-level
// cache holds (256 MB) until the gradient's pass or the next kernel reads it is left there: four short pairs of 32000 classes, 63 MB, would take 41.1 us instead of 35.8.  Loads and stores
// of gradients that it cannot hold: exact divergence of 4096 rows of 50257 classes 264 us instead of 273, policy loss of 8192 of 128000 813 instead of 824.
constexpr double CACHED = 192e6;
inline RowPlan row_plan(int rows, int classes, size_t size, bool full, bool grad, bool again, int cus) {
  const int64_t vecs = ((int64_t)classes * (int64_t)size + 15) / 16, most = full ? 8 : 16, alone = 64 * (full ? 4 : 8);
  const double bytes = (double)rows * classes * size;
  const bool few = rows <= cus;
  if (vecs <= 64 * GROUP_VECS / (full ? 2 : 1) && rows > 16 * cus) return {1, true, 4 * cus, false, GROUP_ROWS};
  if (vecs <= (few ? alone / 2 : alone)) return {1, true, 4 * cus, false};
  const bool nt = bytes > CACHED;
  if (!grad) return {few && vecs > 2048 ? 16 : 4, false, MAX_GRID, !again || nt};
  if (few && vecs > 1024 && vecs <= 512 * most) return {8, true, cus, nt};
  if (vecs <= 256 * most) return {4, true, 4 * cus, nt};
  if (vecs <= 512 * most) return {8, true, 2 * cus, nt};
  if (vecs <= 1024 * most) return {16, true, cus, nt};
  return {16, false, MAX_GRID, false};
}
inline int row_grid(int rows, const RowPlan& plan) { return std::min(std::min(MAX_GRID, plan.groups), (rows - 1) / (plan.teams() * plan.rows) + 1); }

struct RowCall {
  RowArgs a;
  PolicyArgs p;
  Sequences seq;
  SeqRows o;
  const int* counts;
  int n_counts;
  double* parts;
};
template <typename T, typename G, Mode MODE, bool GRAD>
void row_launch(const RowPlan& plan, int grid, hipStream_t s, const RowCall& c) {
  constexpr int F = MODE == POLICY_FULL ? 2 : 1;
#define ET_ROW(KERNEL, W, NV, NT) \
  hipLaunchKernelGGL((KERNEL<T, G, W, NV, MODE, GRAD, NT>), dim3(grid), dim3(W == 1 ? 256 : 64 * W), 0, s, c.a, c.p, c.seq, c.o, c.counts, c.n_counts, c.parts)
  constexpr bool SAME = std::is_same<T, G>::value;   // (a gradient of another type than the logits is rare: not both kinds of kernels)
  if (plan.rows > 1) {
    hipLaunchKernelGGL((group_kernel<T, G, GROUP_ROWS, GROUP_VECS, MODE, GRAD>), dim3(grid), dim3(256), 0, s, c.a, c.p, c.seq, c.o, c.counts, c.n_counts, c.parts);
  } else if (plan.waves == 1) {
    // (4096 rows of 200 bf16 classes 10.9 us, as the first part of eight vectors 11.6)
    if (c.a.classes * sizeof(T) <= 64 * 16 * 2) ET_ROW(kept_kernel, 1, 2, false);
    else ET_ROW(kept_kernel, 1, 8 / F, false);
  } else if constexpr (!GRAD) {
    if (plan.waves == 16 && plan.nt) ET_ROW(streamed_kernel, 16, 8 / F, true);
    else if (plan.waves == 16) ET_ROW(streamed_kernel, 16, 8 / F, false);
    else if (plan.nt) ET_ROW(streamed_kernel, 4, 8 / F, true);
    else ET_ROW(streamed_kernel, 4, 8 / F, false);
  } else if (!plan.keep) {
    ET_ROW(streamed_kernel, 16, 8 / F, false);
  } else if (plan.nt && SAME) {
    if (plan.waves == 4) ET_ROW(kept_kernel, 4, 16 / F, SAME);
    else if (plan.waves == 8) ET_ROW(kept_kernel, 8, 16 / F, SAME);
    else ET_ROW(kept_kernel, 16, 16 / F, SAME);
  } else {
    if (plan.waves == 4) ET_ROW(kept_kernel, 4, 16 / F, false);
    else if (plan.waves == 8) ET_ROW(kept_kernel, 8, 16 / F, false);
    else ET_ROW(kept_kernel, 16, 16 / F, false);
  }
#undef ET_ROW
}

// the kernels of one type of logits (a translation unit each)
template <typename T>
void rows_of_policy(const RowPlan& plan, int grid, hipStream_t s, const RowCall& c, bool grad_bf16);
template <typename T>
void rows_of_statistics(const RowPlan& plan, int grid, hipStream_t s, const RowCall& c);

#define ET_ROWS_OF(T)                                                                                                       \
  template <>                                                                                                               \
  void rows_of_policy<T>(const RowPlan& plan, int grid, hipStream_t s, const RowCall& c, bool grad_bf16) {                  \
    if (c.p.ref) {                                                                                                          \
      if (!c.a.grad) row_launch<T, T, POLICY_FULL, false>(plan, grid, s, c);                                                \
      else if (grad_bf16) row_launch<T, bf16, POLICY_FULL, true>(plan, grid, s, c);                                         \
      else row_launch<T, float, POLICY_FULL, true>(plan, grid, s, c);                                                       \
    } else {                                                                                                                \
      if (!c.a.grad) row_launch<T, T, POLICY, false>(plan, grid, s, c);                                                     \
      else if (grad_bf16) row_launch<T, bf16, POLICY, true>(plan, grid, s, c);                                              \
      else row_launch<T, float, POLICY, true>(plan, grid, s, c);                                                            \
    }                                                                                                                       \
  }                                                                                                                         \
  template <>                                                                                                               \
  void rows_of_statistics<T>(const RowPlan& plan, int grid, hipStream_t s, const RowCall& c) {                              \
    row_launch<T, T, STATS, false>(plan, grid, s, c);                                                                       \
  }

}  // namespace rows
}  // namespace et
