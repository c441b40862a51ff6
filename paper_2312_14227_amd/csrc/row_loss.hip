// Losses of log probabilities over rows of logits, with their gradients: the clipped policy loss with a divergence term, and the
// preference loss of pairs of sequences (et_policy_loss, et_preference_loss).  The row kernels are in row_loss.h.
//
// The policy's gradient follows from each row alone: one pass.  That of a pair follows from the sums over both its sequences, so a first pass takes the
// rows' statistics, a workgroup per pair adds them up, and a second pass maps the logits to their gradient.
#include "row_loss.h"

namespace et {
namespace rows {
namespace {

__global__ __launch_bounds__(256) void count_kernel(RowArgs a, int* __restrict__ counts) {
  __shared__ int red[4];
  const long long per = ((long long)a.rows + gridDim.x - 1) / gridDim.x;
  const int n = count_rows(a, (int)min((long long)a.rows, per * blockIdx.x), (int)min((long long)a.rows, per * (blockIdx.x + 1)), red);
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// Adds the lines of partial sums, by a workgroup: out = scale * column 0, more[i - 1] = scale * column i.  OF >= 0: divided by that column instead (zero over zero is zero)
template <int THREADS, int COLS, int OF>
__device__ __forceinline__ void finish(const double* __restrict__ parts, int lines, double scale, float* __restrict__ out, float* __restrict__ more, int n_more) {
  __shared__ double red[THREADS / 64][COLS];
  double v[COLS];
#pragma unroll
  for (int i = 0; i < COLS; i++) v[i] = 0;
  constexpr int AT_ONCE = 4;
  for (int l0 = threadIdx.x; l0 < lines; l0 += AT_ONCE * THREADS) {
    double line[AT_ONCE][COLS];
#pragma unroll
    for (int k = 0; k < AT_ONCE; k++)
#pragma unroll
      for (int i = 0; i < COLS; i++) line[k][i] = parts[(size_t)COLS * min(l0 + k * THREADS, lines - 1) + i];
#pragma unroll
    for (int k = 0; k < AT_ONCE; k++)
#pragma unroll
      for (int i = 0; i < COLS; i++) v[i] += l0 + k * THREADS < lines ? line[k][i] : 0.0;
  }
#pragma unroll
  for (int i = 0; i < COLS; i++) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v[i] += __shfl_xor(v[i], o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][i] = v[i];
  }
  __syncthreads();
  if (threadIdx.x >= COLS) return;
  double n = 0, s = 0;
  for (int w = 0; w < THREADS / 64; w++) {
    s += red[w][threadIdx.x];
    if (OF >= 0) n += red[w][OF < 0 ? 0 : OF];
  }
  if (OF >= 0) scale = n > 0 ? 1 / n : 0;
  if (threadIdx.x == 0) *out = (float)(s * scale);
  else if (more && (int)threadIdx.x <= n_more) more[threadIdx.x - 1] = (float)(s * scale);
}
template <int THREADS, int COLS, int OF>
__global__ __launch_bounds__(THREADS) void finish_kernel(const double* __restrict__ parts, int lines, double scale, float* __restrict__ out, float* __restrict__ more,
                                                         int n_more) {
  finish<THREADS, COLS, OF>(parts, lines, scale, out, more, n_more);
}
// (2048 lines of workgroups' sums: 256 threads take 1.4 us less than 1024; 4096: 0.4 less; 8000 of pairs': 0.9 more)
template <int COLS, int OF>
void finish_launch(hipStream_t s, const double* parts, int lines, double scale, float* out, float* more, int n_more) {
  if (lines <= 4096) hipLaunchKernelGGL((finish_kernel<256, COLS, OF>), dim3(1), dim3(256), 0, s, parts, lines, scale, out, more, n_more);
  else hipLaunchKernelGGL((finish_kernel<1024, COLS, OF>), dim3(1), dim3(1024), 0, s, parts, lines, scale, out, more, n_more);
}

// ---- preference
struct PairArgs {
  const float* ref;
  double beta, eps, per_pair;
  float* logp;
};
// log(1 + exp x): infinity of infinity, 0 of minus infinity, and NaN of NaN (which no comparison picks)
__device__ __forceinline__ double softplus(double x) { return x == INFINITY ? x : (x <= 0 ? 0.0 : x) + log1p_d(exp_d(-fabs(x))); }
// of a pair's margin: the factor of its gradient, and its loss
__device__ __forceinline__ float pair_factor(const PairArgs& q, double z) {
  const double up = 1.0 / (1.0 + exp_d(-z)), down = 1.0 / (1.0 + exp_d(z));
  return (float)(((q.eps != 0 ? q.eps * up : 0.0) - (q.eps != 1 ? (1 - q.eps) * down : 0.0)) * q.beta * q.per_pair);
}
__device__ __forceinline__ double pair_loss(const PairArgs& q, double z) {
  return (q.eps != 1 ? (1 - q.eps) * softplus(-z) : 0.0) + (q.eps != 0 ? q.eps * softplus(z) : 0.0);
}
__device__ __forceinline__ double pair_margin(const PairArgs& q, int pair, double chosen, double other) {
  return q.beta * ((chosen - (q.ref ? (double)q.ref[2 * pair] : 0.0)) - (other - (q.ref ? (double)q.ref[2 * pair + 1] : 0.0)));
}

// Pairs of single rows, a wave each: both rows stay in registers.  One pass and two launches instead of two passes and three: 32 pairs of 200 bf16 classes 7.4 us instead of 9.0,
// 8000 pairs 17.6 instead of 27.7, 1000 pairs of 2000 classes 11.3 instead of 13.0.
constexpr int PAIR_VECS = 4;
bool pair_rows_fit(int classes, size_t size) { return (int64_t)classes * (int64_t)size <= 64 * 16 * PAIR_VECS; }
template <typename T, typename G>
__global__ __launch_bounds__(256) void pair_rows_kernel(RowArgs a, PairArgs q, double* __restrict__ parts) {
  constexpr int N = Vec<T>::N, NV = PAIR_VECS;
  const int lane = threadIdx.x & 63, pair = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (2ll * pair + 1 >= a.rows) return;
  u32x4 x[2][NV];
  float xe[2];
  int at[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int r = 2 * pair + i;
    const T* row = (const T*)a.logits + (long long)r * a.ld;
    const RowShape<T, 1> s(a.classes, row, lane);
    at[i] = a.label[r];
#pragma unroll
    for (int v = 0; v < NV; v++)
      if (v < s.mine) x[i][v] = load_vec(row + s.head + (v * 64 + lane) * N);
    xe[i] = lane < s.edge ? (float)row[s.edge_at(lane)] : -INFINITY;
  }
  RowStat stat[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const T* row = (const T*)a.logits + (2ll * pair + i) * a.ld;
    const RowShape<T, 1> s(a.classes, row, lane);
    at[i] = __builtin_amdgcn_readfirstlane(at[i]);
    stat[i] = {0, 0, 0, 0, 0, 0, 0.f, true};
    if (a.masked(at[i])) continue;
    const LabelAt place(s, at[i]);
    const float xa = (float)row[at[i]];
    RunPair run;
    run.start();
#pragma unroll
    for (int v = 0; v < NV; v++)
      if (v < s.mine) {
        if (v == place.v && lane == place.t) take_out<T>(x[i][v], place.k);
        float f[N];
        unpack<T>(x[i][v], f);
        run.add<false>(f, f);
      }
    if (place.v < 0 && lane == place.t) xe[i] = -INFINITY;
    if (lane < s.edge) {
      const float f[1] = {xe[i]};
      run.add<false>(f, f);
    }
    run.over_lanes<false, 64>();
    stat[i] = row_stat(run.x, xa);
  }
  const double L0 = stat[0].none ? 0.0 : stat[0].lp, L1 = stat[1].none ? 0.0 : stat[1].lp, z = pair_margin(q, pair, L0, L1);
  if (lane == 0) {
    if (q.logp) {
      q.logp[2 * pair] = (float)L0;
      q.logp[2 * pair + 1] = (float)L1;
    }
    parts[3 * (size_t)pair] = pair_loss(q, z);
    parts[3 * (size_t)pair + 1] = z;
    parts[3 * (size_t)pair + 2] = z > 0 ? 1.0 : 0.0;
  }
  if (!a.grad) return;
  const float factor = pair_factor(q, z);
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int r = 2 * pair + i;
    const RowShape<T, 1> s(a.classes, (const T*)a.logits + (long long)r * a.ld, lane);
    const LabelAt place(s, at[i]);
    const bool none = stat[i].none;   // (and what a masked row holds is not looked at)
    const float g = i == 0 ? factor : -factor;
    const RowGrad b = {stat[i].m, none ? 0.f : (float)(-g * stat[i].inv_s), 0.f, 0.f, none ? 0.f : (float)(g * (stat[i].rest * stat[i].inv_s))};
    G* const out = (G*)a.grad + (long long)r * a.gld;
#pragma unroll
    for (int v = 0; v < NV; v++)
      if (v < s.mine) {
        float f[N], d[N];
        unpack<T>(x[i][v], f);
        gradient<false>(b, f, f, d);
#pragma unroll
        for (int k = 0; k < N; k++) d[k] = none ? 0.f : v == place.v && lane == place.t && k == place.k ? b.own : d[k];
        store_vec(out + s.head + (v * 64 + lane) * N, d);
      }
    if (lane < s.edge) {
      const float f[1] = {xe[i]};
      float d[1];
      gradient<false>(b, f, f, d);
      out[s.edge_at(lane)] = (G)(none ? 0.f : place.v == -1 && lane == place.t ? b.own : d[0]);
    }
  }
}

// A workgroup a pair, a half of it a sequence: the sums of its rows, eight a thread at once, then the rows' factors.  Where offsets descend several workgroups may write a row's: then none is used
__global__ __launch_bounds__(256) void pair_kernel(Sequences seq, SeqRows o, PairArgs q, double* __restrict__ parts) {
  constexpr int AT_ONCE = 8;
  __shared__ double red[4];
  const int pair = blockIdx.x, i = threadIdx.x >> 7, t = threadIdx.x & 127;
  const int begin = seq.at(2 * pair + i), end = seq.at(2 * pair + i + 1);
  if (t == 0 && end < begin) atomicOr(o.descend, 1);
  double v = 0;
  for (int r0 = begin + t; r0 < end; r0 += AT_ONCE * 128) {
    double lp[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; k++) lp[k] = o.lp[min(r0 + k * 128, end - 1)];
#pragma unroll
    for (int k = 0; k < AT_ONCE; k++) v += r0 + k * 128 < end ? lp[k] : 0.0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  const double L0 = red[0] + red[1], L1 = red[2] + red[3], z = pair_margin(q, pair, L0, L1);
  const float g = pair_factor(q, z);
  for (int r = begin + t; r < end; r += 128) o.g[r] = i == 0 ? g : -g;
  if (t == 0 && q.logp) q.logp[2 * pair + i] = (float)(i == 0 ? L0 : L1);
  if (threadIdx.x == 0) {
    parts[3 * pair] = pair_loss(q, z);
    parts[3 * pair + 1] = z;
    parts[3 * pair + 2] = z > 0 ? 1.0 : 0.0;
  }
}

// The gradient once the factors are known: nothing but a map of the logits.  A wave takes GRAD_VECS vectors a lane of a row at a time, from its first element on,
// at whatever address that lies.  The last workgroup adds up the pairs.
constexpr int GRAD_VECS = 8;
template <typename T, typename G>
__global__ __launch_bounds__(256) void pair_grad_kernel(RowArgs a, Sequences seq, SeqRows o, const double* __restrict__ parts, float* __restrict__ loss,
                                                        float* __restrict__ stats) {
  if (blockIdx.x == gridDim.x - 1) {
    finish<256, 3, -1>(parts, seq.n / 2, 2.0 / seq.n, loss, stats, 2);
    return;
  }
  constexpr int N = Vec<T>::N, PIECE = 64 * N * GRAD_VECS;
  const int begin = seq.at(0), end = seq.at(seq.n), lane = threadIdx.x & 63;
  const int C = a.classes, Cv = C - C % N, pieces = (C - 1) / PIECE + 1;
  const bool descend = *o.descend != 0;
  const long long tasks = (long long)(end - begin) * pieces;
  for (long long task = blockIdx.x * 4ll + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); task < tasks; task += (gridDim.x - 1) * 4ll) {
    const int r = begin + (int)(task / pieces), j0 = (int)(task % pieces) * PIECE;
    G* const out = (G*)a.grad + (long long)r * a.gld;
    const T* x = (const T*)a.logits + (long long)r * a.ld;
    const int at = a.label[r];
    const float s = o.s[r], m = o.m[r], g = o.g[r];
    const bool zero = s == 0.f || descend;
    const float cf = zero ? 0.f : -g / s, own = zero ? 0.f : g * (o.rest[r] / s);
    auto one = [&](float f, int j) { return zero ? 0.f : j == at ? own : cf * exp_of(f - m); };
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
      for (int k = 0; k < N; k++) f[k] = one(f[k], j + k);
      store_vec<G>(out + j, f);
    }
    const int j = Cv + lane;
    if (j < C && Cv >= j0 && Cv < j0 + PIECE) out[j] = (G)one(zero ? 0.f : (float)x[j], j);
  }
}

}  // namespace
}  // namespace rows
}  // namespace et

namespace {

using namespace et_op;

constexpr int MAX_COUNTS = 256;
constexpr size_t POLICY_WS = sizeof(int) * MAX_COUNTS + sizeof(double) * et::rows::COLUMNS * et::rows::MAX_GRID;

constexpr int MOST_PAIRS = 1 << 23;   // (a workgroup each: what a launch can have)
size_t preference_ws(int64_t rows, int64_t pairs) { return (size_t)(rows * 24 + pairs * 24 + 256); }

// whether vectors of n floats, either may be missing, have a byte in common
bool meet(const float* a, const float* b, int64_t n) { return a && b && Span(a, 1, n, 0, 4).meets(Span(b, 1, n, 0, 4)); }

// the arguments that both losses have in common
int check_rows(int32_t rows, int32_t classes, const void* logits, int32_t dtype, int64_t stride, const int32_t* label, const void* grad,
               int32_t grad_dtype, int64_t grad_stride, const void* ws, const float* loss) {
  if (rows < 1 || rows > 1 << 30 || classes < 1 || classes > 1 << 28 || !logits || !label || !ws || !loss || !type_ok(dtype) || (grad && !type_ok(grad_dtype))) return ET_EINVAL;
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

int et_op::policy_loss(int32_t rows, int32_t classes, const void* logits_dev, int32_t dtype, int64_t row_stride, const int32_t* label_dev, const et_policy* p,
                       void* grad_dev, int32_t grad_dtype, int64_t grad_stride, void* workspace_dev, size_t workspace_bytes, hipStream_t s, float* loss_dev,
                       bool check_only, int* launches) {
  const int rc = check_rows(rows, classes, logits_dev, dtype, row_stride, label_dev, grad_dev, grad_dtype, grad_stride, workspace_dev, loss_dev);
  if (rc != ET_OK) return rc;
  if (!p || !p->old_logp_dev || !p->advantage_dev || (p->ref_logp_dev && p->ref_logits_dev)) return ET_EINVAL;
  for (const float* v : {p->old_logp_dev, p->advantage_dev, p->ref_logp_dev, p->weight_dev, (const float*)p->logp_dev, (const float*)p->stats_dev})
    if (!aligned(v, 4)) return ET_EINVAL;
  for (const float* v : {p->old_logp_dev, p->advantage_dev, p->ref_logp_dev, p->weight_dev})
    if (meet(v, p->logp_dev, rows)) return ET_EINVAL;
  if (!(p->clip_low >= 0 && p->clip_low <= 1 && p->clip_high >= 0 && std::isfinite(p->clip_high) && std::isfinite(p->kl_coef))) return ET_EINVAL;
  if (p->ref_logits_dev) {
    if (p->ref_stride < classes || p->ref_stride > (INT64_MAX >> 4) / rows || !aligned(p->ref_logits_dev, type_size(dtype))) return ET_EINVAL;
    if (grad_dev && Span(grad_dev, rows, classes, grad_stride, type_size(grad_dtype)).meets(Span(p->ref_logits_dev, rows, classes, p->ref_stride, type_size(dtype))))
      return ET_EINVAL;
  }
  if (workspace_bytes < POLICY_WS) return ET_ENOMEM;
  if (check_only) return ET_OK;
  const OnDeviceOf on(s);
  if (!on.ok) return ET_EHIP;
  et::rows::RowCall c = {};
  c.a = {logits_dev, row_stride, label_dev, grad_dev, grad_stride, rows, classes};
  c.p = {p->old_logp_dev, p->advantage_dev, p->ref_logp_dev, p->weight_dev, p->ref_logits_dev, p->ref_stride,
         1.0 - (double)p->clip_low, 1.0 + (double)p->clip_high, (double)p->kl_coef, p->logp_dev};
  int* counts = (int*)workspace_dev;
  c.counts = counts;
  c.parts = (double*)(counts + MAX_COUNTS);
  const et::rows::RowPlan plan = et::rows::row_plan(rows, classes, type_size(dtype), c.p.ref != nullptr, grad_dev != nullptr, false, device_cus(on.dev));
  const int grid = et::rows::row_grid(rows, plan);
  if (grad_dev && !p->weight_dev && rows > et::rows::COUNT_ROWS) {
    c.n_counts = std::min(MAX_COUNTS, rows / 1024);
    hipLaunchKernelGGL(et::rows::count_kernel, dim3(c.n_counts), dim3(256), 0, s, c.a, counts);
  }
  if (dtype == ET_BF16) et::rows::rows_of_policy<bf16>(plan, grid, s, c, grad_dtype == ET_BF16);
  else et::rows::rows_of_policy<float>(plan, grid, s, c, grad_dtype == ET_BF16);
  if (launches) *launches = 2 + (c.n_counts != 0);
  // (without a gradient rows have the weight 1 as they are added up)
  if (!grad_dev && !p->weight_dev)
    et::rows::finish_launch<et::rows::COLUMNS, 4>(s, c.parts, grid, 1.0, loss_dev, p->stats_dev, 3);
  else
    et::rows::finish_launch<et::rows::COLUMNS, -1>(s, c.parts, grid, 1.0, loss_dev, p->stats_dev, 3);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

int et_op::preference_loss(int32_t rows, int32_t pairs, int32_t classes, const void* logits_dev, int32_t dtype, int64_t row_stride, const int32_t* label_dev,
                           const et_preference* p, void* grad_dev, int32_t grad_dtype, int64_t grad_stride, void* workspace_dev, size_t workspace_bytes, hipStream_t s,
                           float* loss_dev, bool check_only, int* launches) {
  const int rc = check_rows(rows, classes, logits_dev, dtype, row_stride, label_dev, grad_dev, grad_dtype, grad_stride, workspace_dev, loss_dev);
  if (rc != ET_OK) return rc;
  if (!p || pairs < 1 || pairs > MOST_PAIRS || (!p->offsets_dev && rows != 2 * pairs)) return ET_EINVAL;
  if (!aligned(p->offsets_dev, 4) || !aligned(p->ref_logp_dev, 4) || !aligned(p->logp_dev, 4) || !aligned(p->stats_dev, 4)) return ET_EINVAL;
  if (meet(p->ref_logp_dev, p->logp_dev, 2 * (int64_t)pairs)) return ET_EINVAL;
  if (!(p->beta > 0 && std::isfinite(p->beta) && p->label_smoothing >= 0 && p->label_smoothing <= 1)) return ET_EINVAL;
  if (workspace_bytes < preference_ws(rows, pairs)) return ET_ENOMEM;
  if (check_only) return ET_OK;
  const OnDeviceOf on(s);
  if (!on.ok) return ET_EHIP;
  et::rows::RowCall c = {};
  c.a = {logits_dev, row_stride, label_dev, grad_dev, grad_stride, rows, classes};
  c.seq = {p->offsets_dev, rows, 2 * pairs};
  const et::rows::PairArgs q = {p->ref_logp_dev, (double)p->beta, (double)p->label_smoothing, 1.0 / pairs, p->logp_dev};
  if (!p->offsets_dev && et::rows::pair_rows_fit(classes, type_size(dtype))) {
    if (launches) *launches = 2;
    double* parts = (double*)workspace_dev;
#define ET_PAIR_ROWS(T, G) hipLaunchKernelGGL((et::rows::pair_rows_kernel<T, G>), dim3((pairs + 3) / 4), dim3(256), 0, s, c.a, q, parts)
    if (dtype == ET_BF16) {
      if (grad_dtype == ET_BF16) ET_PAIR_ROWS(bf16, bf16); else ET_PAIR_ROWS(bf16, float);
    } else {
      if (grad_dtype == ET_BF16) ET_PAIR_ROWS(float, bf16); else ET_PAIR_ROWS(float, float);
    }
#undef ET_PAIR_ROWS
    et::rows::finish_launch<3, -1>(s, parts, pairs, 1.0 / pairs, loss_dev, p->stats_dev, 2);
    return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
  }
  if (launches) *launches = 3;
  c.o.lp = (double*)workspace_dev;
  double* parts = c.o.lp + rows;
  c.o.m = (float*)(parts + 3 * (size_t)pairs);
  c.o.s = c.o.m + rows;
  c.o.rest = c.o.s + rows;
  c.o.g = c.o.rest + rows;
  c.o.descend = (int*)(c.o.g + rows);
  const et::rows::RowPlan plan = et::rows::row_plan(rows, classes, type_size(dtype), false, false, grad_dev != nullptr, device_cus(on.dev));
  const int grid = plan.waves == 1 ? et::rows::row_grid(rows, plan) : std::min(rows, 1 << 20);
  if (dtype == ET_BF16) et::rows::rows_of_statistics<bf16>(plan, grid, s, c);
  else et::rows::rows_of_statistics<float>(plan, grid, s, c);
  hipLaunchKernelGGL(et::rows::pair_kernel, dim3(pairs), dim3(256), 0, s, c.seq, c.o, q, parts);
  if (grad_dev) {
    const int64_t piece = 64 * et::rows::GRAD_VECS * (16 / (int64_t)type_size(dtype)), tasks = rows * ((classes + piece - 1) / piece);
    const int groups = (int)std::min<int64_t>((tasks + 3) / 4, 1 << 20);
#define ET_PAIR_GRAD(T, G) hipLaunchKernelGGL((et::rows::pair_grad_kernel<T, G>), dim3(groups + 1), dim3(256), 0, s, c.a, c.seq, c.o, parts, loss_dev, p->stats_dev)
    if (dtype == ET_BF16) {
      if (grad_dtype == ET_BF16) ET_PAIR_GRAD(bf16, bf16); else ET_PAIR_GRAD(bf16, float);
    } else {
      if (grad_dtype == ET_BF16) ET_PAIR_GRAD(float, bf16); else ET_PAIR_GRAD(float, float);
    }
#undef ET_PAIR_GRAD
    return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
  }
  et::rows::finish_launch<3, -1>(s, parts, pairs, 1.0 / pairs, loss_dev, p->stats_dev, 2);
  return hipGetLastError() == hipSuccess ? ET_OK : ET_EHIP;
}

extern "C" {

size_t et_policy_loss_ws_bytes(int32_t rows) { return rows < 1 || rows > 1 << 30 ? 0 : POLICY_WS; }
size_t et_preference_loss_ws_bytes(int32_t rows, int32_t pairs) { return rows < 1 || rows > 1 << 30 || pairs < 1 || pairs > MOST_PAIRS ? 0 : preference_ws(rows, pairs); }

int et_policy_loss(int32_t rows, int32_t classes, const void* logits_dev, int32_t dtype, int64_t row_stride, const int32_t* label_dev,
                   const et_policy* policy, void* grad_dev, int32_t grad_dtype, int64_t grad_stride, void* workspace_dev, size_t workspace_bytes,
                   void* hip_stream, float* loss_dev) {
  return et_op::policy_loss(rows, classes, logits_dev, dtype, row_stride, label_dev, policy, grad_dev, grad_dtype, grad_stride, workspace_dev, workspace_bytes,
                            (hipStream_t)hip_stream, loss_dev, false, nullptr);
}

int et_preference_loss(int32_t rows, int32_t pairs, int32_t classes, const void* logits_dev, int32_t dtype, int64_t row_stride,
                       const int32_t* label_dev, const et_preference* preference, void* grad_dev, int32_t grad_dtype, int64_t grad_stride,
                       void* workspace_dev, size_t workspace_bytes, void* hip_stream, float* loss_dev) {
  return et_op::preference_loss(rows, pairs, classes, logits_dev, dtype, row_stride, label_dev, preference, grad_dev, grad_dtype, grad_stride, workspace_dev,
                                workspace_bytes, (hipStream_t)hip_stream, loss_dev, false, nullptr);
}

}  // extern "C"
