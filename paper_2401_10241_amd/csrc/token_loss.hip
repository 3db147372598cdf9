// Losses on the log-probabilities of given tokens, and the gradient of the logits they come from: with
//   lse_r = log sum_j exp(z_rj),  logp_r = z_r,target(r) - lse_r,  c_r = d(loss) / d(logp_r)
// every loss here has  d(loss) / d(z_rj) = c_r ([j = target(r)] - exp(z_rj - lse_r)).
// A row counts if its target lies in [0, vocab), its weight is not zero and, where there are sequences, one of them holds it;
// the logits of the others are not read.
#include <math.h>

#include "../../include/zb_stage.h"
#include "zb_common.h"

namespace zb {

namespace {

constexpr int kThreads = 256;

struct Rows {
  const int* targets;
  const float* weight;  // null: 1 each
  const int* offsets;   // null: no sequences
  int sequences, vocab;  // sequences < 0: no row counts
  __device__ __forceinline__ bool counts(int row) const {
    const int t = targets[row];
    return sequences >= 0 && t >= 0 && t < vocab && (!weight || weight[row] != 0.f) && (!offsets || (row >= offsets[0] && row < offsets[sequences]));
  }
  __device__ __forceinline__ double weight_of(int row) const { return weight ? (double)weight[row] : 1.0; }
};

// (m, s) stands for s * exp(m); an empty or all -infinity part has m = -infinity and s = 0
__device__ __forceinline__ void lse_merge(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = (m == -INFINITY ? 0.f : s * __expf(m - top)) + (m2 == -INFINITY ? 0.f : s2 * __expf(m2 - top));
  m = top;
}

// lse and log-probability of a row, by one workgroup
template <typename T>
__global__ __launch_bounds__(kThreads) void row_logp_kernel(const T* __restrict__ logits, long stride, Rows of, float* __restrict__ logp,
                                                            float* __restrict__ lse) {
  __shared__ float red_m[kThreads / 64], red_s[kThreads / 64];
  const int row = blockIdx.x;
  const int vocab = of.vocab;
  if (!of.counts(row)) {
    if (threadIdx.x == 0) { if (logp) logp[row] = 0.f; if (lse) lse[row] = 0.f; }
    return;
  }
  const T* z = logits + (long)row * stride;
  float m = -INFINITY, s = 0.f;
  for (int c = threadIdx.x; c < vocab; c += kThreads) {
    const float x = to_f32(z[c]);
    if (x != x) { m = x; s = x; }  // a NaN stays
    else if (m == m) lse_merge(m, s, x, 1.f);
  }
  for (int o = 32; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    if (m2 != m2 || m != m) { m = NAN; s = NAN; }
    else lse_merge(m, s, m2, s2);
  }
  if ((threadIdx.x & 63) == 0) { red_m[threadIdx.x >> 6] = m; red_s[threadIdx.x >> 6] = s; }
  __syncthreads();
  if (threadIdx.x) return;
  m = red_m[0]; s = red_s[0];
  for (int w = 1; w < kThreads / 64; ++w) {
    if (red_m[w] != red_m[w] || m != m) { m = NAN; s = NAN; }
    else lse_merge(m, s, red_m[w], red_s[w]);
  }
  if (m == -INFINITY) s = NAN;  // a row of nothing but -infinity has no softmax
  const double ls = log((double)s);
  if (lse) lse[row] = (float)((double)m + ls);
  if (logp) logp[row] = (float)(((double)to_f32(z[of.targets[row]]) - (double)m) - ls);
}

// coef ([j = target] - exp(z_j - lse)), or zeros where the row does not count
template <typename T>
__global__ __launch_bounds__(kThreads) void row_grad_kernel(const T* logits, long stride, Rows of, const float* __restrict__ lse,
                                                            const float* __restrict__ coef, T* dlogits, long dstride) {
  const int row = blockIdx.x;
  const int vocab = of.vocab, t = of.targets[row];
  const float k = of.counts(row) ? coef[row] : 0.f;
  const bool counts = k != 0.f;  // (also NaN)
  const float l = counts ? lse[row] : 0.f;
  const T* z = logits + (long)row * stride;
  T* d = dlogits + (long)row * dstride;
  for (int c = threadIdx.x; c < vocab; c += kThreads)
    d[c] = counts ? from_f32<T>(k * ((c == t ? 1.f : 0.f) - __expf(to_f32(z[c]) - l))) : from_f32<T>(0.f);
}

struct PolicyArgs {
  const float *old_logp, *ref_logp, *advantage;
  double lo, hi, kl, scale;
};
// loss of a row and its derivative by the row's log-probability
__device__ __forceinline__ double policy_row(const PolicyArgs& a, const Rows& of, int row, double logp, double* slope) {
  const double adv = a.advantage[row], rho = exp(logp - (double)a.old_logp[row]);
  const double w = of.weight_of(row) * a.scale;
  const double held = rho < a.lo ? a.lo : rho > a.hi ? a.hi : rho;
  double loss = -fmin(rho * adv, held * adv);
  double g = (adv > 0 && rho > a.hi) || (adv < 0 && rho < a.lo) ? 0.0 : -adv * rho;
  if (a.kl != 0.0) {
    const double d = (double)a.ref_logp[row] - logp, e = expm1(d);
    loss += a.kl * (e - d);
    g -= a.kl * e;
  }
  *slope = w * g;
  return w * loss;
}

__global__ __launch_bounds__(kThreads) void policy_coef_kernel(PolicyArgs a, Rows of, int rows,
                                                               const float* __restrict__ logp, float* __restrict__ coef,
                                                               double* __restrict__ part) {
  const int row = blockIdx.x * kThreads + threadIdx.x;
  if (row >= rows) return;
  double slope = 0.0, loss = 0.0;
  if (of.counts(row)) loss = policy_row(a, of, row, logp[row], &slope);
  coef[row] = (float)slope;
  part[row] = loss;
}

// sum of n values in a fixed order, by one workgroup
__global__ __launch_bounds__(kThreads) void sum_kernel(const double* __restrict__ part, int n, float* __restrict__ out) {
  __shared__ double red[kThreads];
  double acc = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) acc += part[i];
  red[threadIdx.x] = acc;
  __syncthreads();
  for (int o = kThreads / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *out = (float)red[0];
}

struct PairArgs {
  const float* ref_logp;
  double beta, smoothing, scale;
};
__device__ __forceinline__ void sequence_rows(const int* offsets, int q, int rows, int* a, int* b) {
  const int x = offsets[q], y = offsets[q + 1];
  *a = x < 0 ? 0 : x > rows ? rows : x;
  *b = y < *a ? *a : y > rows ? rows : y;
}
__device__ __forceinline__ double neg_log_sigmoid(double y) { return fmax(-y, 0.0) + log1p(exp(-fabs(y))); }

// One workgroup per pair: both sequences' sums of w (logp - ref), the pair's loss, and the coefficient of every row.
__global__ __launch_bounds__(kThreads) void pair_kernel(PairArgs a, Rows of, int rows,
                                                        const float* __restrict__ logp, float* __restrict__ rewards,
                                                        float* __restrict__ coef, double* __restrict__ part) {
  __shared__ double red[2][kThreads];
  int lo[2], hi[2];
  for (int q = 0; q < 2; ++q) {
    sequence_rows(of.offsets, 2 * blockIdx.x + q, rows, &lo[q], &hi[q]);
    double acc = 0.0;
    for (int r = lo[q] + threadIdx.x; r < hi[q]; r += kThreads)
      if (of.counts(r)) acc += of.weight_of(r) * ((double)logp[r] - (double)a.ref_logp[r]);
    red[q][threadIdx.x] = acc;
  }
  __syncthreads();
  for (int o = kThreads / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) { red[0][threadIdx.x] += red[0][threadIdx.x + o]; red[1][threadIdx.x] += red[1][threadIdx.x + o]; }
    __syncthreads();
  }
  const double sc = red[0][0], sr = red[1][0], x = a.beta * (sc - sr);
  if (threadIdx.x == 0) {
    if (rewards) { rewards[2 * blockIdx.x] = (float)(a.beta * sc); rewards[2 * blockIdx.x + 1] = (float)(a.beta * sr); }
    part[blockIdx.x] = a.scale * ((1.0 - a.smoothing) * neg_log_sigmoid(x) + a.smoothing * neg_log_sigmoid(-x));
  }
  const double slope = a.scale * a.beta * (a.smoothing / (1.0 + exp(-x)) - (1.0 - a.smoothing) / (1.0 + exp(x)));
  for (int q = 0; q < 2; ++q)
    for (int r = lo[q] + threadIdx.x; r < hi[q]; r += kThreads)
      coef[r] = (float)((q ? -slope : slope) * of.weight_of(r));
}

__global__ __launch_bounds__(kThreads) void fill_zero_kernel(float* p, int n) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

constexpr int kMaxRows = 1 << 24;
bool valid_logits(const zb_logits* x) {
  if (!x || x->rows < 0 || x->rows > kMaxRows || x->vocab < 1 || x->vocab > kEmbeddingMaxVocab || x->row_stride < x->vocab) return false;
  if (x->row_stride > (int64_t)1 << 32 || (x->dtype != ZB_FP32 && x->dtype != ZB_BF16)) return false;
  if (x->rows == 0) return true;
  const uintptr_t es = x->dtype == ZB_BF16 ? 2 : 4;
  return x->logits && x->targets && !((uintptr_t)x->logits & (es - 1)) && !((uintptr_t)x->targets & 3);
}
bool valid_dlogits(const zb_logits* x, const void* d, int64_t* stride) {
  if (*stride == 0) *stride = x->row_stride;
  if (*stride < x->vocab || *stride > (int64_t)1 << 32) return false;
  return !((uintptr_t)d & (x->dtype == ZB_BF16 ? 1 : 3));
}
bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

struct Workspace {  // rows: one partial loss, lse, log-probability and coefficient each
  double* part;
  float *lse, *logp, *coef;
};
size_t workspace_bytes(int rows, int pairs) {
  const size_t n = (size_t)(rows > pairs ? rows : pairs);
  return n * sizeof(double) + 3 * (size_t)rows * sizeof(float) + 256;
}
Workspace carve(void* base, int rows, int pairs) {
  Workspace w;
  w.part = (double*)base;
  w.lse = (float*)(w.part + (rows > pairs ? rows : pairs));
  w.logp = w.lse + rows;
  w.coef = w.logp + rows;
  return w;
}

#define ZB_BY_TYPE(x, call)                                     \
  do {                                                          \
    if ((x)->dtype == ZB_BF16) { using T = bf16_t; call; }      \
    else { using T = float; call; }                             \
  } while (0)

void launch_logp(const zb_logits* x, const Rows& of, float* logp, float* lse, hipStream_t s) {
  ZB_BY_TYPE(x, (row_logp_kernel<T><<<x->rows, kThreads, 0, s>>>((const T*)x->logits, x->row_stride, of, logp, lse)));
}
void launch_grad(const zb_logits* x, const Rows& of, const float* lse, const float* coef, void* d, int64_t stride, hipStream_t s) {
  ZB_BY_TYPE(x, (row_grad_kernel<T><<<x->rows, kThreads, 0, s>>>((const T*)x->logits, x->row_stride, of, lse, coef, (T*)d, stride)));
}
zb_status launched() { return hipGetLastError() == hipSuccess ? ZB_OK : ZB_EDEVICE; }

}  // namespace
}  // namespace zb

using namespace zb;

extern "C" {

zb_status zb_token_logprobs(const zb_logits* x, float* logp, float* lse, void* hip_stream) {
  if (!valid_logits(x) || (x->rows && !logp) || misaligned(logp, 4) || misaligned(lse, 4)) return ZB_EINVAL;
  if (x->rows == 0) return ZB_OK;
  OnDeviceOf on((hipStream_t)hip_stream);
  if (!on.ok) return ZB_EDEVICE;
  launch_logp(x, Rows{x->targets, nullptr, nullptr, 0, x->vocab}, logp, lse, (hipStream_t)hip_stream);
  return launched();
}

zb_status zb_token_logprobs_backward(const zb_logits* x, const float* lse, const float* dlogp, void* dlogits, int64_t dlogits_stride,
                                     void* hip_stream) {
  if (!valid_logits(x) || !valid_dlogits(x, dlogits, &dlogits_stride) || misaligned(lse, 4) || misaligned(dlogp, 4)) return ZB_EINVAL;
  if (x->rows == 0) return ZB_OK;
  if (!lse || !dlogp || !dlogits) return ZB_EINVAL;
  OnDeviceOf on((hipStream_t)hip_stream);
  if (!on.ok) return ZB_EDEVICE;
  launch_grad(x, Rows{x->targets, nullptr, nullptr, 0, x->vocab}, lse, dlogp, dlogits, dlogits_stride, (hipStream_t)hip_stream);
  return launched();
}

zb_status zb_loss_workspace_bytes(int32_t rows, int32_t pairs, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxRows || pairs < 0 || pairs > kMaxRows) return ZB_EINVAL;
  *bytes = workspace_bytes(rows, pairs);
  return ZB_OK;
}

zb_status zb_policy_loss(const zb_logits* x, const zb_policy* p, float* loss, float* logp, void* dlogits, int64_t dlogits_stride,
                         void* workspace, size_t workspace_size, void* hip_stream) {
  if (!valid_logits(x) || !p || !loss || !valid_dlogits(x, dlogits, &dlogits_stride)) return ZB_EINVAL;
  if (!(p->clip_low >= 0 && p->clip_low <= 1 && p->clip_high >= 0 && p->kl_coef >= 0) || !isfinite(p->clip_high) ||
      !isfinite(p->kl_coef) || !isfinite(p->scale))
    return ZB_EINVAL;
  if (x->rows && (!p->old_logp || !p->advantage || (p->kl_coef != 0 && !p->ref_logp))) return ZB_EINVAL;
  if (!workspace || misaligned(workspace, 8) || workspace_size < workspace_bytes(x->rows, 0)) return ZB_EINVAL;
  if (misaligned(loss, 4) || misaligned(logp, 4) || misaligned(p->old_logp, 4) || misaligned(p->advantage, 4) || misaligned(p->ref_logp, 4) ||
      misaligned(p->weight, 4))
    return ZB_EINVAL;
  const hipStream_t s = (hipStream_t)hip_stream;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  const Workspace w = carve(workspace, x->rows, 0);
  if (x->rows) {
    const Rows of{x->targets, p->weight, nullptr, 0, x->vocab};
    const PolicyArgs a{p->old_logp, p->ref_logp, p->advantage, 1.0 - p->clip_low, 1.0 + p->clip_high, p->kl_coef, p->scale};
    float* lp = logp ? logp : w.logp;
    launch_logp(x, of, lp, w.lse, s);
    policy_coef_kernel<<<(x->rows + kThreads - 1) / kThreads, kThreads, 0, s>>>(a, of, x->rows, lp, w.coef, w.part);
    if (dlogits) launch_grad(x, of, w.lse, w.coef, dlogits, dlogits_stride, s);
  }
  sum_kernel<<<1, kThreads, 0, s>>>(w.part, x->rows, loss);
  return launched();
}

zb_status zb_preference_loss(const zb_logits* x, const zb_preference* p, float* loss, float* logp, float* rewards, void* dlogits,
                             int64_t dlogits_stride, void* workspace, size_t workspace_size, void* hip_stream) {
  if (!valid_logits(x) || !p || !loss || !valid_dlogits(x, dlogits, &dlogits_stride)) return ZB_EINVAL;
  if (p->pairs < 0 || p->pairs > kMaxRows || !isfinite(p->beta) || !isfinite(p->scale) || !(p->label_smoothing >= 0 && p->label_smoothing <= 1))
    return ZB_EINVAL;
  if ((p->pairs && !p->offsets) || (x->rows && p->pairs && !p->ref_logp)) return ZB_EINVAL;
  if (!workspace || misaligned(workspace, 8) || workspace_size < workspace_bytes(x->rows, p->pairs)) return ZB_EINVAL;
  if (misaligned(loss, 4) || misaligned(logp, 4) || misaligned(rewards, 4) || misaligned(p->offsets, 4) || misaligned(p->ref_logp, 4) ||
      misaligned(p->weight, 4))
    return ZB_EINVAL;
  const hipStream_t s = (hipStream_t)hip_stream;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  const Workspace w = carve(workspace, x->rows, p->pairs);
  float* lp = logp ? logp : w.logp;
  const Rows of{x->targets, p->weight, p->pairs ? p->offsets : nullptr, p->pairs ? 2 * p->pairs : -1, x->vocab};
  if (x->rows) {
    fill_zero_kernel<<<(x->rows + kThreads - 1) / kThreads, kThreads, 0, s>>>(w.coef, x->rows);
    launch_logp(x, of, lp, w.lse, s);
  }
  if (p->pairs) {
    const PairArgs a{p->ref_logp, p->beta, p->label_smoothing, p->scale};
    pair_kernel<<<p->pairs, kThreads, 0, s>>>(a, of, x->rows, lp, rewards, w.coef, w.part);
  }
  if (x->rows && dlogits) launch_grad(x, of, w.lse, w.coef, dlogits, dlogits_stride, s);
  sum_kernel<<<1, kThreads, 0, s>>>(w.part, p->pairs, loss);
  return launched();
}

}  // extern "C"
