// Losses on the log-probabilities of given tokens, and the gradient of the logits they come from: with
//   lse_r = log sum_j exp(z_rj),  logp_r = z_r,target(r) - lse_r,  c_r = d(loss) / d(logp_r)
// every loss here has  d(loss) / d(z_rj) = c_r ([j = target(r)] - exp(z_rj - lse_r)).
// The target's entry is c_r (1 - p), p its probability: 1 - p comes from the other tokens' exponentials, which are added up without the target's, and so
// does log p where the target has nearly all of the row.
// A row counts if its target lies in [0, vocab), its weight is not zero and, where there are sequences, one of them holds it;
// the logits of the others are not read.
#include <math.h>

#include "token_loss.h"

namespace zb {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504f;

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

// A row as it lies in memory: `head` elements up to the first address that is a multiple of 16, `full` 16-byte vectors, `tail`
// elements.  The elements before and behind the vectors are at most VE - 1 each and belong to the first 2 VE lanes.
template <typename T> struct Span {
  static constexpr int VE = 16 / sizeof(T);
  int head, full, tail;
  __device__ __forceinline__ Span(const T* row, int vocab) {
    head = (int)(((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T));
    if (head > vocab) head = vocab;
    full = (vocab - head) / VE;
    tail = vocab - head - full * VE;
  }
  // index of the element that this lane has beside the vectors, -1 for none
  __device__ __forceinline__ int edge(int lane) const {
    if (lane < VE) return lane < head ? lane : -1;
    return lane - VE < tail ? head + full * VE + lane - VE : -1;  // (tail < VE: lanes from 2 VE on have none)
  }
  // the vector that element j is in, -1 if it lies beside them
  __device__ __forceinline__ int vector_of(int j) const { return j >= head && j < head + full * VE ? (j - head) / VE : -1; }
};
template <typename T> __device__ __forceinline__ void unpack(const uint4& r, float (&x)[16 / sizeof(T)]);
template <> __device__ __forceinline__ void unpack<float>(const uint4& r, float (&x)[4]) {
  x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
}
template <> __device__ __forceinline__ void unpack<bf16_t>(const uint4& r, float (&x)[8]) {
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
template <typename T> __device__ __forceinline__ uint4 pack(const float (&x)[16 / sizeof(T)]);
template <> __device__ __forceinline__ uint4 pack<float>(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <> __device__ __forceinline__ uint4 pack<bf16_t>(const float (&x)[8]) {
  union { bf16x8 v; uint4 u; } c;
#pragma unroll
  for (int i = 0; i < 8; ++i) c.v[i] = (bf16_t)x[i];
  return c.u;
}
template <typename T> __device__ __forceinline__ uint4 empty_pack();  // all -infinity
template <> __device__ __forceinline__ uint4 empty_pack<float>() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
template <> __device__ __forceinline__ uint4 empty_pack<bf16_t>() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }

// A vector whose element e is -infinity.
template <typename T> __device__ __forceinline__ uint4 without(const uint4& r, int e);
template <> __device__ __forceinline__ uint4 without<float>(const uint4& r, int e) {
  const unsigned none = 0xFF800000u;
  return make_uint4(e == 0 ? none : r.x, e == 1 ? none : r.y, e == 2 ? none : r.z, e == 3 ? none : r.w);
}
template <> __device__ __forceinline__ uint4 without<bf16_t>(const uint4& r, int e) {
  unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i == e >> 1) w[i] = e & 1 ? (w[i] & 0xFFFFu) | 0xFF800000u : (w[i] & 0xFFFF0000u) | 0xFF80u;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Keeps a row as it was loaded: without it the 32-bit forms of one pass over it are kept for the next, in twice the registers.
template <int NV> __device__ __forceinline__ void as_loaded(uint4 (&r)[NV]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(r[i].x), "+v"(r[i].y), "+v"(r[i].z), "+v"(r[i].w));
}

// exp(x - top), without the bias of a log2(e) of 24 bits: log-probabilities are added over sequences, where errors of one sign would add up
// while the values cancel.  (What is left is the exponent's rounding, 2^-24 (x - top) of the result in either direction.)
__device__ __forceinline__ float exp_of(float x, float top) {
  const float d = x - top;
  return __builtin_amdgcn_exp2f(fmaf(d, kLog2e, d * 1.925963033e-8f));
}
// The same for an entry of a gradient of type T: stored in bf16, the bias (a share of 2e-8 (x - top)) is far below half a step, 2^-8.
template <typename T> __device__ __forceinline__ float exp_in(float x, float top) { return exp_of(x, top); }
template <> __device__ __forceinline__ float exp_in<bf16_t>(float x, float top) { return __builtin_amdgcn_exp2f((x - top) * kLog2e); }
// Sum of a vector's exponentials.  Vectors are added up in 64 bits: one large term would round off a part of each small one that follows it.
template <int VE> __device__ __forceinline__ double exp_sum(const float (&x)[VE], float top) {
  float t[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) t[e] = exp_of(x[e], top);
#pragma unroll
  for (int w = VE / 2; w > 0; w /= 2)
#pragma unroll
    for (int e = 0; e < w; ++e) t[e] += t[e + w];
  return (double)t[0];
}
// log(s) of 1 <= s < 2^19 (or NaN): the exponent apart, the rest from 2 atanh(z), z = (f - 1) / (f + 1), |z| < 0.172, to 1e-12
__device__ __forceinline__ double log_of(double s) {
  const unsigned high = (unsigned)__double2hiint(s);
  int e = (int)(high >> 20) - 1023;
  double f = __hiloint2double((int)((high & 0x000FFFFFu) | 0x3FF00000u), __double2loint(s));
  if (f > 1.41421356) { f *= 0.5; ++e; }
  const double z = (f - 1.0) / (f + 1.0), q = z * z;
  double t = 1.0 / 15.0;
  t = fma(t, q, 1.0 / 13.0); t = fma(t, q, 1.0 / 11.0); t = fma(t, q, 1.0 / 9.0); t = fma(t, q, 1.0 / 7.0); t = fma(t, q, 1.0 / 5.0);
  t = fma(t, q, 1.0 / 3.0);
  return s == s ? fma((double)e, 0.6931471805599453, 2.0 * fma(z * q, t, z)) : s;
}

// what the lanes of a workgroup of N waves hold, reduced in a fixed order; `red` is read after the barrier only
template <int N> __device__ __forceinline__ float block_max(float v, float* red) {
  v = wave_max(v);
  if (N == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < N; ++w) v = fmaxf(v, red[w]);
  return v;
}
template <int N> __device__ __forceinline__ double block_sum(double v, double* red) {
  v = wave_sum(v);
  if (N == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < N; ++w) v += red[w];
  return v;
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
// NT: the caches are told that the line is not needed again
template <bool NT> __device__ __forceinline__ uint4 get16(const uint4* at) {
  if (!NT) return *at;
  const u32x4 t = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
  return make_uint4(t.x, t.y, t.z, t.w);
}
template <bool NT> __device__ __forceinline__ void put16(void* at, const uint4& v) {
  const u32x4 t = {v.x, v.y, v.z, v.w};
  if (NT) __builtin_nontemporal_store(t, reinterpret_cast<u32x4*>(at));
  else *reinterpret_cast<u32x4*>(at) = t;
}

// zeros in a row's gradient, by THREADS lanes
template <typename T, bool NT> __device__ __forceinline__ void clear_row(T* d, int vocab, int threads) {
  const Span<T> sp(d, vocab);
  const int lane = threadIdx.x;
  uint4* v = reinterpret_cast<uint4*>(d + sp.head);
  for (int k = lane; k < sp.full; k += threads) put16<NT>(v + k, make_uint4(0, 0, 0, 0));
  const int e = sp.edge(lane);
  if (e >= 0) d[e] = from_f32<T>(0.f);
}

struct PolicyArgs {
  const float *old_logp, *ref_logp, *advantage;
  double lo, hi, log_lo, log_hi, kl, scale, grad_scale;  // borders of the ratio and of its logarithm
};
// exp(d), off by 1e-11 of it: 2^k e^r with |r| <= log(2) / 2 and nine terms of the series, a chain that one lane runs in a few hundred
// cycles.  (Advantages have both signs: the sum of the rows' losses is far smaller than the losses, so 32 bits are not enough here.)
__device__ __forceinline__ double exp_near(double d) {
  if (!(fabs(d) < 700.0)) return d > 0.0 ? (double)INFINITY : d < 0.0 ? 0.0 : d;
  const double k = rint(d * 1.4426950408889634);
  const double r = fma(k, -0.6931471805599453, d);
  double t = 1.0 / 362880.0;
  t = fma(t, r, 1.0 / 40320.0); t = fma(t, r, 1.0 / 5040.0); t = fma(t, r, 1.0 / 720.0); t = fma(t, r, 1.0 / 120.0);
  t = fma(t, r, 1.0 / 24.0); t = fma(t, r, 1.0 / 6.0); t = fma(t, r, 0.5); t = fma(t, r, 1.0); t = fma(t, r, 1.0);
  return ldexp(t, (int)k);
}
// exp(d) - d - 1, and exp(d) - 1 in *up; the digits that the subtractions would take near 0 come from the series
__device__ __forceinline__ double exp_above_line(double d, double* up) {
  if (!(fabs(d) <= 0.5)) {
    const double e = exp_near(d);
    *up = e - 1.0;
    return e < INFINITY ? e - d - 1.0 : e;
  }
  double t = 1.0 / 39916800.0;  // 1 / 11!
  t = fma(t, d, 1.0 / 3628800.0); t = fma(t, d, 1.0 / 362880.0); t = fma(t, d, 1.0 / 40320.0); t = fma(t, d, 1.0 / 5040.0);
  t = fma(t, d, 1.0 / 720.0); t = fma(t, d, 1.0 / 120.0); t = fma(t, d, 1.0 / 24.0); t = fma(t, d, 1.0 / 6.0); t = fma(t, d, 0.5);
  const double k = d * d * t;
  *up = k + d;
  return k;
}
// What a row's loss reads.
struct PolicyTerms {
  float advantage, old_logp, ref_logp, weight;
};
__device__ __forceinline__ PolicyTerms terms_of(const PolicyArgs& a, const Rows& of, int row) {
  return {a.advantage[row], a.old_logp[row], a.kl != 0.0 ? a.ref_logp[row] : 0.f, of.weight ? of.weight[row] : 1.f};
}
// Loss of a row and its derivative by the row's log-probability; what is compared with a border is the ratio's logarithm.
__device__ __forceinline__ double policy_row(const PolicyArgs& a, const PolicyTerms& in, double logp, double* slope) {
  const double adv = in.advantage, x = logp - (double)in.old_logp, rho = exp_near(x), w = in.weight;
  const bool above = x > a.log_hi, below = x < a.log_lo;
  const double held = above ? a.hi : below ? a.lo : rho;
  // (an advantage of 0 asks for nothing, however far the ratio is)
  double loss = adv == 0 ? 0.0 : -fmin(rho * adv, held * adv);
  double g = adv == 0 || (adv > 0 && above) || (adv < 0 && below) ? 0.0 : -adv * rho;
  if (a.kl != 0.0) {
    double up;
    loss += a.kl * exp_above_line((double)in.ref_logp - logp, &up);
    g -= a.kl * up;
  }
  *slope = a.grad_scale * w * g;
  return a.scale * w * loss;
}

// Sum of n values by the THREADS lanes of a workgroup, in an order that only n decides; lane 0 has it.
template <int THREADS, class F> __device__ __forceinline__ double sum_of(int n, F&& value) {
  __shared__ double red[THREADS / 64];
  double acc = 0.0;
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * THREADS) {  // four loads on their way at a time
    double x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = i0 + k * THREADS < n ? value(i0 + k * THREADS) : 0.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) acc += x[k];
  }
  acc = wave_sum(acc);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = acc;
  __syncthreads();
  acc = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) acc += red[w];
  return acc;
}
__global__ __launch_bounds__(1024) void sum_kernel(const double* __restrict__ part, int n, float* __restrict__ out) {
  const double s = sum_of<1024>(n, [&](int i) { return part[i]; });
  if (threadIdx.x == 0) *out = (float)s;
}
// A launch of up to kSumInPlace workgroups adds their partial losses itself: the workgroup that is through last does, reading past the
// caches of the XCDs what the others wrote past them.  `done` counts modulo the workgroups, so it is 0 again for the next call.
constexpr int kSumInPlace = 256;
struct Total {
  float* loss;     // null: a kernel of its own adds the partial losses
  unsigned* done;
};
// By one lane, once in a workgroup; *last tells whether all the others have been here.  It comes before a row's gradient is written: the count
// waits until what its XCD has written is past the caches.
__device__ __forceinline__ void announce(const Total& t, double* part, double mine, bool* last) {
  *last = false;
  if (!t.loss) {
    part[blockIdx.x] = mine;
    return;
  }
  __hip_atomic_store(part + blockIdx.x, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  *last = __builtin_amdgcn_atomic_inc32(t.done, gridDim.x - 1, __ATOMIC_ACQ_REL, "agent") == gridDim.x - 1;
}
template <int THREADS> __device__ __forceinline__ void add_up(const Total& t, const double* part, const bool* last) {  // by the whole workgroup
  if (!t.loss) return;
  __syncthreads();
  if (!*last) return;
  const double s = sum_of<THREADS>((int)gridDim.x, [&](int i) { return __hip_atomic_load(part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
  if (threadIdx.x == 0) *t.loss = (float)s;
}

// 1 - p of a target with the exponential `hit` beside `others`, inv = 1 / (hit + others); either form where it rounds less
__device__ __forceinline__ float missed(float hit, float others, float inv) { return hit < others ? 1.f - hit * inv : others * inv; }

struct RowOut {  // what the row kernels leave of a row; null: not wanted
  float *logp, *lse;
  float *top, *inv;  // p_j = exp(z_j - top) * inv
  float* miss;       // 1 - p of the target
  double *logp64;    // logp before its rounding
  double* part;      // with a policy: its loss
  Total total;
};
__device__ __forceinline__ void put_row(const RowOut& o, int row, double logp, double lse, float top, float s, float hit, float others) {
  if (o.logp) o.logp[row] = (float)logp;
  if (o.lse) o.lse[row] = (float)lse;
  if (o.top) {
    const float inv = 1.0f / s;
    o.top[row] = top; o.inv[row] = inv; o.miss[row] = missed(hit, others, inv);
  }
  if (o.logp64) o.logp64[row] = logp;
}
__device__ __forceinline__ void put_no_row(const RowOut& o, int row) {
  if (o.logp) o.logp[row] = 0.f;
  if (o.lse) o.lse[row] = 0.f;
  if (o.top) { o.top[row] = 0.f; o.inv[row] = 0.f; o.miss[row] = 0.f; }
  if (o.logp64) o.logp64[row] = 0.0;
}

// The policy loss, one workgroup per row, the row in registers (NV vectors a lane): read once for the maximum, the sum and the
// gradient, which follows from the row's own log-probability.  Bound by HBM: 4096 rows of 50432 bf16, 800 of them without weight, 141 us =
// 5.3 TB/s of what has to move (a large copy moves 4.9); 1023 rows of 32003 fp32 51 us.  While one lane works out the row's
// coefficient nothing of that row moves, so a CU holds two rows of 100 KB (64 registers a lane): one of them at a time takes 209 us.
template <typename T, int THREADS, int NV, bool NT>
__device__ __forceinline__ void policy_in_registers(const T* logits, long stride, Rows of, RowOut out, PolicyArgs pol, T* dlogits, long dstride,
                                                    bool* last) {
  constexpr int VE = Span<T>::VE, N = THREADS / 64;
  __shared__ double red_s[N];
  __shared__ float red_m[N], coef_of;
  __shared__ PolicyTerms in;
  const int row = blockIdx.x, lane = threadIdx.x;
  T* d = dlogits + (long)row * dstride;
  if (!of.counts(row)) {
    if (lane == 0) {
      put_no_row(out, row);
      announce(out.total, out.part, 0.0, last);
    }
    if (dlogits) clear_row<T, NT>(d, of.vocab, THREADS);
    return;
  }
  const T* z = logits + (long)row * stride;
  const Span<T> sp(z, of.vocab);
  const uint4* v = reinterpret_cast<const uint4*>(z + sp.head);
  uint4 r[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int k = i * THREADS + lane;
    r[i] = k < sp.full ? get16<NT>(v + k) : empty_pack<T>();
  }
  const int edge = sp.edge(lane), target = of.targets[row], vt = sp.vector_of(target);
  const float xe = edge >= 0 && edge != target ? to_f32(z[edge]) : -INFINITY, zy = to_f32(z[target]);
  if (lane == 0) in = terms_of(pol, of, row);  // (on their way with the row; kept apart from it, whose lanes have no registers to spare)
  const bool owner = vt < 0 ? edge == target : vt % THREADS == lane;  // the lane whose entry the target is; it keeps it apart from the others
  if (owner) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i * THREADS + lane == vt) r[i] = without<T>(r[i], (target - sp.head) % VE);
  }
  float m = xe;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[VE];
    unpack<T>(r[i], x);
#pragma unroll
    for (int e = 0; e < VE; ++e) m = fmaxf(m, x[e]);
  }
  m = fmaxf(block_max<N>(m, red_m), zy);
  as_loaded(r);
  double acc = (double)exp_of(xe, m);  // (a NaN, an infinity and a row of nothing but -infinity make the sum NaN)
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[VE];
    unpack<T>(r[i], x);
    acc += exp_sum<VE>(x, m);
  }
  const double rest = block_sum<N>(acc, red_s), s64 = rest + (double)exp_of(zy, m);
  const float s = (float)s64, others = (float)rest;
  double loss = 0.0;
  if (lane == 0) {
    const double l = log_of(s64), lp = ((double)zy - (double)m) - l;
    double slope;
    loss = policy_row(pol, in, lp, &slope);
    put_row(out, row, lp, (double)m + l, m, s, exp_of(zy, m), others);
    coef_of = (float)slope;
  }
  if (dlogits) __syncthreads();
  if (lane == 0) announce(out.total, out.part, loss, last);
  if (!dlogits) return;
  const float coef = coef_of, inv = 1.f / s, neg = -coef * inv;
  if (coef == 0.f) {
    clear_row<T, NT>(d, of.vocab, THREADS);
    return;
  }
  const bool same = (((uintptr_t)d ^ (uintptr_t)z) & 15) == 0;
  as_loaded(r);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int k = i * THREADS + lane;
    if (k >= sp.full) break;
    float x[VE];
    unpack<T>(r[i], x);
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = neg * exp_in<T>(x[e], m);
    T* at = d + sp.head + k * VE;
    if (same) {
      put16<NT>(at, pack<T>(x));
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) at[e] = from_f32<T>(x[e]);
    }
  }
  if (edge >= 0) d[edge] = from_f32<T>(neg * exp_in<T>(xe, m));
  if (owner) d[target] = from_f32<T>(coef * missed(exp_of(zy, m), others, inv));  // (the lane that wrote the vector around it)
}
template <typename T, int THREADS, int NV, int WAVES, bool NT>
__global__ __launch_bounds__(THREADS, WAVES) void policy_row_kernel(const T* logits, long stride, Rows of, RowOut out, PolicyArgs pol, T* dlogits,
                                                                    long dstride) {
  __shared__ bool last;
  policy_in_registers<T, THREADS, NV, NT>(logits, stride, of, out, pol, dlogits, dstride, &last);
  add_up<THREADS>(out.total, out.part, &last);
}

// lse and log-probability, one workgroup per row: maximum and sum in one pass, U vectors of a lane at a time, the sum scaled anew when the lane's
// maximum grows.  Bound by HBM: 4096 rows of 50432 bf16 65 us = 6.4 TB/s (with the row in registers 82).  With POLICY, for
// rows that registers do not hold, the policy loss: the row is read again for the gradient, so its first read keeps its place in the caches whatever
// NT (1536 rows of 131072 bf16 177 us, with the first read past the caches 214).
template <typename T, int THREADS, int U, bool POLICY, bool NT>
__device__ __forceinline__ void row_in_passes(const T* logits, long stride, Rows of, RowOut out, PolicyArgs pol, T* dlogits, long dstride, bool* last) {
  constexpr int VE = Span<T>::VE, N = THREADS / 64;
  __shared__ double red_s[N];
  __shared__ float red_m[N], coef_of;
  const int row = blockIdx.x, lane = threadIdx.x;
  T* d = dlogits + (long)row * dstride;
  if (!of.counts(row)) {
    if (lane == 0) {
      put_no_row(out, row);
      if (POLICY) announce(out.total, out.part, 0.0, last);
    }
    if (POLICY && dlogits) clear_row<T, NT>(d, of.vocab, THREADS);
    return;
  }
  const T* z = logits + (long)row * stride;
  const Span<T> sp(z, of.vocab);
  const uint4* v = reinterpret_cast<const uint4*>(z + sp.head);
  const int edge = sp.edge(lane), target = of.targets[row], vt = sp.vector_of(target);
  const bool owner = vt < 0 ? edge == target : vt % THREADS == lane;  // the lane whose entry the target is; it keeps it apart from the others
  const int own_vector = owner ? vt : -1;
  const float xe = edge >= 0 && edge != target ? to_f32(z[edge]) : -INFINITY, zy = to_f32(z[target]);
  float mine = xe;
  double part = edge >= 0 ? 1.0 : 0.0;  // the lane's sum counts exp(x - mine)
  if (xe != xe) part = (double)xe;
  for (int k0 = lane; k0 < sp.full; k0 += U * THREADS) {
    uint4 r[U];
#pragma unroll
    for (int i = 0; i < U; ++i) r[i] = k0 + i * THREADS < sp.full ? get16<NT && !POLICY>(v + k0 + i * THREADS) : empty_pack<T>();
    if (own_vector >= k0 && own_vector < k0 + U * THREADS) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (k0 + i * THREADS == own_vector) r[i] = without<T>(r[i], (target - sp.head) % VE);
    }
    float top = mine;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float x[VE];
      unpack<T>(r[i], x);
#pragma unroll
      for (int e = 0; e < VE; ++e) top = fmaxf(top, x[e]);
    }
    if (top > mine) {
      part = mine == -INFINITY ? (part != part ? part : 0.0) : part * (double)exp_of(mine, top);
      mine = top;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float x[VE];
      unpack<T>(r[i], x);
      if (mine > -INFINITY) {
        part += exp_sum<VE>(x, mine);
      } else {  // nothing but -infinity so far, or a NaN
#pragma unroll
        for (int e = 0; e < VE; ++e) part += x[e] == x[e] ? 0.0 : (double)x[e];
      }
    }
  }
  const float m = fmaxf(block_max<N>(mine, red_m), zy);
  // lanes without a finite logit add nothing, unless they saw a NaN; a row without one is undefined
  const double own = mine == -INFINITY && m > -INFINITY ? (part != part ? part : 0.0) : part * (double)exp_of(mine, m);
  const double rest = block_sum<N>(own, red_s), s64 = rest + (double)exp_of(zy, m);
  const float s = (float)s64, others = (float)rest;
  double loss = 0.0;
  if (lane == 0) {
    const double l = log_of(s64), lp = ((double)zy - (double)m) - l;
    if (POLICY) {
      double slope;
      loss = policy_row(pol, terms_of(pol, of, row), lp, &slope);
      coef_of = (float)slope;
    }
    put_row(out, row, lp, (double)m + l, m, s, exp_of(zy, m), others);
  }
  if (!POLICY) return;
  if (dlogits) __syncthreads();
  if (lane == 0) announce(out.total, out.part, loss, last);
  if (!dlogits) return;
  const float coef = coef_of, inv = 1.f / s, neg = -coef * inv;
  if (coef == 0.f) {
    clear_row<T, NT>(d, of.vocab, THREADS);
    return;
  }
  const bool same = (((uintptr_t)d ^ (uintptr_t)z) & 15) == 0;
  for (int k = lane; k < sp.full; k += THREADS) {  // (a lane reads its entries before it writes them: d may be z)
    float x[VE];
    unpack<T>(get16<NT>(v + k), x);
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = neg * exp_in<T>(x[e], m);
    T* at = d + sp.head + k * VE;
    if (same) {
      put16<NT>(at, pack<T>(x));
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) at[e] = from_f32<T>(x[e]);
    }
  }
  if (edge >= 0) d[edge] = from_f32<T>(neg * exp_in<T>(xe, m));
  if (owner) d[target] = from_f32<T>(coef * missed(exp_of(zy, m), others, inv));  // (the lane that wrote the vector around it)
}
template <typename T, int THREADS, int U, bool POLICY, bool NT>
__global__ __launch_bounds__(THREADS) void row_kernel(const T* logits, long stride, Rows of, RowOut out, PolicyArgs pol, T* dlogits, long dstride) {
  __shared__ bool last;
  row_in_passes<T, THREADS, U, POLICY, NT>(logits, stride, of, out, pol, dlogits, dstride, &last);
  if (POLICY) add_up<THREADS>(out.total, out.part, &last);
}

// coef ([j = target] - exp(z_j - top) inv), inv null: 1, with the target's 1 - p from `misses` where there are any, by workgroups of
// kThreads * kGradVectors vectors of a row.  Bound by HBM: the rows of six pairs of about 500 tokens x 50432 bf16, which have just been read for
// their log-probabilities, 144 us = 6.8 TB/s with the rows without weight, which are not read.  us of log-probabilities and gradient with 2 /
// 4 / 8 vectors a lane: 228 / 232 / 256; from the last row to the first, towards what the caches may still hold: 232.
constexpr int kGradVectors = 2;
template <typename T, bool NT>
__global__ __launch_bounds__(kThreads) void grad_kernel(const T* logits, long stride, Rows of, const float* __restrict__ coefs,
                                                        const float* __restrict__ tops, const float* __restrict__ invs,
                                                        const float* __restrict__ misses, T* dlogits, long dstride, int parts, int row0) {
  constexpr int VE = Span<T>::VE;
  const int at_row = blockIdx.x / parts, part = blockIdx.x - at_row * parts, row = row0 + at_row, lane = threadIdx.x;
  const float coef = of.counts(row) ? coefs[row] : 0.f;
  const T* z = logits + (long)row * stride;
  T* d = dlogits + (long)row * dstride;
  const bool same = (((uintptr_t)d ^ (uintptr_t)z) & 15) == 0;
  const Span<T> sp(z, of.vocab);
  const int k0 = part * kThreads * kGradVectors + lane, edge = part == 0 ? sp.edge(lane) : -1;
  if (coef == 0.f) {
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i) {
      const int k = k0 + i * kThreads;
      if (k >= sp.full) break;
      T* at = d + sp.head + k * VE;
      if (same) {
        put16<NT>(at, make_uint4(0, 0, 0, 0));
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) at[e] = from_f32<T>(0.f);
      }
    }
    if (edge >= 0) d[edge] = from_f32<T>(0.f);
    return;
  }
  const float top = tops[row], inv = invs ? invs[row] : 1.f, miss = misses ? misses[row] : 0.f, neg = -coef * inv;
  const int target = of.targets[row];
  const uint4* v = reinterpret_cast<const uint4*>(z + sp.head);
  uint4 r[kGradVectors];
#pragma unroll
  for (int i = 0; i < kGradVectors; ++i) {
    const int k = k0 + i * kThreads;
    if (k < sp.full) r[i] = get16<NT>(v + k);
  }
#pragma unroll
  for (int i = 0; i < kGradVectors; ++i) {
    const int k = k0 + i * kThreads, j = sp.head + k * VE;
    if (k >= sp.full) break;
    float x[VE];
    unpack<T>(r[i], x);
    const bool hot = target >= j && target < j + VE;
    float y = 0.f;
    if (hot) {
#pragma unroll
      for (int e = 0; e < VE; ++e) if (j + e == target) y = x[e];
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = neg * exp_in<T>(x[e], top);
    T* at = d + j;
    if (same) {
      put16<NT>(at, pack<T>(x));
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) at[e] = from_f32<T>(x[e]);
    }
    if (hot) d[target] = from_f32<T>(coef * (misses ? miss : 1.f - exp_of(y, top) * inv));
  }
  if (edge >= 0) {
    const float p = exp_of(to_f32(z[edge]), top) * inv;
    d[edge] = from_f32<T>(edge == target ? coef * (misses ? miss : 1.f - p) : -coef * p);
  }
}

struct PairArgs {
  const float* ref_logp;
  double beta, smoothing, scale, grad_scale;
};
__device__ __forceinline__ void sequence_rows(const int* offsets, int q, int rows, int* a, int* b) {
  const int x = offsets[q], y = offsets[q + 1];
  *a = x < 0 ? 0 : x > rows ? rows : x;
  *b = y < *a ? *a : y > rows ? rows : y;
}

// One workgroup per pair: both sequences' sums of w (logp - ref), the pair's loss, and the coefficient of every row.  A chain of loads, sums
// and one lane's exponential: 5.9 us for two pairs of 50 tokens, 9.0 for six of 500.
constexpr int kPairThreads = 1024;
__global__ __launch_bounds__(kPairThreads) void pair_kernel(PairArgs a, Rows of, int rows, const double* __restrict__ logp, float* __restrict__ rewards,
                                                            float* __restrict__ coef, double* part, Total total) {
  __shared__ double red[2][kPairThreads / 64], slope_of;
  __shared__ bool last;
  int lo[2], hi[2];
  for (int q = 0; q < 2; ++q) {
    sequence_rows(of.offsets, 2 * blockIdx.x + q, rows, &lo[q], &hi[q]);
    double acc = 0.0;
    for (int r = lo[q] + threadIdx.x; r < hi[q]; r += kPairThreads) {
      const double gap = logp[r] - (double)a.ref_logp[r];  // (whatever a row that does not count holds there)
      if (of.counts(r)) acc += of.weight_of(r) * gap;
    }
    acc = wave_sum(acc);
    if ((threadIdx.x & 63) == 0) red[q][threadIdx.x >> 6] = acc;
  }
  __syncthreads();
  double loss = 0.0;
  if (threadIdx.x == 0) {
    double s[2];
    for (int q = 0; q < 2; ++q) {
      s[q] = red[q][0];
      for (int w = 1; w < kPairThreads / 64; ++w) s[q] += red[q][w];
      if (rewards) rewards[2 * blockIdx.x + q] = (float)(a.beta * s[q]);
    }
    const double x = a.beta * (s[0] - s[1]), e = exp(-fabs(x)), l = log1p(e);  // -log sigma(x) = max(-x, 0) + l
    // (x may be infinite: a share of 0 takes nothing of an infinite term)
    const double kept = 1.0 - a.smoothing;
    loss = a.scale * ((kept != 0.0 ? kept * (fmax(-x, 0.0) + l) : 0.0) + (a.smoothing != 0.0 ? a.smoothing * (fmax(x, 0.0) + l) : 0.0));
    const double above = x >= 0 ? 1.0 / (1.0 + e) : e / (1.0 + e);  // sigma(x)
    const double below = x >= 0 ? e / (1.0 + e) : 1.0 / (1.0 + e);  // sigma(-x)
    slope_of = a.grad_scale * a.beta * (a.smoothing * above - (1.0 - a.smoothing) * below);
  }
  __syncthreads();
  if (threadIdx.x == 0) announce(total, part, loss, &last);
  const double slope = slope_of;
  for (int q = 0; q < 2; ++q)
    for (int r = lo[q] + threadIdx.x; r < hi[q]; r += kPairThreads) coef[r] = (float)((q ? -slope : slope) * of.weight_of(r));
  add_up<kPairThreads>(total, part, &last);
}

bool valid_logits(const zb_logits* x) {
  if (!x || x->rows < 0 || x->rows > kLossMaxRows || x->vocab < 1 || x->vocab > kEmbeddingMaxVocab || x->row_stride < x->vocab) return false;
  if (x->row_stride > (int64_t)1 << 32 || (x->dtype != ZB_FP32 && x->dtype != ZB_BF16)) return false;
  if (x->rows == 0) return true;
  const uintptr_t es = x->dtype == ZB_BF16 ? 2 : 4;
  return x->logits && x->targets && !((uintptr_t)x->logits & (es - 1)) && !((uintptr_t)x->targets & 3);
}
bool valid_dlogits(const zb_logits* x, const void* d, int64_t* stride) {
  if (*stride == 0) *stride = x->row_stride;
  if (*stride < x->vocab || *stride > (int64_t)1 << 32 || (d && d == x->logits && *stride != x->row_stride)) return false;
  return !((uintptr_t)d & (x->dtype == ZB_BF16 ? 1 : 3));
}
bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

struct Workspace {  // a counter; per row a partial loss, the log-probability, what makes probabilities of logits, the target's 1 - p, the coefficient
  unsigned* done;
  double *part, *logp;
  float *top, *inv, *miss, *coef;
};
Workspace carve(void* base, int rows, int pairs) {
  Workspace w;
  w.done = (unsigned*)base;
  w.part = (double*)((char*)base + ZB_WORKSPACE_KEPT_BYTES);
  w.logp = w.part + (rows > pairs ? rows : pairs);
  w.top = (float*)(w.logp + rows);
  w.inv = w.top + rows;
  w.miss = w.inv + rows;
  w.coef = w.miss + rows;
  return w;
}

// Lines that no cache would hold until they are wanted again: logits of over 64 MB, a quarter of the last cache (the gradient and
// what comes next want their place in it too); where the logits are read again next, of over all of it.  us with / without: log-probabilities of
// 4096 x 50432 bf16 65 / 74, policy loss of the same 142 / 150; 768 rows (77 MB) 16.6 / 16.6 and 37 / 45, 512 rows (52 MB) 11.9 / 12.1 and 24 / 26, 64
// rows 7.4 / 7.3 and 12.6 / 12.7: small logits lose nothing by staying.
bool past_caches(const zb_logits* x, bool again = false) {
  return (size_t)x->rows * x->vocab * (x->dtype == ZB_BF16 ? 2 : 4) > (size_t)(again ? 256 : 64) << 20;
}

#define ZB_NT(call)                                                          \
  do {                                                                       \
    if (past_caches(x)) { constexpr bool NT = true; call; }                  \
    else { constexpr bool NT = false; call; }                                \
  } while (0)

template <typename T> hipError_t launch_logp(const zb_logits* x, const Rows& of, const RowOut& out, bool nt, hipStream_t s) {
  const int vectors = x->vocab / Span<T>::VE;
#define ZB_LOGP(THREADS, U, NT) \
  row_kernel<T, THREADS, U, false, NT><<<x->rows, THREADS, 0, s>>>((const T*)x->logits, x->row_stride, of, out, PolicyArgs{}, (T*)nullptr, 0)
#define ZB_ROWS(THREADS, U)                                    \
  do {                                                         \
    if (nt) ZB_LOGP(THREADS, U, true);                         \
    else ZB_LOGP(THREADS, U, false);                           \
  } while (0)
  // Lanes of a workgroup by the length of a row.  us of 8192 rows of 2048 / 4096 / 8192 / 16384 bf16 and 4096 of 32000 / 50432: 64 lanes 9.1 /
  // 14.1, 256 lanes 19.4 / 19.1 / 22.1 / 46.9 / 50.7 / 68.5, 512 - / - / 35.1 / 49.1 / 47.4 / 65.1, 1024 55.2 / 73.9 of the last two.  Where fewer rows
  // leave CUs idle, 512 / 1024 lanes: 100 rows of 32000 bf16 6.0 / 6.1, 50432 fp32 9.1 / 8.3, 262144 fp32 30.5 / 25.8, 511 rows of the same 9.8 / 10.1,
  // 18.0 / 18.2, 91.5 / 93.2.
  if (vectors <= 512) ZB_ROWS(64, 4);
  else if (vectors <= 2048) ZB_ROWS(256, 4);
  else if (x->rows >= 512) ZB_ROWS(512, 4);
  else ZB_ROWS(1024, 2);
#undef ZB_ROWS
#undef ZB_LOGP
  return hipGetLastError();
}
hipError_t launch_logp(const zb_logits* x, const Rows& of, const RowOut& out, bool nt, hipStream_t s) {
  return x->dtype == ZB_BF16 ? launch_logp<bf16_t>(x, of, out, nt, s) : launch_logp<float>(x, of, out, nt, s);
}

template <typename T>
hipError_t launch_policy(const zb_logits* x, const Rows& of, const RowOut& out, const PolicyArgs& pol, void* dlogits, int64_t dstride, hipStream_t s) {
  const int vectors = x->vocab / Span<T>::VE;  // at most: a row's start may leave one fewer
  // Shapes that hold a row in registers and leave room for a second one on the CU, WAVES per SIMD keep the registers to that.  Up to 512 x 8 vectors the
  // fewest lanes do best; from there on twice the lanes as long as 64 registers each hold a row (1024 x 7), and then 512 again with up to 128.
  // us of 4096 rows (fewer from 7168 vectors on), bf16 / fp32, the shape taken first:
  //   4000 vectors   512 x 8  101 / 100   1024 x 7 109 / 98       7168 vectors  1024 x 7  154 / 153   512 x 16 169 / 154
  //   4096           512 x 8   99 / 99    1024 x 7 111 / 100      7176          512 x 16  173 / 159   1024 x 8 164 / 155
  //   4104          1024 x 7  115 / 102   512 x 16 134 / 114      8192          512 x 16  162 / 148   1024 x 8 166 / 151
  //   6304          1024 x 7  155 / 154   512 x 16 177 / 162      8200          512 x 25  186 / 172   1024 x 13 227 / 185
  // 512 x 25 keeps up to 18 registers in memory; us of it and of the row in passes: 8200 vectors 185 / 172 and 183 / 174, 10000 186 / 174 and
  // 193 / 182, 12608 185 / 170 and 188 / 180.
#define ZB_ROWS(THREADS, NV, WAVES)                                                                                                              \
  if (vectors <= THREADS * NV) {                                                                                                                 \
    ZB_NT((policy_row_kernel<T, THREADS, NV, WAVES, NT><<<x->rows, THREADS, 0, s>>>((const T*)x->logits, x->row_stride, of, out, pol, (T*)dlogits, \
                                                                                   dstride)));                                                   \
    return hipGetLastError();                                                                                                                    \
  }
  ZB_ROWS(64, 4, 1)
  ZB_ROWS(256, 4, 1)
  ZB_ROWS(512, 4, 1)
  ZB_ROWS(512, 8, 6)
  ZB_ROWS(1024, 7, 8)
  ZB_ROWS(512, 16, 4)
  ZB_ROWS(512, 25, 4)
#undef ZB_ROWS
  ZB_NT((row_kernel<T, 1024, 4, true, NT><<<x->rows, 1024, 0, s>>>((const T*)x->logits, x->row_stride, of, out, pol, (T*)dlogits, dstride)));
  return hipGetLastError();
}
template <typename T>
hipError_t launch_grad(const zb_logits* x, const Rows& of, const float* coef, const float* top, const float* inv, const float* miss, void* d, int64_t stride,
                       hipStream_t s) {
  const int per = kThreads * kGradVectors, vectors = x->vocab / Span<T>::VE, parts = vectors > per ? (vectors + per - 1) / per : 1;
  const int most = (int)((1LL << 32) / kThreads - 1) / parts;  // rows of a launch
  for (int row0 = 0; row0 < x->rows; row0 += most) {
    const unsigned wgs = (unsigned)(x->rows - row0 < most ? x->rows - row0 : most) * (unsigned)parts;
    ZB_NT((grad_kernel<T, NT><<<wgs, kThreads, 0, s>>>((const T*)x->logits, x->row_stride, of, coef, top, inv, miss, (T*)d, stride, parts, row0)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
hipError_t launch_grad(const zb_logits* x, const Rows& of, const float* coef, const float* top, const float* inv, const float* miss, void* d, int64_t stride,
                       hipStream_t s) {
  return x->dtype == ZB_BF16 ? launch_grad<bf16_t>(x, of, coef, top, inv, miss, d, stride, s)
                             : launch_grad<float>(x, of, coef, top, inv, miss, d, stride, s);
}
zb_status said(hipError_t e) { return e == hipSuccess ? ZB_OK : ZB_EDEVICE; }

}  // namespace

size_t loss_workspace_bytes(int rows, int pairs) {
  const size_t n = (size_t)(rows > pairs ? rows : pairs);
  return n * sizeof(double) + (size_t)rows * (sizeof(double) + 4 * sizeof(float)) + 256;
}

bool valid_policy(const zb_policy* p) {
  return p->clip_low >= 0 && p->clip_low <= 1 && p->clip_high >= 0 && p->kl_coef >= 0 && isfinite(p->clip_high) && isfinite(p->kl_coef) && isfinite(p->scale);
}
bool valid_preference(const zb_preference* p) {
  return p->pairs >= 0 && p->pairs <= kLossMaxRows && isfinite(p->beta) && isfinite(p->scale) && p->label_smoothing >= 0 && p->label_smoothing <= 1;
}

zb_status policy_loss(const zb_logits* x, const zb_policy* p, double grad_scale, float* loss, float* logp, void* dlogits, int64_t dlogits_stride,
                      void* workspace, size_t workspace_size, hipStream_t s) {
  if (!valid_logits(x) || !p || !loss || !valid_dlogits(x, dlogits, &dlogits_stride) || !valid_policy(p)) return ZB_EINVAL;
  if (x->rows && (!p->old_logp || !p->advantage || (p->kl_coef != 0 && !p->ref_logp))) return ZB_EINVAL;
  if (!workspace || misaligned(workspace, 8) || workspace_size < loss_workspace_bytes(x->rows, 0)) return ZB_EINVAL;
  if (misaligned(loss, 4) || misaligned(logp, 4) || misaligned(p->old_logp, 4) || misaligned(p->advantage, 4) || misaligned(p->ref_logp, 4) ||
      misaligned(p->weight, 4))
    return ZB_EINVAL;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  const Workspace w = carve(workspace, x->rows, 0);
  if (x->rows) {
    const Rows of{x->targets, p->weight, nullptr, 0, x->vocab};
    const PolicyArgs a{p->old_logp, p->ref_logp, p->advantage, 1.0 - p->clip_low, 1.0 + p->clip_high, log(1.0 - p->clip_low), log1p(p->clip_high), p->kl_coef, p->scale, grad_scale};
    RowOut out{logp};
    out.part = w.part;
    if (x->rows <= kSumInPlace) out.total = Total{loss, w.done};
    const hipError_t e = x->dtype == ZB_BF16 ? launch_policy<bf16_t>(x, of, out, a, dlogits, dlogits_stride, s)
                                             : launch_policy<float>(x, of, out, a, dlogits, dlogits_stride, s);
    if (e != hipSuccess || out.total.loss) return said(e);
  }
  sum_kernel<<<1, 1024, 0, s>>>(w.part, x->rows, loss);
  return said(hipGetLastError());
}

zb_status preference_loss(const zb_logits* x, const zb_preference* p, double grad_scale, float* loss, float* logp, float* rewards, void* dlogits,
                          int64_t dlogits_stride, void* workspace, size_t workspace_size, hipStream_t s) {
  if (!valid_logits(x) || !p || !loss || !valid_dlogits(x, dlogits, &dlogits_stride) || !valid_preference(p)) return ZB_EINVAL;
  if ((p->pairs && !p->offsets) || (x->rows && p->pairs && !p->ref_logp)) return ZB_EINVAL;
  if (!workspace || misaligned(workspace, 8) || workspace_size < loss_workspace_bytes(x->rows, p->pairs)) return ZB_EINVAL;
  if (misaligned(loss, 4) || misaligned(logp, 4) || misaligned(rewards, 4) || misaligned(p->offsets, 4) || misaligned(p->ref_logp, 4) ||
      misaligned(p->weight, 4))
    return ZB_EINVAL;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  const Workspace w = carve(workspace, x->rows, p->pairs);
  const Rows of{x->targets, p->weight, p->pairs ? p->offsets : nullptr, p->pairs ? 2 * p->pairs : -1, x->vocab};
  if (x->rows) {
    RowOut out{logp};
    out.top = w.top; out.inv = w.inv; out.miss = w.miss; out.logp64 = w.logp;
    if (launch_logp(x, of, out, !dlogits && past_caches(x), s) != hipSuccess) return ZB_EDEVICE;
  }
  if (p->pairs) {
    const PairArgs a{p->ref_logp, p->beta, p->label_smoothing, p->scale, grad_scale};
    pair_kernel<<<p->pairs, kPairThreads, 0, s>>>(a, of, x->rows, w.logp, rewards, w.coef, w.part, p->pairs <= kSumInPlace ? Total{loss, w.done} : Total{});
    if (hipGetLastError() != hipSuccess) return ZB_EDEVICE;
  }
  if (x->rows && dlogits && launch_grad(x, of, w.coef, w.top, w.inv, w.miss, dlogits, dlogits_stride, s) != hipSuccess) return ZB_EDEVICE;
  if (!p->pairs || p->pairs > kSumInPlace) sum_kernel<<<1, 1024, 0, s>>>(w.part, p->pairs, loss);
  return said(hipGetLastError());
}

}  // namespace zb

using namespace zb;

extern "C" {

// (a caller that asks for lse is about to have the gradient made of the same logits)
zb_status zb_token_logprobs(const zb_logits* x, float* logp, float* lse, void* hip_stream) {
  if (!valid_logits(x) || (x->rows && !logp) || misaligned(logp, 4) || misaligned(lse, 4)) return ZB_EINVAL;
  if (x->rows == 0) return ZB_OK;
  OnDeviceOf on((hipStream_t)hip_stream);
  if (!on.ok) return ZB_EDEVICE;
  return said(launch_logp(x, Rows{x->targets, nullptr, nullptr, 0, x->vocab}, RowOut{logp, lse}, past_caches(x, lse != nullptr), (hipStream_t)hip_stream));
}

zb_status zb_token_logprobs_backward(const zb_logits* x, const float* lse, const float* dlogp, void* dlogits, int64_t dlogits_stride,
                                     void* hip_stream) {
  if (!valid_logits(x) || !valid_dlogits(x, dlogits, &dlogits_stride) || misaligned(lse, 4) || misaligned(dlogp, 4)) return ZB_EINVAL;
  if (x->rows == 0) return ZB_OK;
  if (!lse || !dlogp || !dlogits) return ZB_EINVAL;
  OnDeviceOf on((hipStream_t)hip_stream);
  if (!on.ok) return ZB_EDEVICE;
  return said(launch_grad(x, Rows{x->targets, nullptr, nullptr, 0, x->vocab}, dlogp, lse, nullptr, nullptr, dlogits, dlogits_stride, (hipStream_t)hip_stream));
}

zb_status zb_loss_workspace_bytes(int32_t rows, int32_t pairs, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kLossMaxRows || pairs < 0 || pairs > kLossMaxRows) return ZB_EINVAL;
  *bytes = loss_workspace_bytes(rows, pairs);
  return ZB_OK;
}

zb_status zb_policy_loss(const zb_logits* x, const zb_policy* p, float* loss, float* logp, void* dlogits, int64_t dlogits_stride,
                         void* workspace, size_t workspace_size, void* hip_stream) {
  return policy_loss(x, p, p ? p->scale : 0.0, loss, logp, dlogits, dlogits_stride, workspace, workspace_size, (hipStream_t)hip_stream);
}

zb_status zb_preference_loss(const zb_logits* x, const zb_preference* p, float* loss, float* logp, float* rewards, void* dlogits,
                             int64_t dlogits_stride, void* workspace, size_t workspace_size, void* hip_stream) {
  return preference_loss(x, p, p ? p->scale : 0.0, loss, logp, rewards, dlogits, dlogits_stride, workspace, workspace_size, (hipStream_t)hip_stream);
}

}  // extern "C"
