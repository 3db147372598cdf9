// AdamW over many tensors at once, wherever they lie, with moments in 32 or in 8 bits, and the squared norm and
// non-finite flag of their gradients.  With g the gradient times the clip coefficient, step t:
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  theta -= lr (wd theta + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
// 8 bits: 256 consecutive values of a tensor share the scales  top_m = max |m|,  top_v = max v  and are held as
//   m = sign(c) (c / 127)^2 top_m, c in [-127, 127],   v = (c / 255)^4 top_v, c in [0, 255].
// Both are finer near zero: a value 1e-4 (m) or 1e-9 (v) times the block's largest still has a code, in steps that for v
// are 1.6 % of the value at the top and 6 % at a two-hundredth of it.  A running average moves by a share 1 - b of its
// distance per step, often less than half a code, so rounding to the nearest code would hold it still: of the two codes
// around a value the upper is taken with the probability that keeps the mean, by a number made of seed, step and place
// (the same bits on every run).  The moments are computed in 64 bits before they are rounded, so codes do not depend on
// the order of operations either; theta moves by the moments before their rounding.  A positive v keeps code 1 at least:
// its root is divided by.
#include <math.h>

#include "../../include/zb_stage.h"
#include "zb_common.h"

namespace zb {

namespace {

constexpr int kThreads = 256, kPerThread = 4, kChunk = kThreads * kPerThread;  // values of a workgroup
constexpr int kBlock = 256;                                                   // values that share scales: a wave's
static_assert(kBlock == kWave * kPerThread, "a wave holds one block");

struct Tensor {
  float* theta;
  const void* grad;
  bf16_t* copy16;
  void *m, *v;
  float *m_scale, *v_scale;
  long n, first;
  unsigned wg0;    // first workgroup of this tensor
  unsigned flags;  // kGrad16 | kDecay | kWide
};
constexpr unsigned kGrad16 = 1, kDecay = 2, kWide = 4;  // kWide: all accesses of four values are aligned
constexpr int kTensors = 44;                            // per launch: the arguments of a launch are limited to 4 KB
struct Table {
  int count;
  Tensor t[kTensors];
};
static_assert(sizeof(Table) <= 3840, "launch arguments");

struct Hyper {
  double b1, b2;
  float b1f, b1c, b2f, b2c, lr, eps, decay;  // b1c = 1 - b1
  double clip;
  unsigned seed;
};
struct Clock {  // zb_adamw_step's `state`
  long t;
  int go;
  float coef32;
  double coef, bc1, bc2;
  long unused[3];
};
static_assert(sizeof(Clock) == ZB_ADAMW_STATE_BYTES, "header and kernel file disagree");

__device__ __forceinline__ const Tensor& tensor_of(const Table& tab, unsigned wg) {
  int a = 0, b = tab.count;
  while (b - a > 1) {
    const int mid = (a + b) >> 1;
    if (tab.t[mid].wg0 <= wg) a = mid; else b = mid;
  }
  return tab.t[a];
}

__device__ __forceinline__ void load_grad(const Tensor& q, long i, int live, bool wide, float (&g)[4]) {
  if (q.flags & kGrad16) {
    const bf16_t* p = (const bf16_t*)q.grad + i;
    if (wide) {
      const bf16x4 x = *(const bf16x4*)p;
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = (float)x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = e < live ? (float)p[e] : 0.f;
    }
  } else {
    const float* p = (const float*)q.grad + i;
    if (wide) {
      const f32x4 x = *(const f32x4*)p;
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = e < live ? p[e] : 0.f;
    }
  }
}
__device__ __forceinline__ void load_f32(const float* p, int live, bool wide, float (&x)[4]) {
  if (wide) {
    const f32x4 y = *(const f32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = y[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = e < live ? p[e] : 0.f;
  }
}
__device__ __forceinline__ void store_f32(float* p, int live, bool wide, const float (&x)[4]) {
  if (wide) {
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[e];
    *(f32x4*)p = y;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) if (e < live) p[e] = x[e];
  }
}
__device__ __forceinline__ unsigned load_codes(const void* base, long i, int live, bool wide) {
  const unsigned char* p = (const unsigned char*)base + i;
  if (wide) return *(const unsigned*)p;
  unsigned w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) if (e < live) w |= (unsigned)p[e] << (8 * e);
  return w;
}
__device__ __forceinline__ void store_codes(void* base, long i, int live, bool wide, unsigned w) {
  unsigned char* p = (unsigned char*)base + i;
  if (wide) { *(unsigned*)p = w; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (e < live) p[e] = (unsigned char)(w >> (8 * e));
}

__device__ __forceinline__ void move_theta(float& th, float m, float v, const Hyper& hp, float decay, float bc1, float bc2) {
  th = th - hp.lr * (decay * th + (m / bc1) / (sqrtf(v / bc2) + hp.eps));
}

constexpr double kUnitM = 1.0 / (127.0 * 127.0), kUnitV = 1.0 / (255.0 * 255.0 * 255.0 * 255.0);
__device__ __forceinline__ double value_m(int c, double unit) { return (double)(c * (c < 0 ? -c : c)) * unit; }
__device__ __forceinline__ double value_v(unsigned c, double unit) { const unsigned s = c * c; return (double)(s * s) * unit; }

// two numbers in (0, 1) for one place of one step
__device__ __forceinline__ void dither(unsigned long place, unsigned long t, unsigned seed, double* um, double* uv) {
  unsigned x = (unsigned)place * 0x9E3779B1u + (unsigned)(place >> 32) * 0x85EBCA77u + (unsigned)t * 0xC2B2AE3Du + seed;
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x46A2CA6Bu;
  x ^= x >> 16;
  *um = ((double)(x & 0xFFFFu) + 0.5) * (1.0 / 65536);
  *uv = ((double)(x >> 16) + 0.5) * (1.0 / 65536);
}

// The largest code c <= MOST with value(c) <= x: guessed in 32 bits from the ratio x / unit, then set right by the values
// themselves; *lo and *hi get value(c) and value(c + 1).
template <int MOST, class V> __device__ __forceinline__ int code_below(double x, int guess, V&& value, double* lo, double* hi) {
  int c = guess < 0 ? 0 : guess > MOST ? MOST : guess;
  if (value(c) > x) c = c > 0 ? c - 1 : 0;
  if (c < MOST && value(c + 1) <= x) ++c;
  *lo = value(c);
  *hi = value(c + 1);
  return c;
}
__device__ __forceinline__ unsigned encode_m(double m, double unit, double inv, double u) {
  const double x = fabs(m);
  double lo, hi;
  int c = code_below<127>(x, (int)__builtin_amdgcn_sqrtf((float)(x * inv)), [&](int k) { return value_m(k, unit); }, &lo, &hi);
  if (c < 127 && u * (hi - lo) < x - lo) ++c;
  if (!(unit > 0.0)) c = 0;
  return (unsigned)(m < 0 ? -c : c) & 0xFFu;
}
__device__ __forceinline__ unsigned encode_v(double x, double unit, double inv, double u) {
  double lo, hi;
  int c = code_below<255>(x, (int)__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf((float)(x * inv))),
                          [&](int k) { return (double)(k * k) * (double)(k * k) * unit; }, &lo, &hi);
  if (c < 255 && u * (hi - lo) < x - lo) ++c;
  if (c < 1 && x > 0.0) c = 1;
  if (!(unit > 0.0)) c = 0;
  return (unsigned)c;
}

// whether to step, the clip coefficient, the time stamp and what depends on it
__global__ void clock_kernel(Clock* k, Hyper hp, const double* sq, const int* nonfinite) {
  k->go = 1;
  k->coef = 1.0;
  if (sq) {
    k->go = !*nonfinite && isfinite(*sq) ? 1 : 0;
    const double c = hp.clip / (sqrt(*sq) + 1e-6);
    k->coef = c < 1.0 ? c : 1.0;
  }
  k->coef32 = (float)k->coef;
  if (!k->go) return;
  k->t += 1;
  k->bc1 = 1.0 - pow(hp.b1, (double)k->t);
  k->bc2 = 1.0 - pow(hp.b2, (double)k->t);
}

template <bool BITS8> __global__ __launch_bounds__(kThreads) void adamw_many_kernel(Table tab, Hyper hp, const Clock* __restrict__ clk) {
  if (!clk->go) return;
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long i = (long)(blockIdx.x - q.wg0) * kChunk + threadIdx.x * kPerThread;
  const int live = q.n - i >= 4 ? 4 : q.n > i ? (int)(q.n - i) : 0;
  const bool wide = live == 4 && (q.flags & kWide);
  const float bc1 = (float)clk->bc1, bc2 = (float)clk->bc2, decay = q.flags & kDecay ? hp.decay : 0.f;
  float g[4], th[4], m32[4], v32[4];
  load_grad(q, i, live, wide, g);
  load_f32(q.theta + i, live, wide, th);
  if (!BITS8) {
    load_f32((const float*)q.m + i, live, wide, m32);
    load_f32((const float*)q.v + i, live, wide, v32);
    const float coef = clk->coef32;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float ge = g[e] * coef;
      m32[e] = hp.b1f * m32[e] + hp.b1c * ge;
      v32[e] = hp.b2f * v32[e] + hp.b2c * (ge * ge);
    }
    store_f32((float*)q.m + i, live, wide, m32);
    store_f32((float*)q.v + i, live, wide, v32);
  } else {
    const unsigned cm = load_codes(q.m, i, live, wide), cv = load_codes(q.v, i, live, wide);
    const long block = i / kBlock;
    const bool in = block * kBlock < q.n;
    const double um = in ? (double)q.m_scale[block] * kUnitM : 0.0, uv = in ? (double)q.v_scale[block] * kUnitV : 0.0;
    double m[4], v[4];
    float tm = 0.f, tv = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double ge = (double)g[e] * clk->coef;
      m[e] = hp.b1 * value_m((int)(signed char)(cm >> (8 * e)), um) + (1.0 - hp.b1) * ge;
      v[e] = hp.b2 * value_v((cv >> (8 * e)) & 0xFFu, uv) + (1.0 - hp.b2) * (ge * ge);
      m32[e] = (float)m[e];
      v32[e] = (float)v[e];
      tm = fmaxf(tm, fabsf(m32[e]));
      tv = fmaxf(tv, v32[e]);
    }
    tm = fminf(wave_max(tm), 3.4028235e38f);
    tv = fminf(wave_max(tv), 3.4028235e38f);
    const double nm = (double)tm * kUnitM, nv = (double)tv * kUnitV;
    const double im = nm > 0.0 ? 1.0 / nm : 0.0, iv = nv > 0.0 ? 1.0 / nv : 0.0;
    unsigned wm = 0, wv = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      double a, b;
      dither((unsigned long)(q.first + i + e), (unsigned long)clk->t, hp.seed, &a, &b);
      wm |= encode_m(m[e], nm, im, a) << (8 * e);
      wv |= encode_v(v[e], nv, iv, b) << (8 * e);
    }
    store_codes(q.m, i, live, wide, wm);
    store_codes(q.v, i, live, wide, wv);
    if (in && (threadIdx.x & 63) == 0) { q.m_scale[block] = tm; q.v_scale[block] = tv; }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) move_theta(th[e], m32[e], v32[e], hp, decay, bc1, bc2);
  store_f32(q.theta + i, live, wide, th);
  if (q.copy16) {
    bf16_t* c = q.copy16 + i;
    if (wide) {
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (bf16_t)th[e];
      *(bf16x4*)c = y;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) if (e < live) c[e] = (bf16_t)th[e];
    }
  }
}

// moments held in 8 bits as values: Tensor.theta is where m's go, Tensor.grad v's
__global__ __launch_bounds__(kThreads) void read_moments_kernel(Table tab) {
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long i = (long)(blockIdx.x - q.wg0) * kChunk + threadIdx.x * kPerThread;
  const int live = q.n - i >= 4 ? 4 : q.n > i ? (int)(q.n - i) : 0;
  if (!live) return;
  const bool wide = live == 4 && (q.flags & kWide);
  const unsigned cm = load_codes(q.m, i, live, wide), cv = load_codes(q.v, i, live, wide);
  const double um = (double)q.m_scale[i / kBlock] * kUnitM, uv = (double)q.v_scale[i / kBlock] * kUnitV;
  float m[4], v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = (float)value_m((int)(signed char)(cm >> (8 * e)), um);
    v[e] = (float)value_v((cv >> (8 * e)) & 0xFFu, uv);
  }
  store_f32(q.theta + i, live, wide, m);
  store_f32((float*)q.grad + i, live, wide, v);
}

// values into 8 bits, each to the nearer code
__global__ __launch_bounds__(kThreads) void write_moments_kernel(Table tab) {
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long i = (long)(blockIdx.x - q.wg0) * kChunk + threadIdx.x * kPerThread;
  const int live = q.n - i >= 4 ? 4 : q.n > i ? (int)(q.n - i) : 0;
  const bool wide = live == 4 && (q.flags & kWide);
  float m[4], v[4], tm = 0.f, tv = 0.f;
  load_f32(q.theta + i, live, wide, m);
  load_f32((const float*)q.grad + i, live, wide, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) { tm = fmaxf(tm, fabsf(m[e])); tv = fmaxf(tv, v[e]); }
  tm = fminf(wave_max(tm), 3.4028235e38f);
  tv = fminf(wave_max(tv), 3.4028235e38f);
  const double nm = (double)tm * kUnitM, nv = (double)tv * kUnitV;
  const double im = nm > 0.0 ? 1.0 / nm : 0.0, iv = nv > 0.0 ? 1.0 / nv : 0.0;
  unsigned wm = 0, wv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    wm |= encode_m((double)m[e], nm, im, 0.5) << (8 * e);
    wv |= encode_v((double)v[e], nv, iv, 0.5) << (8 * e);
  }
  store_codes(q.m, i, live, wide, wm);
  store_codes(q.v, i, live, wide, wv);
  const long block = i / kBlock;
  if (block * kBlock < q.n && (threadIdx.x & 63) == 0) { q.m_scale[block] = tm; q.v_scale[block] = tv; }
}

// ---- norm ---------------------------------------------------------------------------------------------------------
constexpr int kNormChunk = 16 * kChunk;  // values of a workgroup
__global__ __launch_bounds__(kThreads) void norm_many_kernel(Table tab, double* __restrict__ part_sq, int* __restrict__ part_nf) {
  __shared__ double red[kThreads / 64];
  __shared__ int redf[kThreads / 64];
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long i0 = (long)(blockIdx.x - q.wg0) * kNormChunk + threadIdx.x * kPerThread;
  double acc = 0.0;
  int bad = 0;
  for (int k = 0; k < kNormChunk / kChunk; ++k) {
    const long i = i0 + (long)k * kChunk;
    const int live = q.n - i >= 4 ? 4 : q.n > i ? (int)(q.n - i) : 0;
    if (!live) break;
    float g[4];
    load_grad(q, i, live, live == 4 && (q.flags & kWide), g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bad |= (__float_as_uint(g[e]) & 0x7F800000u) == 0x7F800000u ? 1 : 0;
      acc += (double)g[e] * (double)g[e];
    }
  }
  acc = wave_sum(acc);
  bad = __any(bad);
  if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = acc; redf[threadIdx.x >> 6] = bad; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) { acc += red[w]; bad |= redf[w]; }
    part_sq[blockIdx.x] = acc;
    part_nf[blockIdx.x] = bad;
  }
}
__global__ __launch_bounds__(1024) void norm_sum_kernel(const double* __restrict__ part_sq, const int* __restrict__ part_nf, long parts,
                                                        double* __restrict__ sq_out, int* __restrict__ nf_out) {
  __shared__ double red[1024];
  __shared__ int redf[1024];
  double acc = 0.0;
  int bad = 0;
  for (long i = threadIdx.x; i < parts; i += 1024) { acc += part_sq[i]; bad |= part_nf[i]; }
  red[threadIdx.x] = acc;
  redf[threadIdx.x] = bad;
  __syncthreads();
  for (int o = 512; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) { red[threadIdx.x] += red[threadIdx.x + o]; redf[threadIdx.x] |= redf[threadIdx.x + o]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) { *sq_out = red[0]; *nf_out = redf[0] ? 1 : 0; }
}

// ---- host ---------------------------------------------------------------------------------------------------------
bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
constexpr int64_t kMaxValues = (int64_t)1 << 38;

bool valid_tensors(const zb_adamw_tensor* t, int32_t count) {
  if (count < 0 || count > (1 << 20) || (count && !t)) return false;
  for (int32_t k = 0; k < count; ++k) {
    if (t[k].n < 0 || t[k].n > kMaxValues || t[k].first < 0 || t[k].first > ((int64_t)1 << 60)) return false;
    if (t[k].grad_dtype != ZB_FP32 && t[k].grad_dtype != ZB_BF16) return false;
  }
  return true;
}
bool valid_grads(const zb_adamw_tensor& t) { return t.grad && !misaligned(t.grad, t.grad_dtype == ZB_BF16 ? 2 : 4); }
bool valid_codes(const zb_adamw_tensor& t) {
  return t.m && t.v && t.m_scale && t.v_scale && !misaligned(t.m_scale, 4) && !misaligned(t.v_scale, 4);
}

// Walks the tensors in launches of at most kTensors; start(table, workgroups) issues one.  `chunk` values per workgroup,
// fill(tensor, row of the table) says what the kernel finds there and returns whether its accesses are aligned.
template <class Fill, class Start>
hipError_t for_tables(const zb_adamw_tensor* t, int32_t count, long chunk, Fill&& fill, Start&& start) {
  Table tab;
  tab.count = 0;
  unsigned wgs = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (t[k].n == 0) continue;
    const long need = (t[k].n + chunk - 1) / chunk;
    if (tab.count == kTensors || (tab.count && wgs + need > 0x7FFFFFFF)) {
      hipError_t e = start(tab, wgs);
      if (e != hipSuccess) return e;
      tab.count = 0;
      wgs = 0;
    }
    Tensor& q = tab.t[tab.count++];
    q = Tensor{};
    q.n = t[k].n;
    q.first = t[k].first;
    q.wg0 = wgs;
    q.flags = (t[k].grad_dtype == ZB_BF16 ? kGrad16 : 0) | (t[k].decay ? kDecay : 0);
    if (fill(k, &q)) q.flags |= kWide;
    wgs += (unsigned)need;
  }
  return tab.count ? start(tab, wgs) : hipSuccess;
}

size_t norm_parts(const zb_adamw_tensor* t, int32_t count) {
  size_t n = 0;
  for (int32_t k = 0; k < count; ++k) n += (size_t)((t[k].n + kNormChunk - 1) / kNormChunk);
  return n;
}
bool wide_grad(const zb_adamw_tensor& t) { return !misaligned(t.grad, t.grad_dtype == ZB_BF16 ? 8 : 16); }

}  // namespace
}  // namespace zb

using namespace zb;

extern "C" {

zb_status zb_adamw_workspace_bytes(const zb_adamw_tensor* tensors, int32_t count, size_t* bytes) {
  if (!bytes || !valid_tensors(tensors, count)) return ZB_EINVAL;
  *bytes = norm_parts(tensors, count) * (sizeof(double) + sizeof(int)) + 256;
  return ZB_OK;
}

zb_status zb_adamw_grad_norm(const zb_adamw_tensor* tensors, int32_t count, double* sq_out, int32_t* nonfinite_out, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  size_t need = 0;
  if (!sq_out || !nonfinite_out || misaligned(sq_out, 8) || misaligned(nonfinite_out, 4)) return ZB_EINVAL;
  if (zb_adamw_workspace_bytes(tensors, count, &need) != ZB_OK || !workspace || misaligned(workspace, 8) || workspace_bytes < need) return ZB_EINVAL;
  for (int32_t k = 0; k < count; ++k)
    if (tensors[k].n && !valid_grads(tensors[k])) return ZB_EINVAL;
  const hipStream_t s = (hipStream_t)hip_stream;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  const size_t parts = norm_parts(tensors, count);
  double* sq = (double*)workspace;
  int* nf = (int*)(sq + parts);
  size_t at = 0;
  hipError_t e = for_tables(
      tensors, count, kNormChunk,
      [&](int32_t k, Tensor* q) { q->grad = tensors[k].grad; return wide_grad(tensors[k]); },
      [&](const Table& tab, unsigned wgs) {
        norm_many_kernel<<<wgs, kThreads, 0, s>>>(tab, sq + at, nf + at);
        at += wgs;
        return hipGetLastError();
      });
  if (e != hipSuccess) return ZB_EDEVICE;
  norm_sum_kernel<<<1, 1024, 0, s>>>(sq, nf, (long)parts, sq_out, nonfinite_out);
  return hipGetLastError() == hipSuccess ? ZB_OK : ZB_EDEVICE;
}

zb_status zb_adamw_step(const zb_adamw_config* cfg, const zb_adamw_tensor* tensors, int32_t count, double lr, void* state, const double* sq,
                        const int32_t* nonfinite, void* hip_stream) {
  if (!cfg || !valid_tensors(tensors, count) || !state || misaligned(state, 8)) return ZB_EINVAL;
  if (cfg->bits != 8 && cfg->bits != 32) return ZB_EINVAL;
  if (!(cfg->beta1 > 0 && cfg->beta1 < 1 && cfg->beta2 > 0 && cfg->beta2 < 1 && cfg->eps > 0 && cfg->clip > 0) || !isfinite(cfg->eps) ||
      !isfinite(cfg->weight_decay) || !isfinite(lr))
    return ZB_EINVAL;
  if ((sq == nullptr) != (nonfinite == nullptr) || misaligned(sq, 8) || misaligned(nonfinite, 4)) return ZB_EINVAL;
  if (cfg->bits == 8 && !sq) return ZB_EINVAL;  // codes cannot hold a NaN
  for (int32_t k = 0; k < count; ++k) {
    const zb_adamw_tensor& t = tensors[k];
    if (!t.n) continue;
    if (!t.theta || misaligned(t.theta, 4) || !valid_grads(t) || misaligned(t.copy16, 2)) return ZB_EINVAL;
    if (cfg->bits == 8 ? !valid_codes(t) : (!t.m || !t.v || misaligned(t.m, 4) || misaligned(t.v, 4))) return ZB_EINVAL;
  }
  const hipStream_t s = (hipStream_t)hip_stream;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  Hyper hp;
  hp.b1 = cfg->beta1; hp.b2 = cfg->beta2;
  hp.b1f = (float)cfg->beta1; hp.b1c = (float)(1.0 - cfg->beta1); hp.b2f = (float)cfg->beta2; hp.b2c = (float)(1.0 - cfg->beta2);
  hp.lr = (float)lr; hp.eps = (float)cfg->eps; hp.decay = (float)cfg->weight_decay; hp.clip = cfg->clip; hp.seed = cfg->seed;
  clock_kernel<<<1, 1, 0, s>>>((Clock*)state, hp, sq, nonfinite);
  if (hipGetLastError() != hipSuccess) return ZB_EDEVICE;
  const bool b8 = cfg->bits == 8;
  const hipError_t e = for_tables(
      tensors, count, kChunk,
      [&](int32_t k, Tensor* q) {
        const zb_adamw_tensor& t = tensors[k];
        q->theta = t.theta; q->grad = t.grad; q->copy16 = (bf16_t*)t.copy16; q->m = t.m; q->v = t.v; q->m_scale = t.m_scale; q->v_scale = t.v_scale;
        const uintptr_t a = b8 ? 4 : 16;
        return !misaligned(t.theta, 16) && wide_grad(t) && !misaligned(t.copy16, 8) && !misaligned(t.m, a) && !misaligned(t.v, a);
      },
      [&](const Table& tab, unsigned wgs) {
        if (b8) adamw_many_kernel<true><<<wgs, kThreads, 0, s>>>(tab, hp, (const Clock*)state);
        else adamw_many_kernel<false><<<wgs, kThreads, 0, s>>>(tab, hp, (const Clock*)state);
        return hipGetLastError();
      });
  return e == hipSuccess ? ZB_OK : ZB_EDEVICE;
}

static zb_status move_moments(const zb_adamw_tensor* tensors, int32_t count, const zb_adamw_value* values, bool read, void* hip_stream) {
  if (!valid_tensors(tensors, count) || (count && !values)) return ZB_EINVAL;
  for (int32_t k = 0; k < count; ++k)
    if (tensors[k].n && (!valid_codes(tensors[k]) || !values[k].m || !values[k].v || misaligned(values[k].m, 4) || misaligned(values[k].v, 4)))
      return ZB_EINVAL;
  const hipStream_t s = (hipStream_t)hip_stream;
  OnDeviceOf on(s);
  if (!on.ok) return ZB_EDEVICE;
  const hipError_t e = for_tables(
      tensors, count, kChunk,
      [&](int32_t k, Tensor* q) {
        const zb_adamw_tensor& t = tensors[k];
        q->theta = values[k].m; q->grad = values[k].v; q->m = t.m; q->v = t.v; q->m_scale = t.m_scale; q->v_scale = t.v_scale;
        q->flags &= ~kGrad16;
        return !misaligned(values[k].m, 16) && !misaligned(values[k].v, 16) && !misaligned(t.m, 4) && !misaligned(t.v, 4);
      },
      [&](const Table& tab, unsigned wgs) {
        if (read) read_moments_kernel<<<wgs, kThreads, 0, s>>>(tab);
        else write_moments_kernel<<<wgs, kThreads, 0, s>>>(tab);
        return hipGetLastError();
      });
  return e == hipSuccess ? ZB_OK : ZB_EDEVICE;
}
zb_status zb_adamw_read_moments(const zb_adamw_tensor* tensors, int32_t count, const zb_adamw_value* values, void* hip_stream) {
  return move_moments(tensors, count, values, true, hip_stream);
}
zb_status zb_adamw_write_moments(const zb_adamw_tensor* tensors, int32_t count, const zb_adamw_value* values, void* hip_stream) {
  return move_moments(tensors, count, values, false, hip_stream);
}

}  // extern "C"
