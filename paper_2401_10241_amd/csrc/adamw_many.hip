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
constexpr int kBlock = 256;                                                   // values that share scales
static_assert(kBlock == kWave * kPerThread, "a wave holds one block");

struct Tensor {
  float* theta;
  const void* grad;
  bf16_t* copy16;
  void *m, *v;
  float *m_scale, *v_scale;
  long n, first;
  int wg0;         // first workgroup of this tensor; negative if earlier launches did a part of it
  unsigned flags;  // kGrad16 | kDecay | kWide
};
constexpr unsigned kGrad16 = 1, kDecay = 2, kWide = 4;  // kWide: all accesses of four values are aligned
constexpr int kTensors = 48;                            // per launch: the arguments of a launch are limited to 4 KB
struct Table {
  int count;
  Tensor t[kTensors];
};
static_assert(sizeof(Table) <= 3848, "launch arguments");

struct Hyper {
  double b1, b2;
  double log_b1, log_b2;
  float b1f, b1c, b2f, b2c, lr, eps, decay;  // b1c = 1 - b1
  double clip;
  unsigned seed;
};
struct Clock {  // zb_adamw_step's `state`: the steps taken, and what all values of the step at hand share
  long t;
  int go;
  float coef, bc1, bc2, ib1, ib2;  // clip coefficient, 1 - b^t and its reciprocal
  double km, kv;                   // coef (1 - b1), coef^2 (1 - b2)
  long unused[2];
};
static_assert(sizeof(Clock) == ZB_ADAMW_STATE_BYTES, "header and kernel file disagree");

__device__ __forceinline__ const Tensor& tensor_of(const Table& tab, unsigned wg) {
  int a = 0, b = tab.count;
  while (b - a > 1) {
    const int mid = (a + b) >> 1;
    if (tab.t[mid].wg0 <= (int)wg) a = mid; else b = mid;
  }
  return tab.t[a];
}

// Four values at p, of which `live` exist; wide: all four, aligned.  NT: the caches are told that they are not wanted again.
template <bool NT, class V> __device__ __forceinline__ V get(const void* p) {
  return NT ? __builtin_nontemporal_load((const V*)p) : *(const V*)p;
}
template <bool NT, class V> __device__ __forceinline__ void put(void* p, V x) {
  if (NT) __builtin_nontemporal_store(x, (V*)p);
  else *(V*)p = x;
}
template <class E> struct Vec;
template <> struct Vec<float> { typedef f32x4 type; };
template <> struct Vec<bf16_t> { typedef bf16x4 type; };
template <bool NT, class E> __device__ __forceinline__ typename Vec<E>::type load4(const E* p, int live, bool wide) {
  typedef typename Vec<E>::type V;
  if (wide) return get<NT, V>(p);
  V x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = e < live ? p[e] : (E)0.f;
  return x;
}
template <bool NT, class E> __device__ __forceinline__ void store4(E* p, int live, bool wide, typename Vec<E>::type x) {
  if (wide) {
    put<NT>(p, x);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (e < live) p[e] = x[e];
}
__device__ __forceinline__ f32x4 load_grad(const Tensor& q, long i, int live, bool wide) {
  if (!(q.flags & kGrad16)) return load4<false, float>((const float*)q.grad + i, live, wide);
  const bf16x4 x = load4<false, bf16_t>((const bf16_t*)q.grad + i, live, wide);
  f32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (float)x[e];
  return y;
}
template <bool NT> __device__ __forceinline__ unsigned load_codes(const void* base, long i, int live, bool wide) {
  const unsigned char* p = (const unsigned char*)base + i;
  if (wide) return get<NT, unsigned>(p);
  unsigned w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) if (e < live) w |= (unsigned)p[e] << (8 * e);
  return w;
}
template <bool NT> __device__ __forceinline__ void store_codes(void* base, long i, int live, bool wide, unsigned w) {
  unsigned char* p = (unsigned char*)base + i;
  if (wide) { put<NT>(p, w); return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (e < live) p[e] = (unsigned char)(w >> (8 * e));
}
__device__ __forceinline__ int live_of(long n, long i) { return n - i >= 4 ? 4 : n > i ? (int)(n - i) : 0; }

__device__ __forceinline__ void move_theta(float& th, float m, float v, const Hyper& hp, float decay, float bc1, float bc2) {
  th = th - hp.lr * (decay * th + (m / bc1) / (sqrtf(v / bc2) + hp.eps));
}

// The same with the hardware's root and reciprocal, each off by one unit in the last place: 8-bit states are bound by instructions, and
// their m and v come from 64 bits, so the update stays as exact as the other.  The root takes a v / bc2 below 2^-126 for 0, 1.09e-19 less than it
// is, so an eps below kNearEps, of which that is more than half a step, takes move_theta.
constexpr float kNearEps = 2e-12f;
__device__ __forceinline__ void move_theta_near(float& th, float m, float v, const Hyper& hp, float decay, float ib1, float ib2) {
  th = th - hp.lr * (decay * th + (m * ib1) * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v * ib2) + hp.eps));
}

constexpr double kUnitM = 1.0 / (127.0 * 127.0), kUnitV = 1.0 / (255.0 * 255.0 * 255.0 * 255.0);
constexpr float kMostFloat = 3.4028235e38f;
// Whether a block's scale is off its largest value by more than half a step of 24 bits: cut off at the largest float, or subnormal (not 0).  Then
// values lie past the top code.
__device__ __forceinline__ bool coarse(float top) { return top >= kMostFloat || __float_as_uint(top) - 1u < 0x007FFFFFu; }
// c^4 for c <= 256 in products of 24 bits (256^4 wraps to 0, which differences of neighbours put right again)
__device__ __forceinline__ unsigned fourth(unsigned c) {
  c &= 0x1FFu;
  const unsigned s = c * c & 0x1FFFFu;
  return s * s;
}
__device__ __forceinline__ double value_m(int c, double unit) { return (double)(c * (c < 0 ? -c : c)) * unit; }
__device__ __forceinline__ double value_v(unsigned c, double unit) { return (double)fourth(c) * unit; }

// A number of 32 bits for each place of a step; its halves h, for m the lower one, stand for n / 131072 in (0, 1) with n = 2 h + 1.
struct Places {  // of four values one after the other
  unsigned low, key;
  __device__ __forceinline__ Places(unsigned long place, unsigned long t, unsigned seed) : low((unsigned)place) {
    key = low * 0x9E3779B1u + (unsigned)(place >> 32) * 0x85EBCA77u + (unsigned)t * 0xC2B2AE3Du + seed;
  }
  __device__ __forceinline__ unsigned number(unsigned e) const {
    unsigned x = key + e * 0x9E3779B1u + (low + e < low ? 0x85EBCA77u : 0u);  // (a carry into the upper half of the place)
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x46A2CA6Bu;
    return x ^ (x >> 16);
  }
};

// Code of |m|: y = |m| / unit lies between c^2 and (c + 1)^2, and the upper code is taken if n / 131072 of the way is less than y - c^2
// (n = 65536: the nearer one).  c comes from the root in 32 bits, which may be on the wrong side of a whole number by
// 127 * 1.5 * 2^-23 at most: then y is that near to a code, and only an n within 3 of 0 or 131072 could take another one.  SURE sets c
// right first, for those (risky()) and for blocks whose values may lie past the top code (coarse()).
template <bool SURE> __device__ __forceinline__ unsigned encode_m(double m, double inv, unsigned n) {
  const double y = fabs(m) * inv;
  int c = (int)__builtin_amdgcn_sqrtf((float)y);
  if (SURE) {
    c = c > 127 ? 127 : c;
    if (c > 0 && (double)(c * c) > y) --c;
    else if (c < 127 && (double)((c + 1) * (c + 1)) <= y) ++c;
  }
  const double r = fma(-(double)c, (double)c, y);
  const unsigned w = 2 * (unsigned)c + 1;
  if ((double)((n & 0x3FFFFu) * (w & 0xFFu)) < r * 131072.0 && (!SURE || c < 127)) ++c;  // (at 127, r < 2^-23 y unless coarse(), too little for any n)
  return (unsigned)(m < 0 ? -c : c) & 0xFFu;
}
// The same for v between c^4 and (c + 1)^4, where the root of the root is off by 255 * 1.6 * 2^-23 at most and n within 6; a positive v has
// code 1 at least.
template <bool SURE> __device__ __forceinline__ unsigned encode_v(double x, double inv, unsigned n) {
  const double y = x * inv;
  int c = (int)__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf((float)y));
  if (SURE) {
    c = c > 255 ? 255 : c;
    if (c > 0 && (double)fourth(c) > y) --c;
    else if (c < 255 && (double)fourth(c + 1) <= y) ++c;
  }
  const unsigned low = fourth(c);
  const double r = y - (double)low;
  if ((double)n * (double)(fourth(c + 1) - low) < r * 131072.0 && (!SURE || c < 255)) ++c;
  return c < 1 && y > 0.0 ? 1u : (unsigned)c & 0xFFu;
}
// Remembers whether one of the numbers given is near the ends of its range: in halves of 16 bits, h < 4 or h >= 65532.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
struct Ends {
  u16x2 least = {0xFFFF, 0xFFFF};
  __device__ __forceinline__ void see(unsigned h) {
    union { unsigned u; u16x2 v; } x{h};
    x.v += (u16x2){4, 4};
    least = __builtin_elementwise_min(least, x.v);
  }
  __device__ __forceinline__ bool risky() const { return least[0] < 8 || least[1] < 8; }
};
template <bool SURE>
__device__ __forceinline__ void encode_four(const double (&m)[4], const double (&v)[4], double im, double iv, const Places& at, Ends* ends, unsigned* wm,
                                            unsigned* wv) {
  *wm = *wv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const unsigned h = at.number(e);
    if (!SURE) ends->see(h);
    *wm |= encode_m<SURE>(m[e], im, 2 * (h & 0xFFFFu) + 1) << (8 * e);
    *wv |= encode_v<SURE>(v[e], iv, 2 * (h >> 16) + 1) << (8 * e);
  }
}

// 1 / unit of a block whose largest value is `top`, from the hardware's reciprocal and two steps towards it; 0 gives every code 0
__device__ __forceinline__ double inverse_of(float top, double unit) {
  const double u = (double)top * unit;
  double r = __builtin_amdgcn_rcp(u);
  r = fma(fma(-u, r, 1.0), r, r);
  r = fma(fma(-u, r, 1.0), r, r);
  return top > 0.f ? r : 0.0;
}

// Whether to step, the clip coefficient, the time stamp and what depends on it; two lanes, one for each average.
__global__ __launch_bounds__(64) void clock_kernel(Clock* k, Hyper hp, const double* sq, const int* nonfinite) {
  double coef = 1.0;
  if (sq) {
    const double s = *sq;
    if (*nonfinite || !isfinite(s)) {
      if (threadIdx.x == 0) k->go = 0;
      return;
    }
    const double c = hp.clip / (sqrt(s) + 1e-6);
    coef = c < 1.0 ? c : 1.0;
  }
  const long t = k->t + 1;
  const bool second = threadIdx.x == 1;
  const double bc = 1.0 - exp((double)t * (second ? hp.log_b2 : hp.log_b1));
  if (threadIdx.x > 1) return;
  (second ? k->bc2 : k->bc1) = (float)bc;
  (second ? k->ib2 : k->ib1) = (float)(1.0 / bc);
  if (second) return;
  k->go = 1;
  k->t = t;
  k->coef = (float)coef;
  k->km = coef * (1.0 - hp.b1);
  k->kv = coef * coef * (1.0 - hp.b2);
}

// The largest of a wave's values, a block's: four steps inside each 16 lanes, two across them, which leave it in the last lane.
__device__ __forceinline__ float block_top(float v) {
#define ZB_STEP(CTRL, ROWS) \
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(v), __float_as_uint(v), CTRL, ROWS, 0xF, false)))
  ZB_STEP(0xB1, 0xF);   // lane ^ 1
  ZB_STEP(0x4E, 0xF);   // lane ^ 2
  ZB_STEP(0x141, 0xF);  // mirrored in 8
  ZB_STEP(0x140, 0xF);  // mirrored in 16
  ZB_STEP(0x142, 0xA);  // the first 16 to the second, the third to the fourth
  ZB_STEP(0x143, 0xC);  // the first 32 to the second
#undef ZB_STEP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// The step of four values of a lane from value i on; WHOLE: all lanes have four, aligned.
template <bool BITS8, bool WHOLE, bool NT> struct Four {
  long i;
  int live;
  bool wide, in;
  f32x4 th, g, m, v;
  bf16x4 g16;
  unsigned cm, cv;
  float tm, tv;

  __device__ __forceinline__ void load(const Tensor& q, long at) {
    i = at;
    live = WHOLE ? 4 : live_of(q.n, i);
    wide = WHOLE || (live == 4 && (q.flags & kWide));
    if (q.flags & kGrad16) g16 = load4<NT, bf16_t>((const bf16_t*)q.grad + i, live, wide);
    else g = load4<NT, float>((const float*)q.grad + i, live, wide);
    th = load4<NT, float>(q.theta + i, live, wide);
    if (BITS8) {
      cm = load_codes<NT>(q.m, i, live, wide);
      cv = load_codes<NT>(q.v, i, live, wide);
      in = WHOLE || i / kBlock * kBlock < q.n;
      tm = in ? q.m_scale[i / kBlock] : 0.f;
      tv = in ? q.v_scale[i / kBlock] : 0.f;
    } else {
      m = load4<NT, float>((const float*)q.m + i, live, wide);
      v = load4<NT, float>((const float*)q.v + i, live, wide);
    }
  }

  __device__ __forceinline__ void move(const Tensor& q, const Hyper& hp, const Clock& clk) {
    const float decay = q.flags & kDecay ? hp.decay : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x = th[e];
      if (BITS8 && hp.eps >= kNearEps) move_theta_near(x, m[e], v[e], hp, decay, clk.ib1, clk.ib2);
      else move_theta(x, m[e], v[e], hp, decay, clk.bc1, clk.bc2);
      th[e] = x;
    }
    store4<NT>(q.theta + i, live, wide, th);
    if (q.copy16) {
      bf16x4 c;
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = (bf16_t)th[e];
      store4<NT>(q.copy16 + i, live, wide, c);
    }
  }

  __device__ __forceinline__ void finish(const Tensor& q, const Hyper& hp, const Clock& clk) {
    if (q.flags & kGrad16) {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = (float)g16[e];
    }
    if (!BITS8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float ge = g[e] * clk.coef;
        m[e] = hp.b1f * m[e] + hp.b1c * ge;
        v[e] = hp.b2f * v[e] + hp.b2c * (ge * ge);
      }
      store4<NT>((float*)q.m + i, live, wide, m);
      store4<NT>((float*)q.v + i, live, wide, v);
      move(q, hp, clk);
      return;
    }
    const double dm = (double)tm * (hp.b1 * kUnitM), dv = (double)tv * (hp.b2 * kUnitV);
    double m64[4], v64[4];
    float top_m = 0.f, top_v = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double ge = (double)g[e];
      m64[e] = value_m((int)(signed char)(cm >> (8 * e)), dm) + clk.km * ge;
      v64[e] = value_v((cv >> (8 * e)) & 0xFFu, dv) + clk.kv * (ge * ge);
      m[e] = (float)m64[e];
      v[e] = (float)v64[e];
      top_m = fmaxf(top_m, fabsf(m[e]));
      top_v = fmaxf(top_v, v[e]);
    }
    move(q, hp, clk);  // (theta's registers are free then)
    __builtin_amdgcn_sched_barrier(0);
    top_m = fminf(block_top(top_m), kMostFloat);
    top_v = fminf(block_top(top_v), kMostFloat);
    const double im = inverse_of(top_m, kUnitM), iv = inverse_of(top_v, kUnitV);
    const Places at((unsigned long)(q.first + i), (unsigned long)clk.t, hp.seed);
    unsigned wm, wv;
    Ends ends;
    encode_four<false>(m64, v64, im, iv, at, &ends, &wm, &wv);
    if (ends.risky() || coarse(top_m) || coarse(top_v)) encode_four<true>(m64, v64, im, iv, at, &ends, &wm, &wv);
    store_codes<NT>(q.m, i, live, wide, wm);
    store_codes<NT>(q.v, i, live, wide, wv);
    if (in && (threadIdx.x & 63) == 0) { q.m_scale[i / kBlock] = top_m; q.v_scale[i / kBlock] = top_v; }
  }
};

// One workgroup per 1024 values; which tensor they belong to stands in the launch's arguments.  32 bits: bound by HBM, 315M values with bf16
// gradients and copies 1490 us = 5.9 TB/s (a large copy moves 4.9, a kernel that changes an array in place 5.9).  8 bits: the same 1024 to 1076 us,
// 4.9 to 4.7 TB/s, about 105 instructions a value, half of them for the codes, which the memory's 800 us do not hide all of.
// (Against 1044 us of that time: two chunks a workgroup, the second's loads on their way before the first is worked on, 1057; eight values of a lane
// instead of four, 96 registers, 1530.)
template <bool BITS8, bool NT>
__global__ __launch_bounds__(kThreads) void adamw_many_kernel(Table tab, Hyper hp, const Clock* __restrict__ clk_at) {
  const Clock clk = *clk_at;
  if (!clk.go) return;
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long at = (long)((int)blockIdx.x - q.wg0) * kChunk, i = at + threadIdx.x * kPerThread;
  if (q.n - at >= kChunk && (q.flags & kWide)) {
    Four<BITS8, true, NT> f;
    f.load(q, i);
    f.finish(q, hp, clk);
  } else {
    Four<BITS8, false, NT> f;
    f.load(q, i);
    f.finish(q, hp, clk);
  }
}

// Moments held in 8 bits as values (bound by HBM: 315M values 502 to 527 us, 6.3 to 6.0 TB/s): Tensor.theta is where m's go, Tensor.grad v's
__global__ __launch_bounds__(kThreads) void read_moments_kernel(Table tab) {
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long i = (long)((int)blockIdx.x - q.wg0) * kChunk + threadIdx.x * kPerThread;
  const int live = live_of(q.n, i);
  if (!live) return;
  const bool wide = live == 4 && (q.flags & kWide);
  const unsigned cm = load_codes<false>(q.m, i, live, wide), cv = load_codes<false>(q.v, i, live, wide);
  const double um = (double)q.m_scale[i / kBlock] * kUnitM, uv = (double)q.v_scale[i / kBlock] * kUnitV;
  f32x4 m, v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = (float)value_m((int)(signed char)(cm >> (8 * e)), um);
    v[e] = (float)value_v((cv >> (8 * e)) & 0xFFu, uv);
  }
  store4<false>(q.theta + i, live, wide, m);
  store4<false>((float*)q.grad + i, live, wide, v);
}

// Values into 8 bits, each to the nearer code: 315M values 840 us = 3.7 TB/s, bound by the instructions of the codes set right for every value, which
// a state that is read back once in a while does not need to be spared.
__global__ __launch_bounds__(kThreads) void write_moments_kernel(Table tab) {
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long i = (long)((int)blockIdx.x - q.wg0) * kChunk + threadIdx.x * kPerThread;
  const int live = live_of(q.n, i);
  const bool wide = live == 4 && (q.flags & kWide);
  float tm = 0.f, tv = 0.f;
  const f32x4 m = load4<false, float>(q.theta + i, live, wide), v = load4<false, float>((const float*)q.grad + i, live, wide);
#pragma unroll
  for (int e = 0; e < 4; ++e) { tm = fmaxf(tm, fabsf(m[e])); tv = fmaxf(tv, v[e]); }
  tm = fminf(block_top(tm), kMostFloat);
  tv = fminf(block_top(tv), kMostFloat);
  const double im = inverse_of(tm, kUnitM), iv = inverse_of(tv, kUnitV);
  unsigned wm = 0, wv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    wm |= encode_m<true>((double)m[e], im, 65536) << (8 * e);
    wv |= encode_v<true>((double)v[e], iv, 65536) << (8 * e);
  }
  store_codes<false>(q.m, i, live, wide, wm);
  store_codes<false>(q.v, i, live, wide, wv);
  const long block = i / kBlock;
  if (block * kBlock < q.n && (threadIdx.x & 63) == 0) { q.m_scale[block] = tm; q.v_scale[block] = tv; }
}

// ---- norm ---------------------------------------------------------------------------------------------------------
constexpr int kNormVectors = 16, kNormChunk = kNormVectors * kChunk;  // values of a workgroup
constexpr int kNormInPlace = 256;
struct NormOut {
  double* sq;
  int* nf;
  unsigned* done;  // null: a kernel of its own adds the parts
};
// Sum and flag of n parts by the THREADS lanes of a workgroup, in an order that only n decides; lane 0 writes them.
template <int THREADS, class F> __device__ __forceinline__ void add_parts(long n, F&& part, double* sq, int* nf) {
  __shared__ double red[THREADS / 64];
  __shared__ int redf[THREADS / 64];
  double acc = 0.0;
  int bad = 0;
  for (long i0 = threadIdx.x; i0 < n; i0 += 8 * THREADS) {  // eight loads on their way at a time
    double x[8];
    int f[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = 0.0;
      f[k] = 0;
      if (i0 + k * THREADS < n) part(i0 + k * THREADS, &x[k], &f[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) { acc += x[k]; bad |= f[k]; }
  }
  acc = wave_sum(acc);
  bad = __any(bad);
  if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = acc; redf[threadIdx.x >> 6] = bad; }
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 1; w < THREADS / 64; ++w) { acc += red[w]; bad |= redf[w]; }
  *sq = acc;
  *nf = bad ? 1 : 0;
}
__global__ __launch_bounds__(1024) void norm_sum_kernel(const double* __restrict__ part_sq, const int* __restrict__ part_nf, long parts,
                                                        double* __restrict__ sq_out, int* __restrict__ nf_out) {
  add_parts<1024>(parts, [&](long i, double* x, int* f) { *x = part_sq[i]; *f = part_nf[i]; }, sq_out, nf_out);
}
// One part per workgroup; bound by HBM: 315M bf16 gradients 96 us = 6.6 TB/s.  us of the call with chunks of 4 / 8 / 16 / 32 times 1024
// values: 109 / 101 / 99 / 97; 16 leaves twice the workgroups of 32 to shorter lists.  A launch of up to kNormInPlace of them adds the parts
// itself: the workgroup that is through last does, reading past the caches of the XCDs what the others wrote past them; `done` counts
// modulo the workgroups, so it is 0 again for the next call.
template <bool NT> __global__ __launch_bounds__(kThreads) void norm_many_kernel(Table tab, double* part_sq, int* part_nf, NormOut out) {
  __shared__ double red[kThreads / 64];
  __shared__ int redf[kThreads / 64];
  __shared__ bool last;
  const Tensor& q = tensor_of(tab, blockIdx.x);
  const long start = (long)((int)blockIdx.x - q.wg0) * kNormChunk, i0 = start + threadIdx.x * kPerThread;
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  int bad = 0;
  auto take = [&](const f32x4& g) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bad |= (__float_as_uint(g[e]) & 0x7F800000u) == 0x7F800000u ? 1 : 0;
      acc[e] = fma((double)g[e], (double)g[e], acc[e]);
    }
  };
  if (q.n - start >= kNormChunk && (q.flags & kWide)) {
    if (q.flags & kGrad16) {  // eight loads on their way at a time
      const bf16_t* p = (const bf16_t*)q.grad + start + threadIdx.x * 8;
#pragma unroll
      for (int k = 0; k < kNormVectors / 2; ++k) {
        const bf16x8 x = get<NT, bf16x8>(p + (long)k * kThreads * 8);
        const f32x4 a = {(float)x[0], (float)x[1], (float)x[2], (float)x[3]}, b = {(float)x[4], (float)x[5], (float)x[6], (float)x[7]};
        take(a);
        take(b);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kNormVectors; ++k) take(get<NT, f32x4>((const float*)q.grad + i0 + (long)k * kChunk));
    }
  } else {
    for (int k0 = 0; k0 < kNormVectors && start + k0 * kChunk < q.n; k0 += 4) {
      f32x4 g[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long i = i0 + (long)(k0 + k) * kChunk;
        const int live = live_of(q.n, i);
        g[k] = load_grad(q, i, live, live == 4 && (q.flags & kWide));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) take(g[k]);
    }
  }
  double sum = wave_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
  bad = __any(bad);
  if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = sum; redf[threadIdx.x >> 6] = bad; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) { sum += red[w]; bad |= redf[w]; }
    if (!out.done) {
      part_sq[blockIdx.x] = sum;
      part_nf[blockIdx.x] = bad;
    } else {
      __hip_atomic_store(part_sq + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(part_nf + blockIdx.x, bad, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __builtin_amdgcn_atomic_inc32(out.done, gridDim.x - 1, __ATOMIC_ACQ_REL, "agent") == gridDim.x - 1;
    }
  }
  if (!out.done) return;
  __syncthreads();
  if (!last) return;
  add_parts<kThreads>(gridDim.x, [&](long i, double* x, int* f) {
    *x = __hip_atomic_load(part_sq + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *f = __hip_atomic_load(part_nf + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }, out.sq, out.nf);
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

// Walks the tensors in launches of at most kTensors and kMaxWorkgroups (a launch has less than 2^32 lanes; 2^34 values pass that);
// start(table, workgroups) issues one.  `chunk` values per workgroup, fill(tensor, row of the table) says what the kernel finds
// there and returns whether its accesses are aligned.
constexpr long kMaxWorkgroups = (1L << 32) / kThreads - 1;
template <class Fill, class Start>
hipError_t for_tables(const zb_adamw_tensor* t, int32_t count, long chunk, Fill&& fill, Start&& start) {
  Table tab;
  tab.count = 0;
  long wgs = 0;
  for (int32_t k = 0; k < count; ++k) {
    const long need = (t[k].n + chunk - 1) / chunk;
    for (long done = 0; done < need;) {
      if (tab.count == kTensors || wgs == kMaxWorkgroups) {
        hipError_t e = start(tab, (unsigned)wgs);
        if (e != hipSuccess) return e;
        tab.count = 0;
        wgs = 0;
      }
      Tensor& q = tab.t[tab.count++];
      q = Tensor{};
      q.n = t[k].n;
      q.first = t[k].first;
      q.wg0 = (int)(wgs - done);
      q.flags = (t[k].grad_dtype == ZB_BF16 ? kGrad16 : 0) | (t[k].decay ? kDecay : 0);
      if (fill(k, &q)) q.flags |= kWide;
      const long now = need - done < kMaxWorkgroups - wgs ? need - done : kMaxWorkgroups - wgs;
      done += now;
      wgs += now;
    }
  }
  return tab.count ? start(tab, (unsigned)wgs) : hipSuccess;
}

int32_t live_tensors(const zb_adamw_tensor* t, int32_t count) {
  int32_t n = 0;
  for (int32_t k = 0; k < count; ++k) n += t[k].n > 0;
  return n;
}
size_t norm_parts(const zb_adamw_tensor* t, int32_t count) {
  size_t n = 0;
  for (int32_t k = 0; k < count; ++k) n += (size_t)((t[k].n + kNormChunk - 1) / kNormChunk);
  return n;
}
bool wide_grad(const zb_adamw_tensor& t) { return !misaligned(t.grad, t.grad_dtype == ZB_BF16 ? 8 : 16); }  // for four values

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
  double* sq = (double*)((char*)workspace + ZB_WORKSPACE_KEPT_BYTES);
  int* nf = (int*)(sq + parts);
  const bool alone = parts > 0 && parts <= (size_t)kNormInPlace && live_tensors(tensors, count) <= kTensors;
  const NormOut out{sq_out, nonfinite_out, alone ? (unsigned*)workspace : nullptr};
  // gradients that no cache would hold until the step reads them again
  double held = 0.0;
  for (int32_t k = 0; k < count; ++k) held += (double)tensors[k].n * (tensors[k].grad_dtype == ZB_BF16 ? 2 : 4);
  const bool nt = held > 256.0 * (1 << 20);
  size_t at = 0;
  hipError_t e = for_tables(
      tensors, count, kNormChunk,
      [&](int32_t k, Tensor* q) { q->grad = tensors[k].grad; return !misaligned(tensors[k].grad, 16); },
      [&](const Table& tab, unsigned wgs) {
        if (nt) norm_many_kernel<true><<<wgs, kThreads, 0, s>>>(tab, sq + at, nf + at, out);
        else norm_many_kernel<false><<<wgs, kThreads, 0, s>>>(tab, sq + at, nf + at, out);
        at += wgs;
        return hipGetLastError();
      });
  if (e != hipSuccess) return ZB_EDEVICE;
  if (alone) return ZB_OK;
  norm_sum_kernel<<<1, 1024, 0, s>>>(sq, nf, (long)parts, sq_out, nonfinite_out);
  return hipGetLastError() == hipSuccess ? ZB_OK : ZB_EDEVICE;
}

zb_status zb_adamw_step(const zb_adamw_config* cfg, const zb_adamw_tensor* tensors, int32_t count, double lr, void* state, const double* sq,
                        const int32_t* nonfinite, void* hip_stream) {
  if (!cfg || !valid_tensors(tensors, count) || !state || misaligned(state, 8)) return ZB_EINVAL;
  if (cfg->bits != 8 && cfg->bits != 32) return ZB_EINVAL;
  if (!(cfg->beta1 > 0 && cfg->beta1 < 1 && cfg->beta2 > 0 && cfg->beta2 < 1 && cfg->clip > 0)) return ZB_EINVAL;
  // as the kernels use them; eps is divided by where a value has had no gradient, with a reciprocal that takes normal numbers
  if (!((float)cfg->eps >= 1.17549435e-38f) || !isfinite((float)cfg->eps) || !isfinite((float)cfg->weight_decay) || !isfinite((float)lr)) return ZB_EINVAL;
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
  hp.b1 = cfg->beta1; hp.b2 = cfg->beta2; hp.log_b1 = log(cfg->beta1); hp.log_b2 = log(cfg->beta2);
  hp.b1f = (float)cfg->beta1; hp.b1c = (float)(1.0 - cfg->beta1); hp.b2f = (float)cfg->beta2; hp.b2c = (float)(1.0 - cfg->beta2);
  hp.lr = (float)lr; hp.eps = (float)cfg->eps; hp.decay = (float)cfg->weight_decay; hp.clip = cfg->clip; hp.seed = cfg->seed;
  clock_kernel<<<1, 64, 0, s>>>((Clock*)state, hp, sq, nonfinite);
  if (hipGetLastError() != hipSuccess) return ZB_EDEVICE;
  const bool b8 = cfg->bits == 8;
  // States that no cache would hold until the next step: more than the 256 MB of the last one.  us of 315M values with bf16 gradients with /
  // without the caches' being told: 32 bits 1490 / 1636, 8 bits 1076 / 1110.
  double held = 0.0;
  for (int32_t k = 0; k < count; ++k) held += (double)tensors[k].n * (b8 ? 6 : 12);
  const bool nt = held > 256.0 * (1 << 20);
  const hipError_t e = for_tables(
      tensors, count, kChunk,
      [&](int32_t k, Tensor* q) {
        const zb_adamw_tensor& t = tensors[k];
        q->theta = t.theta; q->grad = t.grad; q->copy16 = (bf16_t*)t.copy16; q->m = t.m; q->v = t.v; q->m_scale = t.m_scale; q->v_scale = t.v_scale;
        const uintptr_t a = b8 ? 4 : 16;
        return !misaligned(t.theta, 16) && wide_grad(t) && !misaligned(t.copy16, 8) && !misaligned(t.m, a) && !misaligned(t.v, a);
      },
      [&](const Table& tab, unsigned wgs) {
        const Clock* clk = (const Clock*)state;
        if (b8 && nt) adamw_many_kernel<true, true><<<wgs, kThreads, 0, s>>>(tab, hp, clk);
        else if (b8) adamw_many_kernel<true, false><<<wgs, kThreads, 0, s>>>(tab, hp, clk);
        else if (nt) adamw_many_kernel<false, true><<<wgs, kThreads, 0, s>>>(tab, hp, clk);
        else adamw_many_kernel<false, false><<<wgs, kThreads, 0, s>>>(tab, hp, clk);
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
