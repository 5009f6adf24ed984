// What the kernels of a dense residual block (layernorm.hip, dropout.hip, linear.hip) share: access to rows that start anywhere, the
// dropout generator, the activations and their derivatives.
#pragma once
#include <math.h>

#include "elem.h"
#include "internal.h"

namespace resist {

constexpr unsigned kMaxThreads = 0xffffffffu;   // of a launch, along an axis

// Rows of a matrix whose stride or width is no multiple of 16 bytes start anywhere an element can: 16-byte accesses that promise no more
// than the element's own alignment (one instruction each all the same: global memory takes any address).
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <typename T> struct Row;
template <> struct Row<float> {
  __device__ static inline void load(const float *p, float (&v)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4_any *>(p), b = *reinterpret_cast<const f32x4_any *>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[e + 4] = b[e]; }
  }
  __device__ static inline void store(float *p, const float (&v)[8]) {
    *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};
template <> struct Row<__bf16> {
  __device__ static inline void load(const __bf16 *p, float (&v)[8]) {
    const u32x4 t = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(t[i]); v[2 * i + 1] = bf16_hi(t[i]); }
  }
  __device__ static inline void store(__bf16 *p, const float (&v)[8]) {
    u32x4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<u32x4_any *>(p) = t;
  }
};
// The `left` elements that a row still has, fewer than eight, on their way at once: past the end the last one again, where a branch for each would wait
// for each (dropout of 16388 x 4095 bf16 with a residual 114 -> 88 us, 4096 x 2047 -> 2047 with GELU, dropout and z 63 -> 59).
template <typename T> __device__ inline void tail_load(const T *p, int left, T (&t)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = p[min(e, left - 1)];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = e < left ? t[e] : (T)0.f;
}
// eight elements of a row, or the `left` < 8 that it still has (the others read as zero, and are not written)
template <typename T> __device__ inline void row_load(const T *p, int left, float (&v)[8]) {
  if (left >= 8) { Row<T>::load(p, v); return; }
  T t[8] = {};
  if (left > 0) tail_load(p, left, t);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)t[e];
}
template <typename T> __device__ inline void row_store(T *p, int left, const float (&v)[8]) {
  if (left >= 8) { Row<T>::store(p, v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < left) p[e] = (T)v[e];
}

// eight elements as they are in memory: requested now, widened when used
template <typename T> struct Raw8;
template <> struct Raw8<float> { f32x4 a, b; };
template <> struct Raw8<__bf16> { u32x4 a; };
__device__ inline void raw_load(const float *p, int left, Raw8<float> &r) {
  if (left >= 8) {
    r.a = *reinterpret_cast<const f32x4_any *>(p);
    r.b = *reinterpret_cast<const f32x4_any *>(p + 4);
  } else {
    float t[8] = {};
    if (left > 0) tail_load(p, left, t);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.a[e] = t[e];
      r.b[e] = t[e + 4];
    }
  }
}
__device__ inline void raw_load(const __bf16 *p, int left, Raw8<__bf16> &r) {
  if (left >= 8) {
    r.a = *reinterpret_cast<const u32x4_any *>(p);
  } else {
    unsigned short t[8] = {};
    if (left > 0) tail_load(reinterpret_cast<const unsigned short *>(p), left, t);
#pragma unroll
    for (int e = 0; e < 4; ++e) r.a[e] = t[2 * e] | (unsigned)t[2 * e + 1] << 16;
  }
}
// what was requested is there from here on
__device__ inline void arrived(Raw8<float> &r) { asm volatile("" : "+v"(r.a), "+v"(r.b)); }
__device__ inline void arrived(Raw8<__bf16> &r) { asm volatile("" : "+v"(r.a)); }
__device__ inline void widen(const Raw8<float> &r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = r.a[e]; v[e + 4] = r.b[e]; }
}
__device__ inline void widen(const Raw8<__bf16> &r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[2 * e] = bf16_lo(r.a[e]); v[2 * e + 1] = bf16_hi(r.a[e]); }
}

// sum of p[i * apart], i = first, first + step, ... below `parts`, in order, in float64, U of them on their way at once
template <int U> __device__ inline double parts_sum(const float *p, size_t apart, int first, int step, int parts) {
  double s = 0.;
  for (int i = first; i < parts; i += U * step) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = p[(size_t)min(i + u * step, parts - 1) * apart];   // the last one, rather than a branch, past the end
#pragma unroll
    for (int u = 0; u < U; ++u) s += i + u * step < parts ? (double)v[u] : 0.;
  }
  return s;
}

// ---- dropout: splitmix64 addressed by position.  Output number c of the sequence started from `state` is a pure function of
// state + (c + 1) * golden, so the mask is computed wherever it is needed and never stored.  state is itself the
// first output of the sequence seeded with the caller's seed: sequences of neighbouring seeds would else be the same one, shifted.
typedef unsigned long long u64;
constexpr u64 kGolden = 0x9E3779B97F4A7C15ull;
__device__ inline u64 splitmix(u64 z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
struct Dropout {
  const u64 *rng;   // device {seed, offset}; NULL: every element is kept
  unsigned thr;     // an element is dropped where its 32 bits are below p * 2^32
  float scale;      // 1 / (1 - p)
};
inline Dropout make_dropout(const DropSpec &s) {
  if (s.p == 0. || !s.rng) return Dropout{nullptr, 0, 1.f};
  return Dropout{reinterpret_cast<const u64 *>(s.rng), (unsigned)nearbyint(s.p * 4294967296.), (float)(1. / (1. - s.p))};
}
// what a word's number is added to: word c is splitmix(base + c * golden)
__device__ inline u64 dropout_base(const u64 *rng) { return splitmix(rng[0] + kGolden) + (rng[1] + 1) * kGolden; }
// elements j .. j+7 of a row (j even), the first word's number times golden added to the base
__device__ inline void dropout8(u64 at, unsigned thr, float scale, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i, at += kGolden) {
    const u64 w = splitmix(at);
    v[2 * i] = (unsigned)w < thr ? 0.f : v[2 * i] * scale;
    v[2 * i + 1] = (unsigned)(w >> 32) < thr ? 0.f : v[2 * i + 1] * scale;
  }
}

// ---- activations.  a(z) and a'(z):
//   ReLU        max(z, 0)                                 1 where z > 0
//   GELU        z Phi(z)                                  Phi(z) + z phi(z)             (normal distribution and its density)
//   GELU, tanh  z s,  s = 1/(1+exp(-2u)),                 s + z s (1 - s) 2 u',  u' = c (1 + 3*0.044715 z^2)
//               u = c (z + 0.044715 z^3), c = sqrt(2/pi)  (z/2 (1 + tanh u) is the same function)
//   SiLU        z s,  s = 1/(1+exp(-z))                   s + z s (1 - s)
constexpr float kGeluC = 0.7978845608028654f, kGeluK = 0.044715f, kInvSqrt2Pi = 0.3989422804014327f, kLog2e = 1.4426950408889634f;
__device__ inline float exp2_f(float x) { return __builtin_amdgcn_exp2f(x); }   // one instruction each, within a step
__device__ inline float rcp_f(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ inline float sigmoid_f(float x) { return rcp_f(1.f + exp2_f(-kLog2e * x)); }
// Far out, where Phi, the logistic and the derivatives are 0 or 1 to the last bit, what grows is held back: it would meet that zero as infinity.  (One
// instruction; of a NaN it makes a number, but the other factor is one as well then.)
__device__ inline float held(float z, float most) { return __builtin_amdgcn_fmed3f(z, -most, most); }
// Q(x) = 1 - Phi(x) for 0 <= x <= 20, and e = exp(-x^2/2), which is phi(x) sqrt(2 pi).  Q(x)/e, Mills' ratio over sqrt(2 pi), is nearly a
// polynomial in t = 1/(1 + c x): this one (of degree 8 without a constant, fitted to the least relative error on 0 ... 14.5, with c) is
// off by 1e-7 of itself, x Q(x) in fp32 by 8e-8 at most.  Half the instructions of erfcf.  -> Q(x)/e
__device__ inline float upper_tail_over(float x, float &e) {
  const float t = rcp_f(__builtin_fmaf(0.3050354009f, x, 1.f));
  float p = 0.03664687152f;
  p = __builtin_fmaf(p, t, -0.1527197052f);
  p = __builtin_fmaf(p, t, 0.1851797860f);
  p = __builtin_fmaf(p, t, -0.03752325448f);
  p = __builtin_fmaf(p, t, 0.1207946772f);
  p = __builtin_fmaf(p, t, 0.1034960125f);
  p = __builtin_fmaf(p, t, 0.1224711978f);
  p = __builtin_fmaf(p, t, 0.1216544519f);
  e = exp2_f(x * x * (-0.5f * kLog2e));
  return p * t;
}
template <int V> __device__ inline void activate(float (&v)[V], int act) {
  if (act == RESIST_ACT_RELU) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = v[k] > 0.f ? v[k] : 0.f;
  } else if (act == RESIST_ACT_GELU) {   // z - z Q(z), or z Q(-z)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float z = v[k], x = fabsf(z) > 20.f ? 20.f : fabsf(z);
      float e;
      const float q = upper_tail_over(x, e);
      v[k] = (z > 0.f ? z : 0.f) - x * q * e;
    }
  } else if (act == RESIST_ACT_GELU_TANH) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = fmaxf(v[k], -20.f) * sigmoid_f(2.f * kGeluC * (v[k] + kGeluK * v[k] * v[k] * v[k]));
  } else if (act == RESIST_ACT_SILU) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = fmaxf(v[k], -200.f) * sigmoid_f(v[k]);
  }
}
// v[k] *= a'(z[k])
template <int V> __device__ inline void times_slope(float (&v)[V], const float (&z)[V], int act) {
  if (act == RESIST_ACT_RELU) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = z[k] > 0.f ? v[k] : 0.f;
  } else if (act == RESIST_ACT_GELU) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      // at x = |z|, Phi(-x) - x phi(x) = (Q/e - x/sqrt(2 pi)) e is a'(-x), and 1 - a'(x)
      const float x = fabsf(z[k]);
      float e;
      const float q = upper_tail_over(x, e), r = e * __builtin_fmaf(-kInvSqrt2Pi, held(x, 20.f), q);
      v[k] *= z[k] > 0.f ? 1.f - r : r;
    }
  } else if (act == RESIST_ACT_GELU_TANH) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float s = sigmoid_f(2.f * kGeluC * (z[k] + kGeluK * z[k] * z[k] * z[k])), t = held(z[k], 20.f);
      v[k] *= s + s * (1.f - s) * t * (2.f * kGeluC + 6.f * kGeluC * kGeluK * t * t);
    }
  } else if (act == RESIST_ACT_SILU) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float s = sigmoid_f(z[k]);
      v[k] *= s + s * (1.f - s) * held(z[k], 200.f);
    }
  }
}

}  // namespace resist
