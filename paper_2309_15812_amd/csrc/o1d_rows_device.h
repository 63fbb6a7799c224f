// Device helpers of the row operators: runs of 16 bytes, activations, and the
// 8-bit checkpoint's rounding.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "o1d_device.h"
#include "o1d_rows.h"

namespace o1d {
namespace rows {

// A run of N elements as float32.  Global accesses of 16 bytes need only the
// element's alignment on gfx950 (unaligned access is on), so rows of odd
// widths take them too: memcpy from an element pointer.
template <typename T, int N>
__device__ __forceinline__ void load_run(const T* p, float (&v)[N]) {
  T t[N];
  __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = to_f32(t[e]);
}
template <typename T, int N>
__device__ __forceinline__ void store_run(T* p, const float (&v)[N]) {
  T t[N];
#pragma unroll
  for (int e = 0; e < N; ++e) t[e] = from_f32<T>(v[e]);
  __builtin_memcpy(p, t, sizeof(t));
}

// The first n (1 .. N) elements of a run; the others read 0.
template <typename T, int N>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[N]) {
  if (n >= N) {
    load_run(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < n ? to_f32(p[e]) : 0.f;
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[N]) {
  if (n >= N) {
    store_run(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}

// ---- activations.  FAST: for results that are rounded to bfloat16.
//
// gelu(x) = x Phi(x), Phi(x) = (1 + erf(x / sqrt 2)) / 2.  float32 results take the
// library's erf: off by about 2^-24 |x| (with erfc the left tail would keep its bits; a weight gradient
// that makes its operand takes 98 us instead of 83 then, a checkpoint read back 53 instead of 41).
//
// For bfloat16 results Phi(x) = Q(|x|) or 1 - Q(|x|) with the upper tail Q(a) =
// exp(-a^2 / 2) R(a), and R a fit whose relative error is 4e-6 for every a: a
// formula with a small absolute error alone loses the values left of -3, where the
// function is small itself.  The products' epilogues are bound by these slots: 22
// per value against 40 with the library's function.
template <bool FAST>
__device__ __forceinline__ float exp_(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST>
__device__ __forceinline__ float recip(float x) { return FAST ? __builtin_amdgcn_rcpf(x) : 1.f / x; }

// R(a) = Q(a) exp(a^2 / 2) for a >= 0 as t P(t), t = 1 / (1 + 0.308 a): P of the fifth degree with the least largest
// relative error over 0 <= a <= 14 (a fit by reweighted least squares), where exp(-a^2 / 2) leaves float32.
__device__ __forceinline__ float tail_ratio(float a) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.308f, a, 1.f));
  float s = fmaf(-0.07543021440505981f, t, 0.18961861729621887f);
  s = fmaf(s, t, 0.007272266782820225f);
  s = fmaf(s, t, 0.1365339308977127f);
  s = fmaf(s, t, 0.11888113617897034f);
  s = fmaf(s, t, 0.12312270700931549f);
  return s * t;
}
// exp(-x^2 / 2)
__device__ __forceinline__ float bell(float x) { return __builtin_amdgcn_exp2f(x * x * (-0.5f * 1.44269504088896341f)); }

template <bool FAST>
__device__ __forceinline__ float gelu_value(float x) {
  if constexpr (FAST) {
    const float q = bell(x) * tail_ratio(fabsf(x));
    return x * (x < 0.f ? q : 1.f - q);
  }
  return x * (0.5f * (1.f + erff(x * 0.70710678118654752f)));
}

// Phi(x) + x exp(-x^2 / 2) / sqrt(2 pi)
template <bool FAST>
__device__ __forceinline__ float gelu_slope(float x) {
  constexpr float kDensity = 0.39894228040143268f;
  if constexpr (FAST) {
    // Q - a exp(-a^2 / 2) / sqrt(2 pi) for x < 0, 1 less that for x >= 0
    const float a = fabsf(x), q = bell(x) * fmaf(-kDensity, a, tail_ratio(a));
    return x < 0.f ? q : 1.f - q;
  }
  const float z = x * 0.70710678118654752f;
  return fmaf(x * kDensity, expf(-z * z), 0.5f * (1.f + erff(z)));
}

// gelu(x) ~ x sigma(2 u), u = sqrt(2 / pi) (x + 0.044715 x^3)   [(1 + tanh u) / 2 = sigma(2 u)]
constexpr float kTanhScale = 1.59576912160573071f;  // 2 sqrt(2 / pi)
constexpr float kTanhCube = 0.044715f;

template <bool FAST>
__device__ __forceinline__ float act_value(float x, int act) {
  switch (act) {
    case kRelu: return x < 0.f ? 0.f : x;
    case kGelu: return gelu_value<FAST>(x);
    case kGeluTanh: return x * recip<FAST>(1.f + exp_<FAST>(-kTanhScale * (x + kTanhCube * x * x * x)));
    case kSilu: return x * recip<FAST>(1.f + exp_<FAST>(-x));
    default: return x;
  }
}

template <bool FAST>
__device__ __forceinline__ float act_slope(float x, int act) {
  switch (act) {
    case kRelu: return x <= 0.f ? 0.f : 1.f;
    case kGelu: return gelu_slope<FAST>(x);
    case kGeluTanh: {
      const float g = recip<FAST>(1.f + exp_<FAST>(-kTanhScale * (x + kTanhCube * x * x * x)));
      // g (1 - g) is 0 long before |x| = 32, and x^2 leaves float32 at 2e19: the other factors end there
      const float c = fminf(fmaxf(x, -32.f), 32.f);
      return g + c * g * (1.f - g) * kTanhScale * fmaf(3.f * kTanhCube * c, c, 1.f);
    }
    case kSilu: {
      const float g = recip<FAST>(1.f + exp_<FAST>(-x));
      return g * fmaf(x, 1.f - g, 1.f);
    }
    default: return 1.f;
  }
}

template <bool FAST, int N>
__device__ __forceinline__ void act_values(float (&v)[N], int act) {
  // one branch for the run, not one per element
  switch (act) {
    case kRelu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_value<FAST>(v[e], kRelu);
      break;
    case kGelu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_value<FAST>(v[e], kGelu);
      break;
    case kGeluTanh:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_value<FAST>(v[e], kGeluTanh);
      break;
    case kSilu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_value<FAST>(v[e], kSilu);
      break;
    default: break;
  }
}

// g[e] *= act'(x[e])
template <bool FAST, int N>
__device__ __forceinline__ void act_slopes(float (&g)[N], const float (&x)[N], int act) {
  switch (act) {
    case kRelu:
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] *= act_slope<FAST>(x[e], kRelu);
      break;
    case kGelu:
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] *= act_slope<FAST>(x[e], kGelu);
      break;
    case kGeluTanh:
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] *= act_slope<FAST>(x[e], kGeluTanh);
      break;
    case kSilu:
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] *= act_slope<FAST>(x[e], kSilu);
      break;
    default: break;
  }
}

// ---- 8-bit checkpoints
//
// A group of 64 columns of a row: amax = max |x|, scale = amax / 127 and q =
// rint(x (127 / amax)), which stands for q scale.  A group with a NaN or an
// infinity has scale NaN and q 0, so that all of it reads NaN; one whose amax
// is below 2^-100 (where 127 / amax nears the end of float32) has scale 0.
// Both quotients are correctly rounded: the integers and scales are the
// same ones wherever they are computed.
struct Scale {
  float inv, scale;
};
__device__ __forceinline__ Scale scale_of(uint32_t amax_bits) {
  Scale s;
  const float amax = __uint_as_float(amax_bits);
  const bool some = amax >= 0x1p-100f && amax_bits < 0x7f800000u;
  s.inv = some ? 127.f / amax : 0.f;
  // amax / 127: one correction of the product with the reciprocal rounds it
  // correctly (checked over all significands)
  constexpr float kInv = 1.f / 127.f;
  const float q0 = amax * kInv, q = fmaf(fmaf(-q0, 127.f, amax), kInv, q0);
  s.scale = some ? q : (amax_bits < 0x7f800000u ? 0.f : __uint_as_float(0x7fc00000u));
  return s;
}

// max |x| as bits, a NaN above infinity above the finite values.  (The
// maximum that passes NaN on is one instruction for two values on gfx950.)
template <int N>
__device__ __forceinline__ uint32_t amax_bits(const float (&v)[N]) {
  float m = fabsf(v[0]);
#pragma unroll
  for (int e = 1; e < N; ++e) m = __builtin_elementwise_maximum(m, fabsf(v[e]));
  return __float_as_uint(m) & 0x7fffffffu;
}

// The largest over eight consecutive lanes (a multiple of eight on), in all of them.
__device__ __forceinline__ uint32_t max8(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));   // quad_perm [1, 0, 3, 2]
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));   // quad_perm [2, 3, 0, 1]
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, true));  // row_half_mirror
  return m;
}

// Eight integers as two words.  Adding 1.5 x 2^23 rounds to the nearest
// integer, ties to even, and leaves it in the sum's low byte.  (A group that is
// not finite or is too small has inv 0 and products 0 or NaN: its integers are 0.)
// The product is rounded before: ties of bfloat16 values depend on it.
__device__ __forceinline__ uint2 round8(const float (&v)[8], const Scale& s) {
#pragma clang fp contract(off)
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = v[e] * s.inv;
    b[e] = __float_as_uint(p + 12582912.f);
  }
  auto four = [&](int e) __attribute__((always_inline)) {
    const uint32_t lo = __builtin_amdgcn_perm(b[e + 1], b[e], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[e + 3], b[e + 2], 0x04000c0cu);
    return s.inv != 0.f ? lo | hi : 0u;
  };
  return make_uint2(four(0), four(4));
}

// A scale as it is read.  Of float32's largest value amax / 127 is rounded up, and
// 127 of it would be infinite: the scale below stands in, 2^-24 smaller.
__device__ __forceinline__ float scale_read(float scale) {
  constexpr float kLast = 0x1.020406p+121f;            // the largest whose 127 is finite
  return __builtin_elementwise_minimum(scale, kLast);  // (NaN stays)
}

// q scale for byte e of a word of integers, rounded once.  (As (q + 128) scale - 128 scale, for the
// conversion of unsigned bytes, it overflows in the top 127th of float32's range.)
__device__ __forceinline__ float unround(uint32_t word, int e, float scale) {
  return (float)(int8_t)(word >> (8 * e)) * scale;
}
__device__ __forceinline__ void unround8(uint2 w, float scale, float (&v)[8]) {
  const uint32_t u[2] = {w.x, w.y};
  const float s = scale_read(scale);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = unround(u[e >> 2], e & 3, s);
}

}  // namespace rows
}  // namespace o1d
