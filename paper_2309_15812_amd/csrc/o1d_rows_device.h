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

// ---- activations.  Fast: for results that are rounded to bfloat16.
//
// gelu(x) = x Phi(x), Phi(x) = (1 + erf(x / sqrt 2)) / 2.  erf: the library's
// in float32; for bfloat16 results Abramowitz and Stegun 7.1.26, whose error
// (1.5e-7) is far below their rounding, at a third of the instructions and
// with the exp(-x^2 / 2) that the derivative needs too.
template <bool FAST>
__device__ __forceinline__ float exp_(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST>
__device__ __forceinline__ float recip(float x) { return FAST ? __builtin_amdgcn_rcpf(x) : 1.f / x; }

// Phi(x) and exp(-x^2 / 2)
template <bool FAST>
__device__ __forceinline__ float normal_cdf(float x, float* density) {
  const float z = x * 0.70710678118654752f;
  if constexpr (FAST) {
    const float a = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, a, 1.f)), e = __expf(-a * a);
    float s = fmaf(1.061405429f, t, -1.453152027f);
    s = fmaf(s, t, 1.421413741f);
    s = fmaf(s, t, -0.284496736f);
    s = fmaf(s, t, 0.254829592f);
    const float half = 0.5f * s * t * e;  // (1 - erf |z|) / 2
    *density = e;
    return x < 0.f ? half : 1.f - half;
  } else {
    *density = expf(-z * z);
    return 0.5f * (1.f + erff(z));
  }
}

// gelu(x) ~ x sigma(2 u), u = sqrt(2 / pi) (x + 0.044715 x^3)   [(1 + tanh u) / 2 = sigma(2 u)]
constexpr float kTanhScale = 1.59576912160573071f;  // 2 sqrt(2 / pi)
constexpr float kTanhCube = 0.044715f;

template <bool FAST>
__device__ __forceinline__ float act_value(float x, int act) {
  float d;
  switch (act) {
    case kRelu: return x < 0.f ? 0.f : x;
    case kGelu: return x * normal_cdf<FAST>(x, &d);
    case kGeluTanh: return x * recip<FAST>(1.f + exp_<FAST>(-kTanhScale * (x + kTanhCube * x * x * x)));
    case kSilu: return x * recip<FAST>(1.f + exp_<FAST>(-x));
    default: return x;
  }
}

template <bool FAST>
__device__ __forceinline__ float act_slope(float x, int act) {
  switch (act) {
    case kRelu: return x <= 0.f ? 0.f : 1.f;
    case kGelu: {
      float d;
      const float phi = normal_cdf<FAST>(x, &d);
      return fmaf(x * 0.39894228040143268f, d, phi);
    }
    case kGeluTanh: {
      const float g = recip<FAST>(1.f + exp_<FAST>(-kTanhScale * (x + kTanhCube * x * x * x)));
      return g + x * g * (1.f - g) * kTanhScale * fmaf(3.f * kTanhCube * x, x, 1.f);
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
  s.scale = some ? amax / 127.f : (amax_bits < 0x7f800000u ? 0.f : __uint_as_float(0x7fc00000u));
  return s;
}

// |x| as bits: their unsigned order is that of the values, with NaN above infinity above the finite ones.
template <int N>
__device__ __forceinline__ uint32_t amax_bits(const float (&v)[N]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  return m;
}

// The largest over eight consecutive lanes (a multiple of eight on), in all of them.
__device__ __forceinline__ uint32_t max8(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));   // quad_perm [1, 0, 3, 2]
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));   // quad_perm [2, 3, 0, 1]
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, true));  // row_half_mirror
  return m;
}

// Eight integers as two words.  (A group that is not finite has inv 0 and
// products 0 or NaN: its integers are set to 0.)
__device__ __forceinline__ uint2 round8(const float (&v)[8], const Scale& s) {
  uint32_t w[2] = {0u, 0u};
  if (s.inv != 0.f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)(int)rintf(v[e] * s.inv) & 0xffu) << (8 * (e & 3));
  }
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void unround8(uint2 w, float scale, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3))) * scale;
}

}  // namespace rows
}  // namespace o1d
