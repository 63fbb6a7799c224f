// Matrix products of rows with an epilogue, on the matrix cores (included by
// o1d_mm_*.hip; the host plan is in o1d_mm.hip).
//
//   C[m][n] = sum_k A[m][k] B[n][k]
//   kFwd    A = x  [m][k], B = W  [n][k]   C = y:  + bias, (saved), activation, + residual
//   kDgrad  A = dy [m][k], B = W  [k][n]   C = dx: * act'(pre)
//   kWgrad  A = dy [k][m], B = x  [k][n]   C = dW: float32 partials per piece of k; db = sum_k A
//
// A workgroup of four waves (WM x WN of them, each 32 TM x 32 TN) stages 128
// bytes of k of its rows in LDS per step; the next step's loads are in flight
// during a step's products.  An operand that is contiguous along k lies in LDS
// as rows of k (144 bytes apart: 16-byte accesses without conflicts), one
// that is contiguous along its rows as it is in memory; from the latter float32
// fragments are read as single words and bfloat16 ones with the transposing
// 8-byte read.  Both types multiply on v_mfma_f32_32x32x16_bf16 and accumulate
// in float32.
//
// float32 operands are staged as three bfloat16 pieces, x = x1 + x2 + x3 with
// x1 the nearest bfloat16 to x, x2 that to x - x1 and x3 the rest: 24 bits, all
// of a float32's.  x y is summed as x1 y1 + x1 y2 + x2 y1 + x2 y2 + x1 y3 + x3 y1,
// six exact products; the ones left out, x2 y3 + x3 y2 and x3 y3, are below 2^-24 |x y| (at
// most 2^-8 and 2^-17 of x and y, as for 1 + 2^-8 - 2^-17), which is float32's own rounding of a
// product.  The six take 3/8 of the time of the float32 instruction, and
// sixteen products enter each rounding of the sum instead of two: measured against
// 64 bits the results are no further off.  Pieces are multiples of 2^-133, bfloat16's
// smallest value, which the instruction keeps: operands below 2^-110 are rounded to that.
//
// B's fragment is the instruction's first operand, so that a lane holds four
// consecutive columns n of one row m, and the other half-wave the next four:
// one swap between the halves gives every lane runs of eight columns, on which
// the epilogue works with 16-byte accesses; two lanes have the 64 columns that
// share a scale in an 8-bit checkpoint.  (Through LDS, with whole lines per
// store, the epilogue was bound by LDS and the group's maxima.)
//
// Measured: float32 4096 x 2048 -> 2048 189 to 213 us: 161 to 182 TFLOP/s of float32, of
// bfloat16 products 0.97 to 1.09 PFLOP/s (the library's own float32 product 147 TFLOP/s, its
// largest bfloat16 ones 1.28 PFLOP/s).  Next to the products' matrix instructions stand
// the pieces (6.5 vector instructions per element staged, hence the large tiles) and LDS;
// where a wave has few steps, the first loads and the epilogue.  bfloat16 products of rows
// that are not whole aligned runs come here, both operands through registers, one
// step ahead.  9409 x 203 -> 509 with residual and pre-activation 18.4 to 19.1 us, the most of what
// it loses by the three matrices of 509 columns, whose rows share cache lines: into 512 15.9, of
// 208 and into 512 (o1d_mmf_kernels.h) 14.5.
//
// Widths need not be multiples of anything: a 16-byte run past a row's end is
// loaded from the row's last 16 bytes and moved to its place, k past the end is
// cleared in both operands (so that no infinity or NaN of a repeated element
// meets a zero), and rows past the end repeat the last row and are not stored.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "o1d_rows.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

constexpr int kMmThreads = 256;

template <typename T>
struct Fmt {
  static constexpr int V = 16 / (int)sizeof(T);
  static constexpr int BK = kStepBytes / (int)sizeof(T);
  static constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;  // bfloat16 pieces of an element
  static constexpr int kFrags = BK / 16;                  // fragments of 16 k in a step
};

// The three pieces of four float32, two words each.  A value that is not
// finite is (+-1, 0, itself): only the third piece meets every other operand
// once (times its first piece, which is 0 only if that operand is below 2^-134), so that the
// sum is what float32 products give: infinite with its sign, or NaN.
__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {
  return (uint32_t)from_f32<uint16_t>(a) | (uint32_t)from_f32<uint16_t>(b) << 16;
}
// (`odd` becomes NaN where a value is not finite or rounds to infinity: then
// split_any has to make the pieces.)
__device__ __forceinline__ void split4(const u32x4& w, uint2 (&p)[3], float& odd) {
  uint32_t words[3][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float a = __uint_as_float(w[2 * i]), b = __uint_as_float(w[2 * i + 1]);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      words[k][i] = pair_bf16(a, b);
      if (k == 2) break;
      a -= __uint_as_float(words[k][i] << 16);
      b -= __uint_as_float(words[k][i] & 0xffff0000u);
    }
    odd += a;
    odd += b;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) p[k] = make_uint2(words[k][0], words[k][1]);
}
__device__ __forceinline__ void split_any(const u32x4& w, uint2 (&p)[3]) {
  float none = 0.f;
  split4(w, p, none);
  uint32_t words[3][2];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    words[k][0] = p[k].x;
    words[k][1] = p[k].y;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bits = w[e];
    if ((bits & 0x7fffffffu) < 0x7f7f8000u) continue;
    uint32_t h[3];
    if ((bits & 0x7fffffffu) >= 0x7f800000u) {
      h[0] = 0x3f80u | (bits >> 16 & 0x8000u);
      h[1] = 0u;
      h[2] = bits >> 16 | ((bits & 0x7fffffffu) > 0x7f800000u ? 0x40u : 0u);
    } else {
      float x = __uint_as_float(bits);
      h[0] = bits >> 16;  // rounded towards zero
      x -= __uint_as_float(h[0] << 16);
      h[1] = from_f32<uint16_t>(x);
      x -= __uint_as_float(h[1] << 16);
      h[2] = from_f32<uint16_t>(x);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
      words[k][e / 2] = e % 2 ? (words[k][e / 2] & 0xffffu) | h[k] << 16 : (words[k][e / 2] & 0xffff0000u) | h[k];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) p[k] = make_uint2(words[k][0], words[k][1]);
}

template <typename T>
struct Frag {
  u32x4 p[Fmt<T>::kPieces];
};

// Moves a run down by `shift` elements (0 .. V; zeros come in from above).
template <typename T>
__device__ __forceinline__ void move_down(u32x4& w, int shift) {
  if constexpr (sizeof(T) == 2) {
    if (shift & 1) {
      w[0] = (w[0] >> 16) | (w[1] << 16);
      w[1] = (w[1] >> 16) | (w[2] << 16);
      w[2] = (w[2] >> 16) | (w[3] << 16);
      w[3] = w[3] >> 16;
    }
  }
  const int words = shift * (int)sizeof(T) / 4;
  if (words & 1) w = u32x4{w[1], w[2], w[3], 0u};
  if (words & 2) w = u32x4{w[2], w[3], 0u, 0u};
  if (words & 4) w = u32x4{0u, 0u, 0u, 0u};
}

// One operand's tile: R rows x a step of k.  KC: contiguous along k.
template <typename T, int R, bool KC>
struct Tile {
  static constexpr int V = Fmt<T>::V, BK = Fmt<T>::BK;
  static constexpr int N = R / 32;                               // runs of a thread
  static constexpr int kPieces = Fmt<T>::kPieces;
  static constexpr int kRunsPerRow = R / V;                      // (not KC)
  // LDS, of each piece: KC: rows of k, 16 bytes more apart than they hold (an
  // odd number of 16 bytes); else rows of R, 64 bytes modulo 128 apart, so that
  // the transposing read's four k lie in different banks
  static constexpr int kPitch = KC ? BK * 2 + 16 : R * 2 + (R * 2 % 128 == 0 ? 64 : 0);
  static constexpr int kPiece = (KC ? R : BK) * kPitch;
  static constexpr int kBytes = kPieces * kPiece;
  u32x4 w[N];

  static __device__ __forceinline__ int k_of(int i) { return ((int)threadIdx.x + kMmThreads * i) / kRunsPerRow; }
  static __device__ __forceinline__ int r_of(int i) {
    if constexpr (kMmThreads % kRunsPerRow == 0) return (int)threadIdx.x % kRunsPerRow * V;
    return ((int)threadIdx.x + kMmThreads * i) % kRunsPerRow * V;
  }

  // rows r0 .. of `rows`, k from k0 on of K
  __device__ __forceinline__ void load(const T* p, long long ld, int r0, int rows, int k0, int K) {
    if constexpr (KC) {
      const char* base = reinterpret_cast<const char*>(p + (long long)r0 * ld);
      const int k = k0 + (int)(threadIdx.x % 8) * V;
      if (K >= V) {
        const uint32_t from = (uint32_t)min(k, K - V);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t r = (uint32_t)min((int)threadIdx.x / 8 + 32 * i, rows - 1 - r0);
          __builtin_memcpy(&w[i], base + (r * (uint32_t)ld + from) * (uint32_t)sizeof(T), 16);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t r = (uint32_t)min((int)threadIdx.x / 8 + 32 * i, rows - 1 - r0);
          T t[V] = {};
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (k + e < K) t[e] = p[(long long)(r0 + (int)r) * ld + k + e];
          __builtin_memcpy(&w[i], t, 16);
        }
      }
    } else {
      const char* base = reinterpret_cast<const char*>(p + (long long)k0 * ld);
      if (rows >= V) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t from = (uint32_t)min(r0 + r_of(i), rows - V);
          const uint32_t k = (uint32_t)min(k_of(i), K - 1 - k0);
          __builtin_memcpy(&w[i], base + (k * (uint32_t)ld + from) * (uint32_t)sizeof(T), 16);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int k = min(k_of(i), K - 1 - k0), r = r0 + r_of(i);
          T t[V] = {};
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (r + e < rows) t[e] = p[(long long)(k0 + k) * ld + r + e];
          __builtin_memcpy(&w[i], t, 16);
        }
      }
    }
  }

  // The same places of an 8-bit checkpoint: the integers of a run and its scale.
  __device__ __forceinline__ void load_held(const int8_t* q, const float* scale, long long ldq, int groups, int r0, int k0,
                                            int K) {
    static_assert(!KC, "checkpoints lie along their rows");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const long long k = k0 + min(k_of(i), K - 1 - k0);
      const int r = r0 + r_of(i) < ldq ? r0 + r_of(i) : 0;  // (columns past the end are not stored)
      uint32_t t[2] = {0u, 0u};
      __builtin_memcpy(t, __builtin_assume_aligned(q + k * ldq + r, V), V);
      w[i] = u32x4{t[0], t[1], __float_as_uint(scale[k * groups + r / kGroup]), 0u};
    }
  }
  // Makes the operand act(x) from what was loaded (k past the end: from zeros, which every activation keeps).  In
  // bfloat16 it is rounded to one piece, as the forward's product was given it: what it loses puts the gradient as far from
  // 64 bits as its own rounding does (50176 x 768 -> 192 from a checkpoint with GELU: 2.4e-3 in all, of which 1.7e-3 is its
  // rounding).  As two pieces and two products the 1.7e-3 are left, at 1.2 to 1.8 times the time: 60 -> 74 us there,
  // 8192 x 2048 -> 2048, whose operand comes from a pass of its own, 102 -> 179.
  __device__ __forceinline__ void make(bool held, int act) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float v[V];
      if (held) {
        const float scale = scale_read(__uint_as_float(w[i][2]));
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = unround(w[i][e / 4], e & 3, scale);
      } else {
        T t[V];
        __builtin_memcpy(t, &w[i], 16);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = to_f32(t[e]);
      }
      act_values<sizeof(T) == 2>(v, act);
      T t[V];
#pragma unroll
      for (int e = 0; e < V; ++e) t[e] = from_f32<T>(v[e]);
      __builtin_memcpy(&w[i], t, 16);
    }
  }

  // Puts runs past the end in their places and clears k past the end.
  // (held: the runs are in their places)
  __device__ __forceinline__ void place(int r0, int rows, int k0, int K, bool held = false) {
    if constexpr (KC) {
      if (k0 + BK <= K || K < V) return;
      const int k = k0 + (int)(threadIdx.x % 8) * V, shift = min(V, max(0, k + V - K));
#pragma unroll
      for (int i = 0; i < N; ++i) move_down<T>(w[i], shift);
    } else {
      if (!held && r0 + R > rows && rows >= V) {
#pragma unroll
        for (int i = 0; i < N; ++i) move_down<T>(w[i], min(V, max(0, r0 + r_of(i) + V - rows)));
      }
      if (k0 + BK > K) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (k0 + k_of(i) >= K) w[i] = u32x4{0u, 0u, 0u, 0u};
      }
    }
  }

  static __device__ __forceinline__ int place_of(int i) {
    return KC ? ((int)threadIdx.x / 8 + 32 * i) * kPitch + (int)(threadIdx.x % 8) * V * 2 : k_of(i) * kPitch + r_of(i) * 2;
  }
  __device__ __forceinline__ void store(char* lds) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + place_of(i)) = w[i];
    } else {
      uint2 p[3];
      float odd = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        split4(w[i], p, odd);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(lds + place_of(i) + k * kPiece) = p[k];
      }
      if (odd != odd) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          split_any(w[i], p);
#pragma unroll
          for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(lds + place_of(i) + k * kPiece) = p[k];
        }
      }
    }
  }

  // Fragment j (16 k of the step) of the 32 rows from `row` on: half-wave h has
  // k 8 (2 j + h) + 0 .. 7.
  static __device__ __forceinline__ Frag<T> frag(const char* lds, int row, int j) {
    const int l = threadIdx.x & 63;
    Frag<T> f;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      if constexpr (KC) {
        f.p[k] = *reinterpret_cast<const u32x4*>(lds + k * kPiece + (row + (l & 31)) * kPitch + (2 * j + (l >> 5)) * 16);
      } else {
        // sixteen lanes read 4 k x 16 rows, four consecutive rows each, and get
        // one row's four k each
        const int g = l >> 4, i = l & 15;
        const char* at =
            lds + k * kPiece + (8 * (2 * j + (g >> 1)) + (i >> 2)) * kPitch + (row + 16 * (g & 1) + 4 * (i & 3)) * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * kPitch));
        __builtin_memcpy(&f.p[k], &lo, 8);
        __builtin_memcpy(reinterpret_cast<char*>(&f.p[k]) + 8, &hi, 8);
      }
    }
    return f;
  }
};

// acc[i][k] += m fragment i times n fragment k.  (The pieces' products outermost:
// consecutive instructions have different sums.)
template <typename T, int TM, int TN>
__device__ __forceinline__ void products(const Frag<T> (&n)[TN], const Frag<T> (&m)[TM], f32x16 (&acc)[TM][TN]) {
  auto add = [&](int a, int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int k = 0; k < TN; ++k)
        acc[i][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, n[k].p[a]),
                                                            __builtin_bit_cast(bf16x8, m[i].p[b]), acc[i][k], 0, 0, 0);
  };
  if constexpr (sizeof(T) == 4) {  // the small ones first
    add(2, 0);
    add(0, 2);
    add(1, 1);
    add(1, 0);
    add(0, 1);
  }
  add(0, 0);
}

// Sum of a fragment's elements.
template <typename T>
__device__ __forceinline__ float add_frag(const Frag<T>& f, float s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    auto lo = [&](int k) __attribute__((always_inline)) { return __uint_as_float(f.p[k][i] << 16); };
    auto hi = [&](int k) __attribute__((always_inline)) { return __uint_as_float(f.p[k][i] & 0xffff0000u); };
    if constexpr (sizeof(T) == 4) {  // (the pieces' sum is the element)
      s += (lo(0) + lo(1)) + lo(2);
      s += (hi(0) + hi(1)) + hi(2);
    } else {
      s += lo(0);
      s += hi(0);
    }
  }
  return s;
}

// The epilogue of eight columns n .. n + 7 of a row m: what it reads besides the
// products is loaded ahead of them, for all runs that a lane has in a row
// (`Ahead`), so that one wait covers them.  WHOLE: the tile lies inside the output.
template <typename T, int KIND, bool WHOLE>
struct Ahead {
  // residual (forward) or pre (input gradient), or the latter's checkpoint in the same registers: its
  // integers and their scale
  uint32_t w[2 * sizeof(T)];

  __device__ __forceinline__ void values(float (&v)[8]) const {
    T e[8];
    __builtin_memcpy(e, w, sizeof(e));
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = to_f32(e[k]);
  }
  __device__ __forceinline__ void load(const MmParams& P, int m, int n) {
    if constexpr (KIND == kFwd) {
      if (P.res) run(static_cast<const T*>(P.res) + (long long)m * P.ldres + n, P.N - n, m < P.M);
    } else {
      if (P.act == kNone) return;
      if (P.q) {
        if (WHOLE || (m < P.M && n < P.N)) {
          const uint2 q = *reinterpret_cast<const uint2*>(P.q + (long long)m * P.ldq + n);
          w[0] = q.x;
          w[1] = q.y;
          w[2] = __float_as_uint(P.scale[(long long)m * P.groups + n / kGroup]);
        }
      } else {
        run(static_cast<const T*>(P.pre) + (long long)m * P.ldpre + n, P.N - n, m < P.M);
      }
    }
  }
  __device__ __forceinline__ void run(const T* p, int left, bool in) {
    if (WHOLE || (in && left >= 8)) {
      __builtin_memcpy(w, p, sizeof(w));
    } else if (in) {
      T e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = k < left ? p[k] : T(0);
      __builtin_memcpy(w, e, sizeof(w));
    }
  }
};

template <typename T, bool WHOLE>
__device__ __forceinline__ void put(T* p, int left, const float (&v)[8]) {
  if constexpr (WHOLE)
    store_run(p, v);
  else
    store_some(p, left, v);
}

template <typename T, int KIND, bool WHOLE>
__device__ __forceinline__ void finish(const MmParams& P, int m, int n, const Ahead<T, KIND, WHOLE>& a, float (&v)[8]) {
  constexpr bool kFast = sizeof(T) == 2;
  const int left = P.N - n;
  if (!WHOLE && (m >= P.M || left <= 0)) return;
  if constexpr (KIND == kFwd) {
    if (P.pre) put<T, WHOLE>(static_cast<T*>(P.pre) + (long long)m * P.ldpre + n, left, v);
    act_values<kFast>(v, P.act);
    if (P.res) {
      float r[8];
      a.values(r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    put<T, WHOLE>(static_cast<T*>(P.out) + (long long)m * P.ldo + n, left, v);
  } else if constexpr (KIND == kDgrad) {
    if (P.act != kNone) {
      float x[8];
      if (P.q) {
        unround8(make_uint2(a.w[0], a.w[1]), __uint_as_float(a.w[2]), x);
      } else {
        a.values(x);
      }
      act_slopes<kFast>(v, x, P.act);
    }
    put<T, WHOLE>(static_cast<T*>(P.out) + (long long)m * P.ldo + n, left, v);
  }
}

// a's lanes 32 .. 63 for b's lanes 0 .. 31
__device__ __forceinline__ void swap_halves(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}

template <typename T, int KIND, int SHAPE>
struct Geo {
  static constexpr Shape S = kShapes[SHAPE];
  static constexpr int BM = 32 * S.tm * S.wm, BN = 32 * S.tn * S.wn;
  using TA = Tile<T, BM, KIND != kWgrad>;
  using TB = Tile<T, BN, KIND == kFwd>;
  static constexpr int kTiles = S.tm * S.tn;  // of 32 x 32, 16 registers each, of a wave
  // float32 in narrow tiles: a step's loads and pieces are most of the registers
  // (three steps in 128 of them: 176 bytes of scratch, up to 1.8 times the time).
  static constexpr bool kNarrow32 = (SHAPE == k128x32 || SHAPE == k32x128) && sizeof(T) == 4;
  // Steps whose loads are on their way (each takes a quarter to a half of the
  // accumulators' registers; where that costs a resident wave, one step).
  static constexpr int kDepth = kNarrow32 ? 2 : (kTiles == 1 ? 3 : (SHAPE == k128x128 ? 2 : 1));
  // waves per SIMD that the accumulators leave room for
  static constexpr int kWaves =
      kTiles == 1 && !kNarrow32 ? 4 : (kTiles <= 2 || (kTiles == 3 && sizeof(T) == 2) ? 3 : 2);
  static constexpr int kLds = TA::kBytes + TB::kBytes;
};

// db[m] of a piece.
template <typename T>
__device__ __forceinline__ void put_db(const MmParams& P, int split, int m, float s) {
  if (P.nsplit == 1)
    static_cast<T*>(P.db)[m] = from_f32<T>(s);
  else
    P.part[(long long)split * ((long long)P.M * P.N + P.M) + (long long)P.M * P.N + m] = s;
}

// The wave's tile, 32 rows x 32 or (of a 64-column group) 64 columns at a time.
// first(): called before the first store.
template <typename T, int KIND, bool WHOLE, int TM, int TN, class F>
__device__ __forceinline__ void epilogue(const MmParams& P, int m0, int n0, int split, const f32x16 (&acc)[TM][TN],
                                         F&& first) {
  constexpr int NB = TN % 2 ? 1 : 2, NR = 2 * NB;  // blocks and (a lane's) runs of eight columns at a time
  const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
  for (int c = 0; c < TN / NB; ++c) {
    const int n = n0 + 32 * NB * c + 8 * half;
    T bias[NR][8];
    const bool biased = KIND == kFwd && P.bias;
    if (biased) {
#pragma unroll
      for (int q = 0; q < NR; ++q) {
        const T* p = static_cast<const T*>(P.bias) + n + 16 * q;
        if (WHOLE || n + 16 * q + 8 <= P.N) {
          __builtin_memcpy(bias[q], p, sizeof(bias[q]));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) bias[q][e] = n + 16 * q + e < P.N ? p[e] : T(0);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = m0 + 32 * i + (lane & 31);
      Ahead<T, KIND, WHOLE> ahead[NR];
      if constexpr (KIND != kWgrad) {
#pragma unroll
        for (int q = 0; q < NR; ++q) ahead[q].load(P, m, n + 16 * q);
      }
      float v[NR][8];
#pragma unroll
      for (int q = 0; q < NR; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[q][e] = acc[i][NB * c + q / 2][8 * (q % 2) + e];
          v[q][4 + e] = acc[i][NB * c + q / 2][8 * (q % 2) + 4 + e];
          swap_halves(v[q][e], v[q][4 + e]);
        }
      if (biased) {
#pragma unroll
        for (int q = 0; q < NR; ++q)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[q][e] += to_f32(bias[q][e]);
      }
      if (c == 0 && i == 0) first();
      if constexpr (KIND == kFwd && NB == 2) {
        if (P.q) {  // (all lanes take part, in range or not)
          uint32_t most = 0;
          if constexpr (!WHOLE) {
#pragma unroll
            for (int q = 0; q < NR; ++q)
#pragma unroll
              for (int e = 0; e < 8; ++e) v[q][e] = n + 16 * q + e < P.N ? v[q][e] : 0.f;
          }
#pragma unroll
          for (int q = 0; q < NR; ++q) most = max(most, amax_bits(v[q]));
          const auto both = __builtin_amdgcn_permlane32_swap(most, most, false, false);
          const Scale s = scale_of(max((uint32_t)both[0], (uint32_t)both[1]));
#pragma unroll
          for (int q = 0; q < NR; ++q)
            if (WHOLE || (m < P.M && n + 16 * q < P.ldq))
              *reinterpret_cast<uint2*>(P.q + (long long)m * P.ldq + n + 16 * q) = round8(v[q], s);
          if (half == 0 && (WHOLE || (m < P.M && n < P.N))) P.scale[(long long)m * P.groups + n / kGroup] = s.scale;
        }
      }
#pragma unroll
      for (int q = 0; q < NR; ++q) {
        if constexpr (KIND == kWgrad) {
          const int at = n + 16 * q;
          if (WHOLE || (m < P.M && at < P.N)) {
            if (P.nsplit == 1)
              put<T, WHOLE>(static_cast<T*>(P.out) + (long long)m * P.N + at, P.N - at, v[q]);
            else
              put<float, WHOLE>(P.part + (long long)split * ((long long)P.M * P.N + P.M) + (long long)m * P.N + at,
                                P.N - at, v[q]);
          }
        } else {
          finish<T, KIND, WHOLE>(P, m, n + 16 * q, ahead[q], v[q]);
        }
      }
    }
  }
}

// MADE (weight gradient): B is act(x), made from x or its checkpoint as it is staged.
template <typename T, int KIND, int SHAPE, bool MADE = false>
__global__ __launch_bounds__(kMmThreads, (Geo<T, KIND, SHAPE>::kWaves)) void mm(MmParams P) {
  using G = Geo<T, KIND, SHAPE>;
  constexpr int TM = G::S.tm, TN = G::S.tn, BK = Fmt<T>::BK;
  extern __shared__ __align__(16) char lds[];
  // consecutive tiles, which share rows of A (weight gradient: the piece of
  // k), on one XCD
  const int per_xcd = (P.nblocks + 7) / 8, id = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (id >= P.nblocks) return;
  const int nt = id % P.tn, rest = id / P.tn, mt = rest % P.tm, split = rest / P.tm;
  const int m0 = mt * G::BM, n0 = nt * G::BN;
  const int s0 = split * P.per, s1 = min(P.steps, s0 + P.per);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / G::S.wn * 32 * TM, wn = wave % G::S.wn * 32 * TN;
  const T *A = static_cast<const T*>(P.a), *B = static_cast<const T*>(P.b);
  // the loads of the next kDepth steps are on their way
  constexpr int D = G::kDepth;
  typename G::TA ta[D];
  typename G::TB tb[D];
  auto load = [&](int d, int s) __attribute__((always_inline)) {
    ta[d].load(A, P.lda, m0, P.M, s * BK, P.K);
    if constexpr (MADE) {
      if (P.bq) {
        tb[d].load_held(P.bq, P.scale, P.ldq, P.groups, n0, s * BK, P.K);
        return;
      }
    }
    tb[d].load(B, P.ldb, n0, P.N, s * BK, P.K);
  };
#pragma unroll
  for (int d = 0; d < D; ++d)
    if (d == 0 || s0 + d < s1) load(d, s0 + d);
  f32x16 acc[TM][TN];
  float dbs[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) dbs[i] = 0.f;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int k = 0; k < TN; ++k)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][k][e] = 0.f;
  const bool sum_a = KIND == kWgrad && P.want_db && nt == 0 && wn == 0;
  for (int first = s0; first < s1; first += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int s = first + d;
      if (s >= s1) break;
      __syncthreads();  // the previous step's fragments are read
      ta[d].place(m0, P.M, s * BK, P.K);
      tb[d].place(n0, P.N, s * BK, P.K, MADE && P.bq);
      if constexpr (MADE) tb[d].make(P.bq, P.act);
      ta[d].store(lds);
      tb[d].store(lds + G::TA::kBytes);
      if (s + D < s1) load(d, s + D);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < Fmt<T>::kFrags; ++j) {
        Frag<T> fm[TM], fn[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) fm[i] = G::TA::frag(lds, wm + 32 * i, j);
#pragma unroll
        for (int i = 0; i < TN; ++i) fn[i] = G::TB::frag(lds + G::TA::kBytes, wn + 32 * i, j);
        if (sum_a) {
#pragma unroll
          for (int i = 0; i < TM; ++i) dbs[i] = add_frag<T>(fm[i], dbs[i]);
        }
        products<T>(fn, fm, acc);
      }
    }
  }
  if constexpr (KIND == kWgrad) {
    if (sum_a) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const float s = dbs[i] + __shfl_xor(dbs[i], 32, 64);
        const int m = m0 + wm + 32 * i + (lane & 31);
        if (lane < 32 && m < P.M) put_db<T>(P, split, m, s);
      }
    }
  }
  if (m0 + G::BM <= P.M && n0 + G::BN <= P.N)
    epilogue<T, KIND, true>(P, m0 + wm, n0 + wn, split, acc, [] {});
  else
    epilogue<T, KIND, false>(P, m0 + wm, n0 + wn, split, acc, [] {});
}

template <typename T, int KIND, int SHAPE, bool MADE = false>
hipError_t launch_shape(const MmPlan& pl, hipStream_t stream) {
  using G = Geo<T, KIND, SHAPE>;
  static std::atomic<int> allowed{0};
  if (!allowed.load(std::memory_order_acquire)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(mm<T, KIND, SHAPE, MADE>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds);
    if (e != hipSuccess) return e;
    allowed.store(1, std::memory_order_release);
  }
  hipLaunchKernelGGL((mm<T, KIND, SHAPE, MADE>), dim3((unsigned)(pl.p.nblocks + 7) / 8 * 8), dim3(kMmThreads), G::kLds, stream,
                     pl.p);
  return hipGetLastError();
}

template <typename T, int KIND, int SHAPE>
hipError_t launch_planned(const MmPlan& pl, hipStream_t stream) {
  if constexpr (shape_used(KIND, (int)sizeof(T), SHAPE)) return launch_shape<T, KIND, SHAPE>(pl, stream);
  return hipErrorInvalidValue;  // (no plan has it)
}

template <typename T, int KIND>
hipError_t launch_kind(const MmPlan& pl, hipStream_t stream) {
  if constexpr (KIND == kWgrad) {
    if (pl.p.made) return pl.shape == k64x64 ? launch_shape<T, KIND, k64x64, true>(pl, stream)
                                             : launch_shape<T, KIND, k192x64, true>(pl, stream);
  }
  switch (pl.shape) {
    case k128x128: return launch_planned<T, KIND, k128x128>(pl, stream);
    case k64x64: return launch_planned<T, KIND, k64x64>(pl, stream);
    case k128x96: return launch_planned<T, KIND, k128x96>(pl, stream);
    case k64x128: return launch_planned<T, KIND, k64x128>(pl, stream);
    case k128x64: return launch_planned<T, KIND, k128x64>(pl, stream);
    case k128x32: return launch_planned<T, KIND, k128x32>(pl, stream);
    case k32x128: return launch_planned<T, KIND, k32x128>(pl, stream);
    case k128x192: return launch_planned<T, KIND, k128x192>(pl, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace
}  // namespace rows
}  // namespace o1d
