// Layer norm over the features of a row, forward and backward (included by
// o1d_ln_f32.hip and o1d_ln_bf16.hip).
//
//   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = (var + eps)^-1/2,  xh = (x - mean) rstd
//   y  = xh w + b
//   dx = rstd (g - mean(g) - xh mean(g xh)),  g = dy w;   dw = sum_rows dy xh,  db = sum_rows dy
//
// Memory bounds both: x once in, y (dx) once out.  A row lies in the registers
// of LPR lanes, CH runs of 16 bytes each, so that the variance is taken of the
// differences from the mean (two passes over registers, one over memory); a
// wave has 64 / LPR rows.  Sums, statistics and the gradients' partial sums are
// float32.  The backward adds dw and db over a workgroup's rows in registers,
// leaves one partial row per workgroup, and col_sum adds those in a fixed order.
//
// Measured: forward 200704 x 96 bfloat16 14.3 us (77 MB in and out, 5.4 TB/s; a large
// copy reaches 5.0 to 6.9 TB/s here); backward 50176 x 192 float32 23.3 us (116 MB,
// 5.0 TB/s) and 3.9 for the sum, 33333 x 211 bfloat16 from a checkpoint 15.0 and 3.9
// (unaligned rows of 422 bytes).  Few rows (49 x 768: 3.5 us) are one wait for memory.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "o1d_rows.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {
namespace {

template <typename T>
constexpr int kRun = 16 / (int)sizeof(T);  // elements of a run

constexpr int kLnWaves = 4;
// Waves of a backward workgroup: eight, so that few workgroups (partial rows of
// dw and db) fill the GPU; with three runs per lane on, registers allow four.
template <int CH>
constexpr int kBwdWaves = ln_bwd_waves(CH);

// Sum over LPR consecutive lanes, in all of them.
template <int LPR>
__device__ __forceinline__ float lanes_sum(float v) {
  auto add = [&](int moved) __attribute__((always_inline)) { v += __int_as_float(moved); };
  add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xF, 0xF, true));
  add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xF, 0xF, true));
  if constexpr (LPR >= 8) add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xF, 0xF, true));  // half rows
  if constexpr (LPR >= 16) add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x140, 0xF, 0xF, true));  // rows
  if constexpr (LPR >= 32) v += __shfl_xor(v, 16, 64);
  if constexpr (LPR >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

// A row over LPR lanes: slot i of lane l is run l + i LPR.  All slots but the
// last are whole; `n` elements of the last slot exist (all, some in the row's
// last run, or none).  Loads are never conditional: a run past the row's end
// is loaded from the row's last 16 bytes, and its elements are moved down to
// their places (by an amount that all rows share).
template <typename T, int LPR, int CH>
struct RowMap {
  static constexpr int V = kRun<T>;
  int at[CH];  // first element of each slot
  int from;    // where the last slot is loaded from
  int n, shift;

  __device__ __forceinline__ explicit RowMap(int C) {
    const int l = threadIdx.x & (LPR - 1);
#pragma unroll
    for (int i = 0; i < CH; ++i) at[i] = (l + i * LPR) * V;
    n = min(V, max(0, C - at[CH - 1]));
    from = min(at[CH - 1], C - V);
    shift = n > 0 ? V - n : 0;
  }

  __device__ __forceinline__ void load_raw(const T* row, int C, uint32_t (&w)[CH][4]) const {
#pragma unroll
    for (int i = 0; i < CH - 1; ++i) __builtin_memcpy(w[i], row + at[i], 16);
    if (C >= V) {
      __builtin_memcpy(w[CH - 1], row + from, 16);
    } else {  // (a row shorter than a run: CH is 1)
      T t[V] = {};
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < n) t[e] = row[e];
      __builtin_memcpy(w[CH - 1], t, 16);
    }
  }

  __device__ __forceinline__ void place(int C, uint32_t (&w)[4]) const {
    if (C % V == 0 || C < V) return;
    if constexpr (sizeof(T) == 2) {
      if (shift & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (w[i] >> 16) | (i < 3 ? w[i + 1] << 16 : 0u);
      }
    }
    const int words = shift * (int)sizeof(T) / 4;
    if (words & 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = i < 3 ? w[i + 1] : 0u;
    }
    if (words & 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = i < 2 ? w[i + 2] : 0u;
    }
  }

  __device__ __forceinline__ void unpack(int C, uint32_t (&w)[CH][4], float (&v)[CH][V]) const {
    place(C, w[CH - 1]);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      T t[V];
      __builtin_memcpy(t, w[i], 16);
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = i < CH - 1 || n > 0 ? to_f32(t[e]) : 0.f;
    }
  }

  __device__ __forceinline__ void load(const T* row, int C, float (&v)[CH][V]) const {
    uint32_t w[CH][4];
    load_raw(row, C, w);
    unpack(C, w, v);
  }

  __device__ __forceinline__ void store(T* row, const float (&v)[CH][V]) const {
#pragma unroll
    for (int i = 0; i < CH - 1; ++i) store_run(row + at[i], v[i]);
    if (n > 0) store_some(row + at[CH - 1], n, v[CH - 1]);
  }

  // The same places of an 8-bit row (padded to 16 bytes: whole runs lie inside it).
  __device__ __forceinline__ void load_held(const int8_t* q, const float* scale, uint32_t (&w)[CH][V / 4],
                                            float (&s)[CH]) const {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int a = i < CH - 1 || n > 0 ? at[i] : 0;
      __builtin_memcpy(w[i], __builtin_assume_aligned(q + a, V), V);
      s[i] = scale[a / kGroup];
    }
  }
  __device__ __forceinline__ void unpack_held(const uint32_t (&w)[CH][V / 4], const float (&s)[CH], float (&v)[CH][V]) const {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const float scale = scale_read(s[i]);
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = i < CH - 1 || e < n ? unround(w[i][e / 4], e & 3, scale) : 0.f;
    }
  }
};

template <typename T, int LPR, int CH>
__global__ __launch_bounds__(64 * kLnWaves) void ln_fwd_rows(LnParams P) {
  constexpr int V = kRun<T>, kRows = 64 / LPR * kLnWaves;
  const RowMap<T, LPR, CH> map(P.C);
  float w[CH][V], b[CH][V];
  map.load(static_cast<const T*>(P.w), P.C, w);
  map.load(static_cast<const T*>(P.b), P.C, b);
  const float inv = 1.f / (float)P.C;
  for (long long row = (long long)blockIdx.x * kRows + threadIdx.x / LPR; row < P.M; row += (long long)gridDim.x * kRows) {
    float x[CH][V];
    map.load(static_cast<const T*>(P.x) + row * P.ldx, P.C, x);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) s += x[i][e];
    // (a quotient, so that rows of one value have exactly that mean)
    const float mean = lanes_sum<LPR>(s) / (float)P.C;
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[i][e] = i < CH - 1 || e < map.n ? x[i][e] - mean : 0.f;
        q = fmaf(x[i][e], x[i][e], q);
      }
    const float rstd = 1.f / sqrtf(lanes_sum<LPR>(q) * inv + P.eps);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) x[i][e] = fmaf(x[i][e] * rstd, w[i][e], b[i][e]);
    map.store(static_cast<T*>(P.y) + row * P.ldy, x);
    if (P.mean && (threadIdx.x & (LPR - 1)) == 0) {
      P.mean[row] = mean;
      P.rstd[row] = rstd;
    }
  }
}

// A row's operands as they are in memory.
template <typename T, int LPR, int CH, bool HELD>
struct BwdRow {
  using Map = RowMap<T, LPR, CH>;
  uint32_t g[CH][4], x[CH][HELD ? kRun<T> / 4 : 4];
  float scale[CH], mean, rstd;

  __device__ __forceinline__ void load(const LnParams& P, const Map& map, long long row, long long ldq, long long groups) {
    map.load_raw(static_cast<const T*>(P.dy) + row * P.ldy, P.C, g);
    if constexpr (HELD)
      map.load_held(P.xq + row * ldq, P.xscale + row * groups, x, scale);
    else
      map.load_raw(static_cast<const T*>(P.x) + row * P.ldx, P.C, x);
    mean = P.mean[row];
    rstd = P.rstd[row];
  }
};

template <typename T, int LPR, int CH, bool HELD>
__global__ __launch_bounds__(64 * kBwdWaves<CH>) void ln_bwd_rows(LnParams P) {
  constexpr int V = kRun<T>, kWaves = kBwdWaves<CH>, kRows = 64 / LPR * kWaves;
  const RowMap<T, LPR, CH> map(P.C);
  float w[CH][V], dw[CH][V], db[CH][V];
  const long long ldq = (P.C + 15) / 16 * 16, groups = (P.C + kGroup - 1) / kGroup;
  const long long stride = (long long)gridDim.x * kRows;
  long long row = (long long)blockIdx.x * kRows + threadIdx.x / LPR;
  BwdRow<T, LPR, CH, HELD> next;
  next.load(P, map, row < P.M ? row : P.M - 1, ldq, groups);
  map.load(static_cast<const T*>(P.w), P.C, w);
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dw[i][e] = db[i][e] = 0.f;
  const float inv = 1.f / (float)P.C;
  for (; row < P.M; row += stride) {
    BwdRow<T, LPR, CH, HELD> now = next;
    next.load(P, map, row + stride < P.M ? row + stride : P.M - 1, ldq, groups);  // during this row's sums
    float x[CH][V], g[CH][V];
    if constexpr (HELD)
      map.unpack_held(now.x, now.scale, x);
    else
      map.unpack(P.C, now.x, x);
    map.unpack(P.C, now.g, g);
    float s = 0.f, sx = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        // (the difference first: x rstd - mean rstd loses what the mean and the spread differ by)
        x[i][e] = (x[i][e] - now.mean) * now.rstd;
        dw[i][e] = fmaf(g[i][e], x[i][e], dw[i][e]);
        db[i][e] += g[i][e];
        g[i][e] *= w[i][e];
        s += g[i][e];
        sx = fmaf(g[i][e], x[i][e], sx);
      }
    s = -lanes_sum<LPR>(s) * inv;
    sx = -lanes_sum<LPR>(sx) * inv;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) x[i][e] = now.rstd * fmaf(x[i][e], sx, g[i][e] + s);
    map.store(static_cast<T*>(P.dx) + row * P.lddx, x);
  }
  // this workgroup's sums: over a wave's rows, then pairs of waves
  __shared__ float sums[kWaves / 2][2][LPR * CH * V];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e)
#pragma unroll
      for (int m = LPR; m < 64; m *= 2) {
        dw[i][e] += __shfl_xor(dw[i][e], m, 64);
        db[i][e] += __shfl_xor(db[i][e], m, 64);
      }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int half = kWaves / 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half && lane < LPR) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sums[wave - half][0][map.at[i] + e] = dw[i][e];
          sums[wave - half][1][map.at[i] + e] = db[i][e];
        }
    }
    __syncthreads();
    if (wave < half && lane < LPR) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dw[i][e] += sums[wave][0][map.at[i] + e];
          db[i][e] += sums[wave][1][map.at[i] + e];
        }
    }
    __syncthreads();
  }
  if (wave == 0 && lane < LPR && gridDim.x == 1) {  // the sums themselves
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (i < CH - 1 || e < map.n) {
          static_cast<T*>(P.dw)[map.at[i] + e] = from_f32<T>(dw[i][e]);
          static_cast<T*>(P.db)[map.at[i] + e] = from_f32<T>(db[i][e]);
        }
  } else if (wave == 0 && lane < LPR) {
    float* part = P.part + (long long)blockIdx.x * 2 * P.C;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (i < CH - 1 || e < map.n) {
          part[map.at[i] + e] = dw[i][e];
          part[P.C + map.at[i] + e] = db[i][e];
        }
  }
}

// ---- rows too long for a wave's registers: a workgroup per row, x read again
// from the caches for each pass.

constexpr int kWide = 256;

__device__ __forceinline__ float block_sum(float v, float* red) {
  v = lanes_sum<64>(v);
  __syncthreads();  // the previous sum is read
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < kWide / 64; ++k) s += red[k];
  return s;
}

template <typename T>
__global__ __launch_bounds__(kWide) void ln_fwd_wide(LnParams P) {
  constexpr int V = kRun<T>;
  __shared__ float red[kWide / 64];
  const float inv = 1.f / (float)P.C;
  const T *w = static_cast<const T*>(P.w), *b = static_cast<const T*>(P.b);
  for (long long row = blockIdx.x; row < P.M; row += gridDim.x) {
    const T* x = static_cast<const T*>(P.x) + row * P.ldx;
    T* y = static_cast<T*>(P.y) + row * P.ldy;
    float s = 0.f, v[V], u[V];
    for (int c = threadIdx.x * V; c < P.C; c += kWide * V) {
      load_some(x + c, P.C - c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) s += v[e];
    }
    const float mean = block_sum(s, red) / (float)P.C;
    float q = 0.f;
    for (int c = threadIdx.x * V; c < P.C; c += kWide * V) {
      load_some(x + c, P.C - c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = c + e < P.C ? v[e] - mean : 0.f;
        q = fmaf(d, d, q);
      }
    }
    const float rstd = 1.f / sqrtf(block_sum(q, red) * inv + P.eps);
    for (int c = threadIdx.x * V; c < P.C; c += kWide * V) {
      float k[V];
      load_some(x + c, P.C - c, v);
      load_some(w + c, P.C - c, u);
      load_some(b + c, P.C - c, k);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = fmaf((v[e] - mean) * rstd, u[e], k[e]);
      store_some(y + c, P.C - c, v);
    }
    if (P.mean && threadIdx.x == 0) {
      P.mean[row] = mean;
      P.rstd[row] = rstd;
    }
  }
}

// A run of x (or of its checkpoint: c is a multiple of the run).
template <typename T, bool HELD>
__device__ __forceinline__ void load_x(const LnParams& P, long long row, int c, float (&v)[kRun<T>]) {
  constexpr int V = kRun<T>;
  if constexpr (HELD) {
    const long long ldq = (P.C + 15) / 16 * 16, groups = (P.C + kGroup - 1) / kGroup;
    uint32_t w[V / 4];
    __builtin_memcpy(w, __builtin_assume_aligned(P.xq + row * ldq + c, V), V);
    const float s = scale_read(P.xscale[row * groups + c / kGroup]);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = unround(w[e / 4], e & 3, s);
  } else {
    load_some(static_cast<const T*>(P.x) + row * P.ldx + c, P.C - c, v);
  }
}

template <typename T, bool HELD>
__global__ __launch_bounds__(kWide) void ln_bwd_wide(LnParams P) {
  constexpr int V = kRun<T>;
  __shared__ float red[kWide / 64];
  const float inv = 1.f / (float)P.C;
  const T* w = static_cast<const T*>(P.w);
  for (long long row = blockIdx.x; row < P.M; row += gridDim.x) {
    const T* dy = static_cast<const T*>(P.dy) + row * P.ldy;
    T* dx = static_cast<T*>(P.dx) + row * P.lddx;
    const float mean = P.mean[row], rstd = P.rstd[row];
    float s = 0.f, sx = 0.f, x[V], g[V], u[V];
    for (int c = threadIdx.x * V; c < P.C; c += kWide * V) {
      load_x<T, HELD>(P, row, c, x);
      load_some(dy + c, P.C - c, g);
      load_some(w + c, P.C - c, u);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s = fmaf(g[e], u[e], s);
        sx = fmaf(g[e] * u[e], (x[e] - mean) * rstd, sx);
      }
    }
    s = block_sum(s, red) * inv;
    sx = block_sum(sx, red) * inv;
    for (int c = threadIdx.x * V; c < P.C; c += kWide * V) {
      load_x<T, HELD>(P, row, c, x);
      load_some(dy + c, P.C - c, g);
      load_some(w + c, P.C - c, u);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = rstd * (g[e] * u[e] - s - (x[e] - mean) * rstd * sx);
      store_some(dx + c, P.C - c, x);
    }
  }
}

// dw and db of long rows: a thread per run of columns, the rows over gridDim.y.
template <typename T, bool HELD>
__global__ __launch_bounds__(kWide) void ln_dw_wide(LnParams P) {
  constexpr int V = kRun<T>;
  const int c = (blockIdx.x * kWide + threadIdx.x) * V;
  if (c >= P.C) return;
  float dw[V] = {}, db[V] = {};
  for (long long row = blockIdx.y; row < P.M; row += gridDim.y) {
    float x[V], g[V];
    load_x<T, HELD>(P, row, c, x);
    load_some(static_cast<const T*>(P.dy) + row * P.ldy + c, P.C - c, g);
    const float mean = P.mean[row], rstd = P.rstd[row];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      dw[e] = fmaf(g[e], (x[e] - mean) * rstd, dw[e]);
      db[e] += g[e];
    }
  }
  float* part = P.part + (long long)blockIdx.y * 2 * P.C;
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (c + e < P.C) {
      part[c + e] = dw[e];
      part[P.C + c + e] = db[e];
    }
}

// Calls f with the forward's lanes and runs per lane (ln_fwd_map).
template <typename T, class F>
bool with_row(int C, F&& f) {
  const LnMap m = ln_fwd_map(C, (int)sizeof(T));
  auto pick = [&](auto lpr) {
    constexpr int L = decltype(lpr)::value;
    switch (m.runs) {
      case 1: if constexpr (L == 4) f(lpr, std::integral_constant<int, 1>{}); break;
      case 2: if constexpr (L == 4) f(lpr, std::integral_constant<int, 2>{}); break;
      case 3: f(lpr, std::integral_constant<int, 3>{}); break;
      case 4: f(lpr, std::integral_constant<int, 4>{}); break;
      case 5: if constexpr (L == 64) f(lpr, std::integral_constant<int, 5>{}); break;
      case 6: if constexpr (L == 64) f(lpr, std::integral_constant<int, 6>{}); break;
      case 7: if constexpr (L == 64) f(lpr, std::integral_constant<int, 7>{}); break;
      case 8: if constexpr (L == 64) f(lpr, std::integral_constant<int, 8>{}); break;
    }
  };
  switch (m.lanes) {
    case 4: pick(std::integral_constant<int, 4>{}); break;
    case 8: pick(std::integral_constant<int, 8>{}); break;
    case 16: pick(std::integral_constant<int, 16>{}); break;
    case 32: pick(std::integral_constant<int, 32>{}); break;
    case 64: pick(std::integral_constant<int, 64>{}); break;
    default: return false;
  }
  return true;
}

template <typename T>
hipError_t ln_fwd_t(const LnParams& p, hipStream_t stream) {
  const bool done = with_row<T>(p.C, [&](auto lpr, auto ch) {
    constexpr int L = decltype(lpr)::value, CH = decltype(ch)::value, R = 64 / L * kLnWaves;
    const long long blocks = cdiv(p.M, R);
    hipLaunchKernelGGL((ln_fwd_rows<T, L, CH>), dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(64 * kLnWaves), 0,
                       stream, p);
  });
  if (!done)
    hipLaunchKernelGGL((ln_fwd_wide<T>), dim3(p.M < 4096 ? p.M : 4096), dim3(kWide), 0, stream, p);
  return hipGetLastError();
}

// Calls f with the backward's lanes and runs per lane (ln_bwd_map).
template <typename T, class F>
bool with_bwd_row(int C, F&& f) {
  const LnMap m = ln_bwd_map(C, (int)sizeof(T));
  auto pick = [&](auto lpr) {
    constexpr int L = decltype(lpr)::value;
    switch (m.runs) {
      case 1: f(lpr, std::integral_constant<int, 1>{}); break;
      case 2: f(lpr, std::integral_constant<int, 2>{}); break;
      case 3: f(lpr, std::integral_constant<int, 3>{}); break;
      case 4: if constexpr (L == 64) f(lpr, std::integral_constant<int, 4>{}); break;
      case 5: if constexpr (L == 64) f(lpr, std::integral_constant<int, 5>{}); break;
      case 6: if constexpr (L == 64) f(lpr, std::integral_constant<int, 6>{}); break;
      case 7: if constexpr (L == 64) f(lpr, std::integral_constant<int, 7>{}); break;
      case 8: if constexpr (L == 64) f(lpr, std::integral_constant<int, 8>{}); break;
    }
  };
  switch (m.lanes) {
    case 4: pick(std::integral_constant<int, 4>{}); break;
    case 8: pick(std::integral_constant<int, 8>{}); break;
    case 16: pick(std::integral_constant<int, 16>{}); break;
    case 32: pick(std::integral_constant<int, 32>{}); break;
    case 64: pick(std::integral_constant<int, 64>{}); break;
    default: return false;
  }
  return true;
}

template <typename T, bool HELD>
hipError_t ln_bwd_held(const LnParams& p, hipStream_t stream) {
  const bool done = with_bwd_row<T>(p.C, [&](auto lpr, auto ch) {
    constexpr int L = decltype(lpr)::value, CH = decltype(ch)::value;
    hipLaunchKernelGGL((ln_bwd_rows<T, L, CH, HELD>), dim3(p.blocks), dim3(64 * kBwdWaves<CH>), 0, stream, p);
  });
  if (!done) {
    hipLaunchKernelGGL((ln_bwd_wide<T, HELD>), dim3(p.M < 4096 ? p.M : 4096), dim3(kWide), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ln_dw_wide<T, HELD>), dim3((unsigned)cdiv(p.C, (long long)kWide * kRun<T>), p.blocks), dim3(kWide),
                       0, stream, p);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t ln_bwd_t(const LnParams& p, hipStream_t stream) {
  return p.xq ? ln_bwd_held<T, true>(p, stream) : ln_bwd_held<T, false>(p, stream);
}

}  // namespace
}  // namespace rows
}  // namespace o1d
