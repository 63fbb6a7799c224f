// Group norm with an activation, channels last, forward and backward (included by
// o1d_gn_f32.hip and o1d_gn_bf16.hip).
//
//   over the n = P D values of a sample's group:  mean = sum x / n,  var = sum (x - mean)^2 / n,
//   rstd = (var + eps)^-1/2,  xh = (x - mean) rstd,  h = xh w + b,  y = act(h)
//   dh = dy act'(h),  g = dh w,  dx = rstd (g - mean(g) - xh mean(g xh));  dw = sum dh xh,  db = sum dh
//
// Memory bounds it: x (and dy) once in, y (dx) once out.  A group's channels are
// a short piece of every pixel's row, so a workgroup takes a bundle of groups, whole
// 64-byte pieces of a row where it can, of all pixels of a sample, and keeps them in registers
// from the statistics to the result; the bundles of a sample run on one XCD, whose L2 they share.
// Samples that no workgroup holds are passed twice, in chunks of pixels.
//
// Measured: forward of 64 x 3136 x 96 bfloat16 in 32 groups 25 us, 3.1 TB/s: 28 vector instructions for each value (two passes
// over registers, silu, bfloat16 both ways) keep the vector units 68% busy; with a select in place of each uniform branch,
// sums by LDS and weights applied after rstd 28.6 us.  Backward of 64 x 784 x 192 float32 36 us, 3.2 TB/s, and 4 us for the sums;
// 46 us with the library's exponential and quotient in the activation.  Backward of 3 x 12707 x 203 bfloat16 in
// two passes 18 and 15 us, and 4 between them.
//
// A thread has one 16-byte run of a row's channels in every row that it takes, so its weights
// and statistics stay in registers.  A bundle's last run starts early enough to be whole;
// the elements that it shares with the run before (`skip`) enter no sum.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "o1d_gn.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {
namespace {

template <typename T>
constexpr int kRun = 16 / (int)sizeof(T);

__device__ __forceinline__ float wave_sum(float v) {
  auto add = [&](int moved) __attribute__((always_inline)) { v += __int_as_float(moved); };
  add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xF, 0xF, true));
  add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xF, 0xF, true));
  add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xF, 0xF, true));  // half rows
  add(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x140, 0xF, 0xF, true));  // rows
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// 1 / (1 + exp(-x)) of float32, to about 2^-23 of itself: exp2 of the product's head and, to first order, of its
// rest, and a reciprocal with one correction.  (The library's exponential and quotient are twice as many instructions, which
// bound the float32 backward.)  exp2's argument stays where the sum is finite.
__device__ __forceinline__ float sigma(float x) {
  constexpr float kLog2e = 1.44269502162933349609375f, kRest = 1.925963033500011e-8f, kLn2 = 0.693147180559945309f;
  const float z = fminf(fmaxf(x, -87.f), 87.f);
  const float head = z * -kLog2e, rest = -fmaf(z, kRest, fmaf(z, kLog2e, head));
  float e = __builtin_amdgcn_exp2f(head);
  e = fmaf(e, rest * kLn2, e);
  const float d = 1.f + e, r = __builtin_amdgcn_rcpf(d);
  return fmaf(fmaf(-d, r, 1.f), r, r);
}
// The activations of a run, with that for float32.
template <bool FAST, int N>
__device__ __forceinline__ void gn_values(float (&v)[N], int act) {
  if (!FAST && act == kSilu) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = v[e] < -87.f ? act_value<false>(v[e], kSilu) : v[e] * sigma(v[e]);
  } else {
    act_values<FAST>(v, act);
  }
}
template <bool FAST, int N>
__device__ __forceinline__ void gn_slopes_of(float (&g)[N], const float (&h)[N], int act) {
  if (!FAST && act == kSilu) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float s = sigma(h[e]);
      g[e] *= h[e] < -87.f ? act_slope<false>(h[e], kSilu) : s * fmaf(h[e], 1.f - s, 1.f);
    }
  } else {
    act_slopes<FAST>(g, h, act);
  }
}

// i / D, for the i below 2^16 that occur: the high half of the product with 2^32 / D rounded up.  (A quotient by an
// unknown divisor is 30 instructions, and every thread has one for each channel of its run.)
__device__ __forceinline__ int by_d(const GnParams& P, int i) { return P.D == 1 ? i : (int)__umulhi((uint32_t)i, P.over_d); }

// A thread's place: its run of channels and its first row; and the bundle's.
template <typename T, int THREADS>
struct GnAt {
  static constexpr int V = kRun<T>;
  int n, c0, CB, g0, groups;  // sample, first channel, channels, first group and groups of the bundle
  int runs, slots, slot;      // runs of a row, rows at a time, this thread's
  int s, skip, left;          // first channel of the run within the bundle (may be negative), elements to leave
                              // out, elements there are (fewer than V only where C is)
  bool active;

  __device__ __forceinline__ void place(const GnParams& P, int sample, int bundle) {
    n = sample;
    g0 = bundle * P.gb;
    groups = min(P.gb, P.G - g0);
    c0 = g0 * P.D;
    CB = groups * P.D;
    runs = (CB + V - 1) / V;
    slots = THREADS / runs;
    const int run = (int)threadIdx.x % runs;
    slot = (int)threadIdx.x / runs;
    active = slot < slots;
    s = min(run * V, CB - V);
    if (P.C < V) s = 0;
    left = min(V, P.C);
    skip = run * V - s;
  }
  __device__ __forceinline__ bool counts(int e) const { return active && e >= skip && e < left; }
  __device__ __forceinline__ int group(const GnParams& P, int e) const {
    return by_d(P, min(max(s + e, 0), CB - 1));  // (within the bundle)
  }
  // A row's run: 16 bytes, or the few channels there are.
  template <typename U>
  __device__ __forceinline__ void load(const U* row, uint32_t (&w)[4]) const {
    if (left == V) {
      __builtin_memcpy(w, row + c0 + s, 16);
    } else {
      U t[V] = {};
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < left) t[e] = row[e];
      __builtin_memcpy(w, t, 16);
    }
  }
  // (A run that starts in the bundle is stored whole: the elements it shares with the one
  // before have the same values there.)
  __device__ __forceinline__ void store(T* row, const float (&v)[V]) const {
    if (s >= 0 && left == V) {
      store_run(row + c0 + s, v);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e >= skip && e < left) row[c0 + s + e] = from_f32<T>(v[e]);
    }
  }
  __device__ __forceinline__ void vector(const void* p, float (&v)[V]) const {
    uint32_t w[4];
    load(static_cast<const T*>(p), w);
    values(w, v);
  }
  static __device__ __forceinline__ void values(const uint32_t (&w)[4], float (&v)[V]) {
    T t[V];
    __builtin_memcpy(t, w, 16);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = to_f32(t[e]);
  }
};

// LDS of the reductions: every thread's sums, and partial sums per channel.
template <typename T, int THREADS>
struct GnLds {
  float each[THREADS * kRun<T>];
  static constexpr int kMost = THREADS * kRun<T> < kGnMostChannels ? THREADS * kRun<T> : kGnMostChannels;
  float some[kMost];
  float group[2][kMost];
};

// Column sums of the threads' v in `some`, as J rows of CB; returns J.
template <typename T, int THREADS>
__device__ __forceinline__ int channel_parts(const GnAt<T, THREADS>& at, const float (&v)[kRun<T>], GnLds<T, THREADS>& L) {
  if (at.active && at.skip == 0 && at.left == kRun<T>) {
    __builtin_memcpy(L.each + at.slot * at.CB + at.s, v, sizeof(v));
  } else {
#pragma unroll
    for (int e = 0; e < kRun<T>; ++e)
      if (at.counts(e)) L.each[at.slot * at.CB + at.s + e] = v[e];
  }
  const int J = max(1, min(at.slots, THREADS / at.CB));  // (J CB is at most the larger of THREADS and CB)
  __syncthreads();
  for (int i = threadIdx.x; i < at.CB * J; i += THREADS) {
    const int c = i % at.CB;
    float s = 0.f;
    for (int k = i / at.CB; k < at.slots; k += J) s += L.each[k * at.CB + c];
    L.some[i] = s;
  }
  __syncthreads();
  return J;
}

// out[g] = sum of the threads' v over group g of the bundle.
template <typename T, int THREADS>
__device__ __forceinline__ void group_sums(const GnParams& P, const GnAt<T, THREADS>& at, const float (&v)[kRun<T>],
                                           GnLds<T, THREADS>& L, float* out) {
  const int J = channel_parts<T, THREADS>(at, v, L);
  const int lane = threadIdx.x & 63;
  for (int g = threadIdx.x >> 6; g < at.groups; g += THREADS / 64) {
    float s = 0.f;
    for (int i = lane; i < P.D * J; i += 64) {
      const int j = by_d(P, i);
      s += L.some[j * at.CB + g * P.D + i - j * P.D];
    }
    s = wave_sum(s);
    if (lane == 0) out[g] = s;
  }
  __syncthreads();
}

// What is unpacked from these registers is not kept from one pass over them to the next.
template <int RUNS>
__device__ __forceinline__ void again(uint32_t (&w)[RUNS][4]) {
#pragma unroll
  for (int k = 0; k < RUNS; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[k][i]));
}

template <typename T>
__device__ __forceinline__ const T* row_of(const void* p, const GnParams& P, int n, GnRow r, long long ld) {
  return static_cast<const T*>(p) + ((long long)n * P.P + r) * ld;
}

// Sample and bundle of a workgroup: those of a sample lie on one XCD.
__device__ __forceinline__ bool unit_of(const GnParams& P, int id, int& sample, int& bundle) {
  const int local = id / 8;
  sample = local / P.bundles * 8 + id % 8;
  bundle = local % P.bundles;
  return sample < P.N;
}

template <typename T, int THREADS, int RUNS>
__global__ __launch_bounds__(THREADS) void gn_fwd_held(GnParams P) {
  constexpr int V = kRun<T>;
  __shared__ GnLds<T, THREADS> L;
  GnAt<T, THREADS> at;
  int sample, bundle;
  if (!unit_of(P, blockIdx.x, sample, bundle)) return;
  at.place(P, sample, bundle);
  uint32_t raw[RUNS][4];
#pragma unroll
  for (int k = 0; k < RUNS; ++k) at.load(row_of<T>(P.x, P, sample, min(at.slot + k * at.slots, P.P - 1), P.ldx), raw[k]);
  float w[V], b[V], v[V], s[V] = {};
  at.vector(P.w, w);
  at.vector(P.b, b);
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    if (at.slot + k * at.slots >= P.P) break;
    at.values(raw[k], v);
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] += v[e];
  }
  const float count = (float)P.P * (float)P.D;
  group_sums<T, THREADS>(P, at, s, L, L.group[0]);
  if constexpr (sizeof(T) == 2) again(raw);
  float mean[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    mean[e] = L.group[0][at.group(P, e)] / count;
    s[e] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    if (at.slot + k * at.slots >= P.P) break;
    at.values(raw[k], v);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = v[e] - mean[e];
      s[e] = fmaf(d, d, s[e]);
    }
  }
  group_sums<T, THREADS>(P, at, s, L, L.group[1]);
  if constexpr (sizeof(T) == 2) again(raw);
  for (int g = threadIdx.x; g < at.groups; g += THREADS) {
    P.mean[(long long)sample * P.G + at.g0 + g] = L.group[0][g] / count;
    P.rstd[(long long)sample * P.G + at.g0 + g] = 1.f / sqrtf(L.group[1][g] / count + P.eps);
  }
  if (!at.active) return;
#pragma unroll
  for (int e = 0; e < V; ++e) w[e] *= 1.f / sqrtf(L.group[1][at.group(P, e)] / count + P.eps);
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    const int r = at.slot + k * at.slots;
    if (r >= P.P) break;
    at.values(raw[k], v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = fmaf(v[e] - mean[e], w[e], b[e]);
    gn_values<sizeof(T) == 2>(v, P.act);
    at.store(const_cast<T*>(row_of<T>(P.out, P, sample, r, P.ldy)), v);
  }
}

// ---- samples in chunks

static_assert(kGnThreads * kRun<float> >= kGnMostChannels, "a run of a row for each thread");

struct GnChunk {
  int chunk, bundle, sample;
  GnRow r0, r1;
};
__device__ __forceinline__ GnChunk chunk_of(const GnParams& P) {
  GnChunk c;
  const int id = blockIdx.x;
  c.bundle = id % P.bundles;
  c.chunk = id / P.bundles % P.chunks;
  c.sample = id / P.bundles / P.chunks;
  c.r0 = (GnRow)c.chunk * (GnRow)P.rows;
  c.r1 = min((GnRow)P.P, c.r0 + (GnRow)P.rows);
  return c;
}

// Statistics of a chunk: a thread's mean and sum of squared differences per
// channel, eight rows at a time, then those of the groups.
template <typename T>
__global__ __launch_bounds__(kGnThreads) void gn_stats(GnParams P) {
  constexpr int V = kRun<T>, B = kGnBatch;
  __shared__ GnLds<T, kGnThreads> L;
  const GnChunk ch = chunk_of(P);
  GnAt<T, kGnThreads> at;
  at.place(P, ch.sample, ch.bundle);
  float mean[V] = {}, sq[V] = {}, count = 0.f;
  for (GnRow r = ch.r0 + at.slot; r < ch.r1; r += B * at.slots) {
    uint32_t raw[B][4];
#pragma unroll
    for (int k = 0; k < B; ++k) at.load(row_of<T>(P.x, P, ch.sample, gn_row(r, k, at.slots, ch.r1), P.ldx), raw[k]);
    const int left = min(B, ((int)(ch.r1 - r) + at.slots - 1) / at.slots);
    float s[V] = {}, v[V];
#pragma unroll
    for (int k = 0; k < B; ++k) {
      at.values(raw[k], v);
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += k < left ? v[e] : 0.f;
    }
    const float more = (float)left, inv = 1.f / more, total = count + more;
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] *= inv;
    float q[V] = {};
#pragma unroll
    for (int k = 0; k < B; ++k) {
      at.values(raw[k], v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = k < left ? v[e] - s[e] : 0.f;
        q[e] = fmaf(d, d, q[e]);
      }
    }
    const float share = more / total, both = count * share;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = s[e] - mean[e];
      mean[e] = fmaf(d, share, mean[e]);
      sq[e] += fmaf(d * d, both, q[e]);
    }
    count = total;
  }
  const float n = (float)(ch.r1 - ch.r0) * (float)P.D;
  float v[V];
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = mean[e] * count;
  group_sums<T, kGnThreads>(P, at, v, L, L.group[0]);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float d = mean[e] - L.group[0][at.group(P, e)] / n;
    v[e] = fmaf(d * d, count, sq[e]);
  }
  group_sums<T, kGnThreads>(P, at, v, L, L.group[1]);
  for (int g = threadIdx.x; g < at.groups; g += kGnThreads) {
    float* part = P.part + (((long long)ch.sample * P.G + at.g0 + g) * P.chunks + ch.chunk) * 2;
    part[0] = L.group[0][g] / n;
    part[1] = L.group[1][g];
  }
}

// What the chunks of a sample's group left, 64 chunks to a lane's register.
constexpr int kGnLeft = kGnMostChunks / 64;
__device__ __forceinline__ void left_of(const float* of, int chunks, float (&a)[kGnLeft], float (&b)[kGnLeft]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < kGnLeft; ++k) {
    const int q = lane + 64 * k;
    a[k] = q < chunks ? of[2 * q] : 0.f;
    b[k] = q < chunks ? of[2 * q + 1] : 0.f;
  }
}

// The chunks' statistics joined, a wave for a sample's group.  (A launch of its own: joined by every workgroup of gn_apply, a
// wave group after group, 1 x 37872 x 144 in 48 groups backward took 20 us longer.)
__global__ __launch_bounds__(kGnThreads) void gn_join(GnParams P) {
  constexpr int kWaves = kGnThreads / 64;
  const int lane = threadIdx.x & 63;
  const float total = (float)P.P * (float)P.D;
  const long long groups = (long long)P.N * P.G;
  for (long long id = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6); id < groups; id += (long long)gridDim.x * kWaves) {
    float m[kGnLeft], sq[kGnLeft], s = 0.f, all = 0.f;
    left_of(P.part + id * P.chunks * 2, P.chunks, m, sq);
    auto count = [&](int k) __attribute__((always_inline)) {  // (none behind the last chunk)
      const int q = lane + 64 * k;
      return q < P.chunks ? (float)min(P.P - q * P.rows, P.rows) * (float)P.D : 0.f;
    };
#pragma unroll
    for (int k = 0; k < kGnLeft; ++k) s = fmaf(count(k), m[k], s);
    const float mean = wave_sum(s) / total;
#pragma unroll
    for (int k = 0; k < kGnLeft; ++k) {
      const float d = m[k] - mean, n = count(k);
      all += n > 0.f ? fmaf(d * d, n, sq[k]) : 0.f;
    }
    const float rstd = 1.f / sqrtf(wave_sum(all) / total + P.eps);
    if (lane == 0) {
      P.mean[id] = mean;
      P.rstd[id] = rstd;
    }
  }
}

// The chunk's results.
template <typename T>
__global__ __launch_bounds__(kGnThreads) void gn_apply(GnParams P) {
  constexpr int V = kRun<T>, B = kGnBatch / 2;
  const GnChunk ch = chunk_of(P);
  GnAt<T, kGnThreads> at;
  at.place(P, ch.sample, ch.bundle);
  GnRow r = ch.r0 + at.slot;
  uint32_t raw[B][4];
  auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < B; ++k) at.load(row_of<T>(P.x, P, ch.sample, gn_row(r, k, at.slots, ch.r1), P.ldx), raw[k]);
  };
  load();
  if (!at.active) return;
  float w[V], b[V], mean[V];
  at.vector(P.w, w);
  at.vector(P.b, b);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const long long g = (long long)ch.sample * P.G + at.g0 + at.group(P, e);
    mean[e] = P.mean[g];
    w[e] *= P.rstd[g];
  }
  for (;;) {
#pragma unroll
    for (int k = 0; k < B; ++k) {
      if (r + k * at.slots >= ch.r1) break;
      float v[V];
      at.values(raw[k], v);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = fmaf(v[e] - mean[e], w[e], b[e]);
      gn_values<sizeof(T) == 2>(v, P.act);
      at.store(const_cast<T*>(row_of<T>(P.out, P, ch.sample, r + k * at.slots, P.ldy)), v);
    }
    r += B * at.slots;
    if (r >= ch.r1) break;
    load();
  }
}

// ---- backward

// xh and dh of a run.
template <typename T>
__device__ __forceinline__ void gn_slopes(const GnParams& P, const float (&mean)[kRun<T>], const float (&rstd)[kRun<T>],
                                          const float (&w)[kRun<T>], const float (&b)[kRun<T>], float (&x)[kRun<T>],
                                          float (&dy)[kRun<T>]) {
  float h[kRun<T>];
#pragma unroll
  for (int e = 0; e < kRun<T>; ++e) {
    x[e] = (x[e] - mean[e]) * rstd[e];
    h[e] = fmaf(x[e], w[e], b[e]);
  }
  gn_slopes_of<sizeof(T) == 2>(dy, h, P.act);
}

// Sums of a workgroup's rows: dw and db per channel to `part`, and (in L.group) over the groups
// of db w and dw w, the sums of g and g xh.
template <typename T, int THREADS>
__device__ __forceinline__ void gn_bwd_join(const GnParams& P, const GnAt<T, THREADS>& at, const float (&dw)[kRun<T>],
                                            const float (&db)[kRun<T>], GnLds<T, THREADS>& L, float* part) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < 2; ++k) {  // db, dw
    const int J = channel_parts<T, THREADS>(at, k ? dw : db, L);
    for (int c = threadIdx.x; c < at.CB; c += THREADS) {
      float s = 0.f;
      for (int j = 0; j < J; ++j) s += L.some[j * at.CB + c];
      part[(k ? 0 : P.C) + at.c0 + c] = s;
      L.each[c] = s * to_f32(static_cast<const T*>(P.w)[at.c0 + c]);
    }
    __syncthreads();
    for (int g = threadIdx.x >> 6; g < at.groups; g += THREADS / 64) {
      float s = 0.f;
      for (int i = lane; i < P.D; i += 64) s += L.each[g * P.D + i];
      s = wave_sum(s);
      if (lane == 0) L.group[k][g] = s;
    }
    __syncthreads();
  }
}

template <typename T, int THREADS, int RUNS>
__global__ __launch_bounds__(THREADS) void gn_bwd_held(GnParams P) {
  constexpr int V = kRun<T>;
  __shared__ GnLds<T, THREADS> L;
  GnAt<T, THREADS> at;
  int sample, bundle;
  if (!unit_of(P, blockIdx.x, sample, bundle)) return;
  at.place(P, sample, bundle);
  uint32_t rx[RUNS][4], rg[RUNS][4];
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    const int r = min(at.slot + k * at.slots, P.P - 1);
    at.load(row_of<T>(P.x, P, sample, r, P.ldx), rx[k]);
    at.load(row_of<T>(P.dy, P, sample, r, P.ldd), rg[k]);
  }
  float w[V], b[V], mean[V], rstd[V], dw[V] = {}, db[V] = {};
  at.vector(P.w, w);
  at.vector(P.b, b);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const long long g = (long long)sample * P.G + at.g0 + at.group(P, e);
    mean[e] = P.mean[g];
    rstd[e] = P.rstd[g];
  }
  float x[V], g[V];
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    if (at.slot + k * at.slots >= P.P) break;
    at.values(rx[k], x);
    at.values(rg[k], g);
    gn_slopes<T>(P, mean, rstd, w, b, x, g);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      dw[e] = fmaf(g[e], x[e], dw[e]);
      db[e] += g[e];
    }
    if constexpr (sizeof(T) == 4) {  // kept for the second pass
      __builtin_memcpy(rx[k], x, 16);
      __builtin_memcpy(rg[k], g, 16);
    }
  }
  gn_bwd_join<T, THREADS>(P, at, dw, db, L, P.part + (long long)sample * 2 * P.C);
  if constexpr (sizeof(T) == 2) {
    again(rx);
    again(rg);
  }
  if (!at.active) return;
  const float inv = 1.f / ((float)P.P * (float)P.D);
  float s[V], sx[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int i = at.group(P, e);
    s[e] = L.group[0][i] * inv;
    sx[e] = L.group[1][i] * inv;
  }
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    const int r = at.slot + k * at.slots;
    if (r >= P.P) break;
    at.values(rx[k], x);
    at.values(rg[k], g);
    if constexpr (sizeof(T) == 2) gn_slopes<T>(P, mean, rstd, w, b, x, g);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = rstd[e] * (fmaf(g[e], w[e], -s[e]) - x[e] * sx[e]);
    at.store(const_cast<T*>(row_of<T>(P.out, P, sample, r, P.ldy)), x);
  }
}

// A thread's runs of x and dy, `B` rows at a time.
template <typename T, int B>
struct GnRows {
  uint32_t x[B][4], g[B][4];
  __device__ __forceinline__ void load(const GnParams& P, const GnAt<T, kGnThreads>& at, const GnChunk& ch, GnRow r) {
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const GnRow row = gn_row(r, k, at.slots, ch.r1);
      at.load(row_of<T>(P.x, P, ch.sample, row, P.ldx), x[k]);
      at.load(row_of<T>(P.dy, P, ch.sample, row, P.ldd), g[k]);
    }
  }
};

template <typename T>
__global__ __launch_bounds__(kGnThreads) void gn_bwd_sums(GnParams P) {
  constexpr int V = kRun<T>, B = kGnBatch / 2;
  __shared__ GnLds<T, kGnThreads> L;
  const GnChunk ch = chunk_of(P);
  GnAt<T, kGnThreads> at;
  at.place(P, ch.sample, ch.bundle);
  GnRows<T, B> rows;
  GnRow r = ch.r0 + at.slot;
  rows.load(P, at, ch, r);
  float w[V], b[V], mean[V], rstd[V], dw[V] = {}, db[V] = {};
  at.vector(P.w, w);
  at.vector(P.b, b);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const long long g = (long long)ch.sample * P.G + at.g0 + at.group(P, e);
    mean[e] = P.mean[g];
    rstd[e] = P.rstd[g];
  }
  for (;;) {
#pragma unroll
    for (int k = 0; k < B; ++k) {
      if (r + k * at.slots >= ch.r1) break;
      float x[V], g[V];
      at.values(rows.x[k], x);
      at.values(rows.g[k], g);
      gn_slopes<T>(P, mean, rstd, w, b, x, g);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dw[e] = fmaf(g[e], x[e], dw[e]);
        db[e] += g[e];
      }
    }
    r += B * at.slots;
    if (r >= ch.r1) break;
    rows.load(P, at, ch, r);
  }
  const long long piece = (long long)ch.sample * P.chunks + ch.chunk;
  gn_bwd_join<T, kGnThreads>(P, at, dw, db, L, P.part + piece * 2 * P.C);
  for (int g = threadIdx.x; g < at.groups; g += kGnThreads) {
    float* part = P.part + (long long)P.N * P.chunks * 2 * P.C + (((long long)ch.sample * P.G + at.g0 + g) * P.chunks + ch.chunk) * 2;
    part[0] = L.group[0][g];
    part[1] = L.group[1][g];
  }
}

// dw and db of all pieces, 32 columns x 32 slices of the pieces in a workgroup, each in order, and in the
// workgroups after those the groups' sums, a wave for a sample's group.
template <typename T>
__global__ __launch_bounds__(1024) void gn_bwd_close(GnParams P) {
  constexpr int kCols = kGnCloseCols, kSlices = 32, kBatch = 8;
  static_assert(kCols * kSlices == 64 * kGnCloseWaves, "a workgroup of either kind");
  __shared__ float red[kSlices][kCols + 1];
  const int blocks = (2 * P.C + kCols - 1) / kCols;
  if ((int)blockIdx.x >= blocks) {
    const long long groups = (long long)P.N * P.G;
    float* const of = P.part + (long long)P.N * P.chunks * 2 * P.C;
    const float inv = 1.f / ((float)P.P * (float)P.D);
    long long id = (long long)((int)blockIdx.x - blocks) * kGnCloseWaves + (threadIdx.x >> 6);
    for (; id < groups; id += (long long)((int)gridDim.x - blocks) * kGnCloseWaves) {
      float g[kGnLeft], gx[kGnLeft], s = 0.f, sx = 0.f;
      left_of(of + id * P.chunks * 2, P.chunks, g, gx);
#pragma unroll
      for (int k = 0; k < kGnLeft; ++k) {
        s += g[k];
        sx += gx[k];
      }
      s = wave_sum(s);
      sx = wave_sum(sx);
      if ((threadIdx.x & 63) == 0) {
        float* const to = of + (groups * P.chunks + id) * 2;
        to[0] = s * inv;
        to[1] = sx * inv;
      }
    }
    return;
  }
  const int col = threadIdx.x % kCols, slice = threadIdx.x / kCols, c = blockIdx.x * kCols + col, parts = P.N * P.chunks;
  float s = 0.f;
  if (c < 2 * P.C) {
    for (int j0 = slice; j0 < parts; j0 += kSlices * kBatch) {
      float v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int j = j0 + u * kSlices;
        v[u] = j < parts ? P.part[(long long)j * 2 * P.C + c] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) s += v[u];
    }
  }
  red[slice][col] = s;
  __syncthreads();
  if (slice == 0 && c < 2 * P.C) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < kSlices; ++k) t += red[k][col];
    static_cast<T*>(c < P.C ? P.dw : P.db)[c < P.C ? c : c - P.C] = from_f32<T>(t);
  }
}

template <typename T>
__global__ __launch_bounds__(kGnThreads) void gn_bwd_apply(GnParams P) {
  constexpr int V = kRun<T>, B = kGnBatch / 2;
  const GnChunk ch = chunk_of(P);
  GnAt<T, kGnThreads> at;
  at.place(P, ch.sample, ch.bundle);
  GnRows<T, B> rows;
  GnRow r = ch.r0 + at.slot;
  rows.load(P, at, ch, r);
  const float* const sums = P.part + ((long long)P.N * P.chunks * (P.C + P.G) + (long long)ch.sample * P.G + at.g0) * 2;
  if (!at.active) return;
  float w[V], b[V], mean[V], rstd[V], s[V], sx[V];
  at.vector(P.w, w);
  at.vector(P.b, b);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int i = at.group(P, e);
    mean[e] = P.mean[(long long)ch.sample * P.G + at.g0 + i];
    rstd[e] = P.rstd[(long long)ch.sample * P.G + at.g0 + i];
    s[e] = sums[2 * i];
    sx[e] = sums[2 * i + 1];
  }
  for (;;) {
#pragma unroll
    for (int k = 0; k < B; ++k) {
      if (r + k * at.slots >= ch.r1) break;
      float x[V], g[V];
      at.values(rows.x[k], x);
      at.values(rows.g[k], g);
      gn_slopes<T>(P, mean, rstd, w, b, x, g);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = rstd[e] * (fmaf(g[e], w[e], -s[e]) - x[e] * sx[e]);
      at.store(const_cast<T*>(row_of<T>(P.out, P, ch.sample, r + k * at.slots, P.ldy)), x);
    }
    r += B * at.slots;
    if (r >= ch.r1) break;
    rows.load(P, at, ch, r);
  }
}

// ---- launches

// Calls f with a plan's threads and runs.
template <bool BACKWARD, int ESIZE, typename F>
bool with_gn(const GnPlan& pl, F&& f) {
  using std::integral_constant;
  constexpr int kBig = gn_big(BACKWARD, ESIZE);
  bool done = false;
  auto with = [&](auto threads) {
    auto runs = [&](auto r) {
      constexpr int TH = decltype(threads)::value, R = decltype(r)::value;
      if constexpr (gn_takes(BACKWARD, ESIZE, TH, R)) {
        if (pl.threads != TH || pl.runs != R) return;
        f(threads, r);
        done = true;
      }
    };
    runs(integral_constant<int, 2>{});
    runs(integral_constant<int, 4>{});
    runs(integral_constant<int, 6>{});
    runs(integral_constant<int, 8>{});
    runs(integral_constant<int, 10>{});
  };
  with(integral_constant<int, 64>{});
  with(integral_constant<int, 256>{});
  with(integral_constant<int, kBig>{});
  return done;
}

inline unsigned gn_units(const GnParams& p) { return (unsigned)(cdiv(p.N, 8) * 8 * p.bundles); }
inline unsigned gn_pieces(const GnParams& p) { return (unsigned)((long long)p.N * p.chunks * p.bundles); }

template <typename T>
hipError_t gn_fwd_t(const GnPlan& pl, const GnParams& p, hipStream_t stream) {
  if (pl.held) {
    const bool done = with_gn<false, (int)sizeof(T)>(pl, [&](auto threads, auto runs) {
      constexpr int TH = decltype(threads)::value, R = decltype(runs)::value;
      hipLaunchKernelGGL((gn_fwd_held<T, TH, R>), dim3(gn_units(p)), dim3(TH), 0, stream, p);
    });
    return done ? hipGetLastError() : hipErrorInvalidValue;
  }
  hipLaunchKernelGGL((gn_stats<T>), dim3(gn_pieces(p)), dim3(kGnThreads), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(gn_join, dim3(gn_join_blocks(p.N, p.G, kGnThreads / 64)), dim3(kGnThreads), 0, stream, p);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gn_apply<T>), dim3(gn_pieces(p)), dim3(kGnThreads), 0, stream, p);
  return hipGetLastError();
}

template <typename T>
hipError_t gn_bwd_t(const GnPlan& pl, const GnParams& p, hipStream_t stream) {
  if (pl.held) {
    const bool done = with_gn<true, (int)sizeof(T)>(pl, [&](auto threads, auto runs) {
      constexpr int TH = decltype(threads)::value, R = decltype(runs)::value;
      hipLaunchKernelGGL((gn_bwd_held<T, TH, R>), dim3(gn_units(p)), dim3(TH), 0, stream, p);
    });
    const hipError_t e = done ? hipGetLastError() : hipErrorInvalidValue;
    return e != hipSuccess ? e : launch_col_sum(sizeof(T) == 4 ? Dtype::F32 : Dtype::BF16, p.part, p.N, 2ll * p.C, p.C, p.dw, p.db, stream);
  }
  hipLaunchKernelGGL((gn_bwd_sums<T>), dim3(gn_pieces(p)), dim3(kGnThreads), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gn_bwd_close<T>), dim3(gn_close_columns(p.C) + gn_join_blocks(p.N, p.G, kGnCloseWaves)), dim3(64 * kGnCloseWaves), 0, stream, p);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gn_bwd_apply<T>), dim3(gn_pieces(p)), dim3(kGnThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace
}  // namespace rows
}  // namespace o1d
