// AdamW over many tensors at once, with states of 32 or 8 bits.
//
//   g = factor gradient,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   w = w (1 - lr decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
//
// factor limits the gradients' norm over all tensors (launch_grad_norm) to max_norm; where
// that norm is not finite, nothing changes, the count of steps included.  The count
// lies in device memory, so that a captured step counts on every replay.
//
// In 8 bits, m and r = sqrt(v) are e4m3 with a float32 scale, the largest / 448, for each 128 values.  The root halves
// v's range; a positive r is at least the type's smallest value, so that no m meets a v that was rounded to zero.
// Every operation is rounded by itself (no fused multiply-add): the 8-bit values do not depend on
// how a compiler joins them.
//
// Memory bounds it: 28 bytes per value in float32, 16.1 (bfloat16 parameters and gradients, their
// float32 values, 8-bit states; 18.1 where the parameters are read beside those).  A thread has eight values, 16 threads a scale; a workgroup
// finds the tensor of each piece of 2048 values among those in its arguments.
//
// Measured, the parameters of 15 blocks (11.9 million values in 105 tensors): float32 66 us, 5.1 TB/s, and 19 us for the norm; in
// bfloat16 with 8-bit states 47 us, 4.1 TB/s.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "o1d_adam.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {
namespace {

constexpr int kAdamBlocks = 2048;  // eight of a CU, all there at once
constexpr int kAdamThreads = 256, kAdamRun = 8, kAdamPiece = kAdamThreads * kAdamRun;

struct AdamList {
  int first[kAdamMost];  // of all pieces
  int at[kAdamMost];     // where its states start, in groups of 128
  void* p[kAdamMost];
  const void* g[kAdamMost];
  long long n[kAdamMost];
  int count, pieces, per;  // pieces of a workgroup, one behind the other
};
static_assert(sizeof(AdamList) + sizeof(AdamState) + sizeof(AdamHyper) + 4 <= 4096, "a kernel's arguments");

// A list's tensors in LDS.  Arguments lie in host memory, a microsecond away: a workgroup reads all of them at once, whatever
// their number, and not one that depends on another (searched there, a step of 7 tensors took 12.3 us, so 11.5).
struct AdamTable {
  int first[kAdamMost], at[kAdamMost];
  void* p[kAdamMost];
  const void* g[kAdamMost];
  long long n[kAdamMost];
};
__device__ __forceinline__ void fill(const AdamList& L, AdamTable& T) {
  const int i = threadIdx.x;
  if (i < kAdamMost) {
    T.first[i] = L.first[i];
    T.at[i] = L.at[i];
    T.p[i] = L.p[i];
    T.g[i] = L.g[i];
    T.n[i] = L.n[i];
  }
  __syncthreads();
}
// The tensor of a piece: the last that starts at or before it.
__device__ __forceinline__ int tensor_of(const AdamTable& T, int count, int piece) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int k = 0; k < (kAdamMost + 63) / 64; ++k) {
    const int i = lane + 64 * k;
    n += __popcll(__ballot(i < count && T.first[min(i, kAdamMost - 1)] <= piece));
  }
  return __builtin_amdgcn_readfirstlane(n) - 1;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, long long left, float (&v)[kAdamRun]) {
  if (left >= kAdamRun) {
    load_run(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < kAdamRun; ++e) v[e] = e < left ? to_f32(p[e]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, long long left, const float (&v)[kAdamRun]) {
  if (left >= kAdamRun) {
    store_run(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < kAdamRun; ++e)
      if (e < left) p[e] = from_f32<T>(v[e]);
  }
}

// Eight e4m3 values times their scale, and back: the scale is the largest of 16 lanes' values / 448.
__device__ __forceinline__ void from8(uint2 w, float scale, float (&v)[kAdamRun]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int u = (int)(k ? w.y : w.x);
    v[4 * k] = __builtin_amdgcn_cvt_f32_fp8(u, 0) * scale;
    v[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8(u, 1) * scale;
    v[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8(u, 2) * scale;
    v[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8(u, 3) * scale;
  }
}
template <bool LEAST>
__device__ __forceinline__ void to8(const float (&v)[kAdamRun], uint8_t* p, float* scale) {
#pragma clang fp contract(off)
  uint32_t most = max8(amax_bits(v));
  most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp((int)most, 0x140, 0xF, 0xF, true));
  // (below that, 448 / amax leaves float32 and a zero's product with it is NaN)
  const float amax = __uint_as_float(most), top = amax < 448 * 0x1p-126f ? 448 * 0x1p-126f : amax;
  const float inv = most ? 448.f * (1.f / top) : 0.f;  // (the reciprocal rounded first, as in the formula's usual evaluation)
  float u[kAdamRun];
#pragma unroll
  for (int e = 0; e < kAdamRun; ++e) {
    u[e] = v[e] * inv;
    if (LEAST && v[e] > 0.f) u[e] = fmaxf(u[e], 0x1p-9f);
  }
  int w[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(u[4 * k], u[4 * k + 1], w[k], false);
    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(u[4 * k + 2], u[4 * k + 3], w[k], true);
  }
  *reinterpret_cast<uint2*>(p) = make_uint2((uint32_t)w[0], (uint32_t)w[1]);
  if ((threadIdx.x & 15) == 0) *scale = most ? top * (1.f / 448.f) : 0.f;
}

struct Coefs {
  float factor, lr, keep, c1, c2;
  int go;
};

// Where the values come from: the parameters, their masters, or the masters where the parameters are still those rounded.
// (The last reads two bytes more for each value of bfloat16: 11.9 million values with 8-bit states, in a row on the same tensors,
// 41.9 us so, 38.4 from the masters alone.)
enum AdamFrom { kOwn, kMaster, kFollow };

template <typename TP, typename TG, bool HELD8, int FROM>
__global__ __launch_bounds__(kAdamThreads) void adam(AdamList L, AdamState S, AdamHyper H, int counts) {
#pragma clang fp contract(off)
  __shared__ Coefs coefs;
  __shared__ AdamTable table;
  fill(L, table);
  int piece = blockIdx.x * L.per, k = tensor_of(table, L.count, piece);
  const int end = min(L.pieces, piece + L.per);
  struct Place {
    TP* p;
    const TG* g;
    long long i, left, at;
    bool in;
  };
  auto place = [&]() __attribute__((always_inline)) {
    while (k + 1 < L.count && table.first[k + 1] <= piece) ++k;
    Place q;
    const long long n = table.n[k];
    q.i = (long long)(piece - table.first[k]) * kAdamPiece + threadIdx.x * kAdamRun;
    q.p = static_cast<TP*>(table.p[k]) + q.i;
    q.g = static_cast<const TG*>(table.g[k]) + q.i;
    q.left = n - q.i;
    q.at = (long long)table.at[k] * kAdamGroup + q.i;
    q.in = q.i < (n + kAdamGroup - 1) / kAdamGroup * kAdamGroup;  // (the same for 16 threads, a group)
    return q;
  };
  float g[kAdamRun], w[kAdamRun], m[kAdamRun], v[kAdamRun], own[kAdamRun];
  uint2 m8, v8;
  float ms, vs;
  auto load = [&](const Place& q) __attribute__((always_inline)) {
    if (!q.in) return;
    load8(q.g, q.left, g);
    if constexpr (FROM != kOwn) load_run(S.master + q.at, w);
    if constexpr (FROM != kMaster) load8(static_cast<const TP*>(q.p), q.left, FROM == kOwn ? w : own);
    if constexpr (HELD8) {
      m8 = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(S.m) + q.at);
      v8 = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(S.v) + q.at);
      ms = S.ms[q.at / kAdamGroup];
      vs = S.vs[q.at / kAdamGroup];
    } else {
      load_run(static_cast<const float*>(S.m) + q.at, m);
      load_run(static_cast<const float*>(S.v) + q.at, v);
    }
  };
  // (the first piece is on its way while one thread works out the step's factors)
  Place q = place();
  load(q);
  if (threadIdx.x == 0) {
    const int t = steps_taken(S.step[0]) + 1;
    Coefs c;
    c.factor = 1.f;
    c.go = 1;
    if (H.norm) {
      const float norm = *H.norm;
      c.go = norm < __builtin_huge_valf();  // (false for NaN)
      if (norm > H.max_norm) c.factor = H.max_norm / norm;
    }
    c.lr = H.lr_at ? *H.lr_at : H.lr;
    c.keep = H.lr_at ? 1.f - c.lr * H.decay : H.keep;
    c.c1 = (float)(1. / (1. - power(H.beta1_64, t)));
    c.c2 = (float)sqrt(1. / (1. - power(H.beta2_64, t)));
    coefs = c;
  }
  __syncthreads();
  const Coefs c = coefs;
  if (c.go) {
    for (;;) {
      if (q.in) {
        if constexpr (HELD8) {
          from8(m8, ms, m);
          from8(v8, vs, v);
        }
#pragma unroll
        for (int e = 0; e < kAdamRun; ++e) {
          if (H.norm) g[e] *= c.factor;
          if constexpr (HELD8) v[e] *= v[e];
          m[e] = H.beta1 * m[e] + H.rest1 * g[e];
          v[e] = H.beta2 * v[e] + H.rest2 * (g[e] * g[e]);
          const float r = sqrtf(v[e]);
          if constexpr (FROM == kFollow) w[e] = to_f32(from_f32<TP>(w[e])) == own[e] ? w[e] : own[e];
          w[e] = w[e] * c.keep - c.lr * ((m[e] * c.c1) / (r * c.c2 + H.eps));
          if constexpr (HELD8) v[e] = r;
          if (e >= q.left) m[e] = v[e] = w[e] = 0.f;  // (behind the tensor's end the states are zeros)
        }
        store8(q.p, q.left, w);
        if constexpr (FROM != kOwn) store_run(S.master + q.at, w);
        if constexpr (HELD8) {
          to8<false>(m, static_cast<uint8_t*>(S.m) + q.at, S.ms + q.at / kAdamGroup);
          to8<true>(v, static_cast<uint8_t*>(S.v) + q.at, S.vs + q.at / kAdamGroup);
        } else {
          store_run(static_cast<float*>(S.m) + q.at, m);
          store_run(static_cast<float*>(S.v) + q.at, v);
        }
      }
      if (++piece >= end) break;
      q = place();
      load(q);
    }
  }
  // The last workgroup to end counts the step: all others have read it.
  if (counts && threadIdx.x == 0) {
    if (atomicAdd(&S.step[1], 1) == (int)gridDim.x - 1) {
      S.step[1] = 0;
      if (c.go) S.step[0] = steps_taken(S.step[0]) + 1;
    }
  }
}

// ---- the gradients' norm: squares are summed in 64 bits, so that none overflows

// (few and large workgroups: their arrivals at one address take turns; 47 MB in 1951 workgroups of 256 threads 38.8 us, in 255
// of 1024 20.2)
constexpr int kNormThreads = 1024, kNormSide = kNormThreads / kAdamThreads;  // pieces side by side

__device__ __forceinline__ double block_sum64(double s) {
  __shared__ double red[kNormThreads / 64];
  __syncthreads();  // (an earlier sum is read)
#pragma unroll
  for (int m = 1; m < 64; m *= 2) s += __shfl_xor(s, m, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.;
#pragma unroll
  for (int k = 0; k < kNormThreads / 64; ++k) s += red[k];
  return s;
}

// A workgroup's sum is its own part; the last of a call's last launch to end adds all parts, in their order, and takes
// the root.  (The parts pass between XCDs: they are written and read by accesses of the device's scope.)
template <typename TG>
__global__ __launch_bounds__(kNormThreads) void squares(AdamList L, double* part, int add, int ends, int parts, int* arrived,
                                                        float* norm) {
  __shared__ int last;
  __shared__ AdamTable table;
  fill(L, table);
  double s = 0.;
  const int end = min(L.pieces, ((int)blockIdx.x + 1) * L.per);
  int piece = min((int)blockIdx.x * L.per + __builtin_amdgcn_readfirstlane(threadIdx.x / kAdamThreads), end - 1);
  const bool any = piece == (int)blockIdx.x * L.per + (int)(threadIdx.x / kAdamThreads);
  int t = tensor_of(table, L.count, piece);
  constexpr int B = 2;  // pieces at a time
  for (; any && piece < end; piece += B * kNormSide) {
    float g[B][kAdamRun];
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const int at = piece + k * kNormSide;
      while (t + 1 < L.count && table.first[t + 1] <= min(at, end - 1)) ++t;
      const long long i = (long long)(at - table.first[t]) * kAdamPiece + threadIdx.x % kAdamThreads * kAdamRun;
      const long long left = at < end ? table.n[t] - i : 0;
      load8(static_cast<const TG*>(table.g[t]) + (left > 0 ? i : 0), left, g[k]);
    }
#pragma unroll
    for (int k = 0; k < B; ++k)
#pragma unroll
      for (int e = 0; e < kAdamRun; ++e) s = fma((double)g[k][e], (double)g[k][e], s);
  }
  s = block_sum64(s);
  if (threadIdx.x == 0) {
    if (add) s += part[blockIdx.x];  // (of the launch before)
    atomicExch(reinterpret_cast<unsigned long long*>(part + blockIdx.x), __builtin_bit_cast(unsigned long long, s));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the part is there before its arrival is)
    last = ends && atomicAdd(arrived, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  s = 0.;
  for (int i = threadIdx.x; i < parts; i += kNormThreads)
    s += __hip_atomic_load(part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  s = block_sum64(s);
  if (threadIdx.x == 0) {
    *norm = (float)sqrt(s);
    *arrived = 0;
  }
}

// Calls f with each launch's list; `last`: the call's last.
template <typename F>
hipError_t with_lists(const AdamTensor* t, int count, F&& f) {
  for (int from = 0; from < count;) {
    AdamList L;
    L.count = L.pieces = 0;
    for (; from < count && L.count < kAdamMost; ++from, ++L.count) {
      const int k = L.count;
      L.first[k] = L.pieces;
      L.at[k] = (int)(t[from].at / kAdamGroup);
      L.p[k] = t[from].p;
      L.g[k] = t[from].g;
      L.n[k] = t[from].n;
      L.pieces += (int)cdiv(t[from].n, kAdamPiece);
    }
    f(L, from == count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename TP, typename TG>
hipError_t adam_t(const AdamTensor* t, int count, const AdamState& s, const AdamHyper& h, hipStream_t stream) {
  return with_lists(t, count, [&](AdamList& L, bool last) {
    L.per = (int)cdiv(L.pieces, kAdamBlocks);
    const dim3 grid((unsigned)cdiv(L.pieces, L.per)), threads(kAdamThreads);
    auto run = [&](auto held8) {
      constexpr bool H8 = decltype(held8)::value;
      if (!s.master)
        hipLaunchKernelGGL((adam<TP, TG, H8, kOwn>), grid, threads, 0, stream, L, s, h, (int)last);
      else if (h.follow)
        hipLaunchKernelGGL((adam<TP, TG, H8, kFollow>), grid, threads, 0, stream, L, s, h, (int)last);
      else
        hipLaunchKernelGGL((adam<TP, TG, H8, kMaster>), grid, threads, 0, stream, L, s, h, (int)last);
    };
    if (s.bits == 8)
      run(std::true_type{});
    else
      run(std::false_type{});
  });
}

}  // namespace

hipError_t launch_adam(Dtype pdt, Dtype gdt, const AdamTensor* t, int count, const AdamState& s, const AdamHyper& h,
                       hipStream_t stream) {
  if (pdt == Dtype::F32)
    return gdt == Dtype::F32 ? adam_t<float, float>(t, count, s, h, stream) : adam_t<float, uint16_t>(t, count, s, h, stream);
  return gdt == Dtype::F32 ? adam_t<uint16_t, float>(t, count, s, h, stream)
                           : adam_t<uint16_t, uint16_t>(t, count, s, h, stream);
}

hipError_t launch_grad_norm(Dtype gdt, const AdamTensor* t, int count, double* part, int* arrived, float* norm,
                            hipStream_t stream) {
  // (a later list adds to the first list's parts)
  int parts = 0;
  return with_lists(t, count, [&](AdamList& L, bool last) {
    const int most = parts ? parts : kNormBlocks, add = parts > 0;
    L.per = (int)cdiv(L.pieces, most);
    const int blocks = (int)cdiv(L.pieces, L.per);
    if (!parts) parts = blocks;
    if (gdt == Dtype::F32)
      hipLaunchKernelGGL((squares<float>), dim3((unsigned)blocks), dim3(kNormThreads), 0, stream, L, part, add, (int)last,
                         parts, arrived, norm);
    else
      hipLaunchKernelGGL((squares<uint16_t>), dim3((unsigned)blocks), dim3(kNormThreads), 0, stream, L, part, add, (int)last,
                         parts, arrived, norm);
  });
}

}  // namespace rows
}  // namespace o1d
