// Products of few rows (included by o1d_few_f32.hip and o1d_few_bf16.hip): forward and input gradient
// where tiles of o1d_mm_kernels.h would leave most of the GPU without work, and
// each of their steps waits for memory.
//
// A workgroup of eight waves computes 16 MB rows x 16 NB columns: NB waves side
// by side, the others with every 8 / NB-th piece of 32 k.  Fragments come from memory
// into registers, kBatch pieces at a time with nothing between them, and
// the waves' sums are joined in LDS in a fixed order before the epilogue.
// Bound by the latency of about K / (32 kBatch 8) rounds of loads; weights are
// read once per 64 rows.  16 x 768 -> 1000 bfloat16 5.0 us.  Products and pieces of float32: as in o1d_mm_kernels.h,
// on v_mfma_f32_16x16x32_bf16 (lane l has row l % 16, k 8 (l / 16) .. + 7).
#pragma once

#include "o1d_mm_kernels.h"

namespace o1d {
namespace rows {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kFewThreads = 512;

// Eight elements as they are in memory.
template <typename T>
struct Run8 {
  T e[8];
};

template <typename T>
__device__ __forceinline__ Frag<T> frag_of(const Run8<T>& r) {
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
    __builtin_memcpy(&f.p[0], r.e, 16);
  } else {
    float odd = 0.f;
    u32x4 w[2];
    __builtin_memcpy(w, r.e, 32);
    uint2 p[2][3];
#pragma unroll
    for (int i = 0; i < 2; ++i) split4(w[i], p[i], odd);
    if (odd != odd) {
#pragma unroll
      for (int i = 0; i < 2; ++i) split_any(w[i], p[i]);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) f.p[k] = u32x4{p[0][k].x, p[0][k].y, p[1][k].x, p[1][k].y};
  }
  return f;
}

// k .. k + 7 (zeros past K) of the row that starts `row` elements from base, or
// (STRIDED) of the column there, whose elements lie ld apart.  (Offsets from the
// workgroup's own rows, in 32 bits: half the registers of addresses.)
template <typename T, bool STRIDED>
__device__ __forceinline__ Run8<T> load8(const T* base, uint32_t row, long long ld, int k, int K) {
  Run8<T> r;
  if constexpr (STRIDED) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const T v = base[(long long)min(k + e, K - 1) * ld + row];
      r.e[e] = k + e < K ? v : T(0);
    }
  } else {
    const uint32_t at = row + (uint32_t)k;
    if (k + 8 <= K) {
      __builtin_memcpy(r.e, reinterpret_cast<const char*>(base) + at * (uint32_t)sizeof(T), sizeof(r.e));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.e[e] = k + e < K ? base[at + e] : T(0);
    }
  }
  return r;
}

template <typename T>
__device__ __forceinline__ f32x4 few_product(const Frag<T>& n, const Frag<T>& m, f32x4 acc) {
  auto add = [&](int i, int k) __attribute__((always_inline)) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, n.p[i]), __builtin_bit_cast(bf16x8, m.p[k]),
                                                  acc, 0, 0, 0);
  };
  if constexpr (sizeof(T) == 4) {
    add(2, 0);
    add(0, 2);
    add(1, 1);
    add(1, 0);
    add(0, 1);
  }
  add(0, 0);
  return acc;
}

// 64 rows: registers for two workgroups per CU, which takes float32 to one piece at
// a time; one workgroup with twice the loads is as fast up to 256 workgroups and
// takes 1.05 to 1.2 times as long above.
template <typename T, int KIND, int MB, int NB>
__global__ __launch_bounds__(kFewThreads, (MB == 4 ? 4 : 2)) void few(MmParams P) {
  constexpr int kSplit = 8 / NB, kBatch = MB == 4 && sizeof(T) == 4 ? 1 : 4, kPitch = 16 * NB + 4;
  __shared__ float red[kSplit][16 * MB][kPitch];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nb = wave % NB, ks = wave / NB;
  const int n0 = blockIdx.x * 16 * NB;
  const long long m0 = (long long)blockIdx.y * 16 * MB;
  const T *A = static_cast<const T*>(P.a) + m0 * P.lda,
          *B = static_cast<const T*>(P.b) + (KIND == kFwd ? (long long)n0 * P.ldb : (long long)n0);
  const uint32_t n = (uint32_t)min(16 * nb + (lane & 15), P.N - 1 - n0);
  const uint32_t br = KIND == kFwd ? n * (uint32_t)P.ldb : n;
  uint32_t ar[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
    ar[i] = (uint32_t)min((long long)(16 * i + (lane & 15)), P.M - 1 - m0) * (uint32_t)P.lda;
  f32x4 acc[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int pieces = (P.K + 31) / 32;
  for (int c0 = ks; c0 < pieces; c0 += kSplit * kBatch) {
    Run8<T> b[kBatch], a[kBatch][MB];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int c = c0 + u * kSplit;
      if (c < pieces) {
        const int k = 32 * c + 8 * (lane >> 4);
        b[u] = load8<T, KIND == kDgrad>(B, br, P.ldb, k, P.K);
#pragma unroll
        for (int i = 0; i < MB; ++i) a[u][i] = load8<T, false>(A, ar[i], 0, k, P.K);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (c0 + u * kSplit < pieces) {
        const Frag<T> fn = frag_of(b[u]);
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i] = few_product<T>(fn, frag_of(a[u][i]), acc[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
    *reinterpret_cast<f32x4*>(&red[ks][16 * i + (lane & 15)][16 * nb + 4 * (lane >> 4)]) = acc[i];
  __syncthreads();
  // eight columns of a row per thread
  if (threadIdx.x >= 16 * MB * 2 * NB) return;
  const int row = threadIdx.x / (2 * NB), col = threadIdx.x % (2 * NB) * 8, at = n0 + col;
  const int m = (int)min(m0 + row, (long long)P.M);
  Ahead<T, KIND, false> ahead;
  ahead.load(P, m, at);
  float v[8] = {};
#pragma unroll
  for (int k = 0; k < kSplit; ++k) {
    float u[8];
    __builtin_memcpy(u, &red[k][row][col], 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += u[e];
  }
  if (KIND == kFwd && P.bias) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < P.N) v[e] += to_f32(static_cast<const T*>(P.bias)[at + e]);
  }
  if constexpr (KIND == kFwd && NB == 4) {
    if (P.q) {  // eight lanes have a group
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = at + e < P.N ? v[e] : 0.f;
      const Scale s = scale_of(max8(amax_bits(v)));
      if (m < P.M && at < P.ldq) *reinterpret_cast<uint2*>(P.q + (long long)m * P.ldq + at) = round8(v, s);
      if (m < P.M && at < P.N && at % kGroup == 0) P.scale[(long long)m * P.groups + at / kGroup] = s.scale;
    }
  }
  finish<T, KIND, false>(P, m, at, ahead, v);
}

template <typename T, int KIND, int NB>
hipError_t launch_few_rows(const MmParams& p, hipStream_t stream) {
  const dim3 block(kFewThreads);
  const unsigned gx = (unsigned)cdiv(p.N, 16 * NB);
  if (p.M <= 16)
    hipLaunchKernelGGL((few<T, KIND, 1, NB>), dim3(gx, 1), block, 0, stream, p);
  else if (p.M <= 32)
    hipLaunchKernelGGL((few<T, KIND, 2, NB>), dim3(gx, 1), block, 0, stream, p);
  else
    hipLaunchKernelGGL((few<T, KIND, 4, NB>), dim3(gx, (unsigned)cdiv(p.M, 64)), block, 0, stream, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_few_t(int kind, const MmParams& p, hipStream_t stream) {
  if (kind == kDgrad) return launch_few_rows<T, kDgrad, 1>(p, stream);
  return p.q ? launch_few_rows<T, kFwd, 4>(p, stream) : launch_few_rows<T, kFwd, 1>(p, stream);
}

}  // namespace
}  // namespace rows
}  // namespace o1d
