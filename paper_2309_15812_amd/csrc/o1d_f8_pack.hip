// Packing of 8-bit floating point operands, and the plan of their products.
//
// A group of 128 values shares the least power of two 2^e with amax 2^-e <= 448
// (e4m3; 57344 for e5m2), amax over its finite values: the largest value stays in
// the type's range and the division is exact, so that a value is rounded once, by the
// conversion (nearest, ties to even).  A value that is not finite becomes NaN.
#include <hip/hip_runtime.h>

#include <atomic>

#include "o1d_f8.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {
namespace {

constexpr int kPackThreads = 256;
template <typename T>
constexpr int kPackPitch = kF8Group + 4 / (int)sizeof(T);  // of the tile's rows: a word more than they hold

template <int TYPE>
__device__ __forceinline__ int exponent_of(uint32_t amax) {
  constexpr int kTop = TYPE == kE4M3 ? 8 : 15;  // 448 = 1.75 2^8, 57344 = 1.75 2^15
  const int e = (int)(amax >> 23) - 127 - kTop + ((amax & 0x7fffffu) > 0x600000u);
  return amax ? max(e, -127) : 0;
}

// Bits of |x| of a finite value, else 0.
__device__ __forceinline__ uint32_t size_of(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// Four values as a word.
template <int TYPE>
__device__ __forceinline__ uint32_t four8(float a, float b, float c, float d, int e) {
  auto at = [&](float x) __attribute__((always_inline)) {
    const float s = ldexpf(x, -e);
    return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? s : __uint_as_float(0x7fc00000u);
  };
  int w = 0;
  if constexpr (TYPE == kE4M3) {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(at(a), at(b), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(at(c), at(d), w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(at(a), at(b), w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(at(c), at(d), w, true);
  }
  return (uint32_t)w;
}

// The largest over 16 consecutive lanes, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t m) {
  m = max8(m);
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xF, 0xF, true));  // row_mirror
}

// A workgroup takes 128 rows x 128 columns.  16 lanes hold a row's group, eight
// columns each, which is packed by rows from there; the tile then lies in LDS, where
// two columns x 32 rows go to a lane, and four waves hold a column's group.
template <typename T, int TYPE>
__global__ __launch_bounds__(kPackThreads) void f8_pack(F8PackParams P) {
  __shared__ uint32_t most[4][kF8Group];
  __shared__ float sums[16][kF8Group];
  __shared__ uint8_t rexp[kF8Group];
  extern __shared__ __align__(16) char lds[];
  T(*tile)[kPackPitch<T>] = reinterpret_cast<T(*)[kPackPitch<T>]>(lds);
  const int r0 = blockIdx.x * kF8Group, c0 = blockIdx.y * kF8Group;
  const int lane16 = threadIdx.x & 15, c = c0 + 8 * lane16;
  const long long ldq = (P.C + kF8Group - 1) / kF8Group * (long long)kF8Group;
  float sum[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = (int)(threadIdx.x >> 4) + 16 * i, r = r0 + row;
    float v[8] = {};
    if (r < P.M && c < P.C) load_some(static_cast<const T*>(P.x) + (long long)r * P.ldx + c, P.C - c, v);
    if (P.q) {
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, size_of(v[e]));
      const int e = exponent_of<TYPE>(max16(m));
      if (r < P.M)
        *reinterpret_cast<uint2*>(P.q + (long long)r * ldq + c) =
            make_uint2(four8<TYPE>(v[0], v[1], v[2], v[3], e), four8<TYPE>(v[4], v[5], v[6], v[7], e));
      if (lane16 == 0) rexp[row] = (uint8_t)(e + 127);
    }
    if (P.qt) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        tile[row][8 * lane16 + e] = from_f32<T>(v[e]);
        sum[e] += v[e];
      }
    }
  }
  if (P.part) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[threadIdx.x >> 4][8 * lane16 + e] = sum[e];
  }
  __syncthreads();
  const long long lem = (P.M + 15) / 16 * 16;
  if (P.q && threadIdx.x < kF8Group && r0 + (int)threadIdx.x < lem)
    P.e[(long long)blockIdx.y * lem + r0 + threadIdx.x] = r0 + (int)threadIdx.x < P.M ? rexp[threadIdx.x] : 127;
  if (!P.qt) return;
  if (P.part && threadIdx.x < kF8Group && c0 + (int)threadIdx.x < P.C) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += sums[k][threadIdx.x];
    P.part[(long long)blockIdx.x * P.C + c0 + threadIdx.x] = s;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float v[2][32];
  uint32_t m[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 32; ++k)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v[j][k] = to_f32(tile[32 * wave + k][2 * lane + j]);
      m[j] = max(m[j], size_of(v[j][k]));
    }
#pragma unroll
  for (int j = 0; j < 2; ++j) most[wave][2 * lane + j] = m[j];
  __syncthreads();
  const long long ldqt = (P.M + kF8Group - 1) / kF8Group * (long long)kF8Group, lec = (P.C + 15) / 16 * 16;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int col = 2 * lane + j;
    const uint32_t a = max(max(most[0][col], most[1][col]), max(most[2][col], most[3][col]));
    const int e = exponent_of<TYPE>(a);
    if (c0 + col < P.C) {
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = four8<TYPE>(v[j][4 * k], v[j][4 * k + 1], v[j][4 * k + 2], v[j][4 * k + 3], e);
      __builtin_memcpy(__builtin_assume_aligned(P.qt + (long long)(c0 + col) * ldqt + r0 + 32 * wave, 16), w, 32);
    }
    if (wave == 0 && c0 + col < lec) P.et[(long long)blockIdx.x * lec + c0 + col] = c0 + col < P.C ? (uint8_t)(e + 127) : 127;
  }
}

template <typename T, int TYPE>
hipError_t launch_pack(const F8PackParams& p, hipStream_t stream) {
  constexpr int kLds = kF8Group * kPackPitch<T> * (int)sizeof(T);
  static std::atomic<int> allowed{0};
  if (!allowed.load(std::memory_order_acquire)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f8_pack<T, TYPE>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    allowed.store(1, std::memory_order_release);
  }
  hipLaunchKernelGGL((f8_pack<T, TYPE>), dim3((unsigned)f8_groups(p.M), (unsigned)f8_groups(p.C)), dim3(kPackThreads),
                     p.qt ? kLds : 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_pack(Dtype dt, const F8PackParams& p, hipStream_t stream) {
  if (dt == Dtype::F32) return p.type == kE4M3 ? launch_pack<float, kE4M3>(p, stream) : launch_pack<float, kE5M2>(p, stream);
  return p.type == kE4M3 ? launch_pack<uint16_t, kE4M3>(p, stream) : launch_pack<uint16_t, kE5M2>(p, stream);
}

F8Plan plan_f8(int kind, int M, int N, int K) {
  F8Plan pl{};
  MmParams& p = pl.p.mm;
  p.M = M;
  p.N = N;
  p.K = (int)f8_ld(K);
  p.steps = f8_groups(K);
  const long long big = cdiv(M, 128) * cdiv(N, 128);
  pl.shape = big >= 256 ? kF8_128x128 : kF8_64x64;
  const Shape& s = kF8Shapes[pl.shape];
  p.tm = (int)cdiv(M, 32 * s.tm * s.wm);
  p.tn = (int)cdiv(N, 32 * s.tn * s.wn);
  long long pieces = 1;
  if (kind == kWgrad) {
    const long long tiles = (long long)p.tm * p.tn;
    pieces = cdiv(512, tiles);
    if (pieces > p.steps / 4) pieces = p.steps / 4;
    if (pieces < 1) pieces = 1;
  }
  p.per = (int)cdiv(p.steps, pieces);
  p.nsplit = (int)cdiv(p.steps, p.per);
  p.nblocks = p.tm * p.tn * p.nsplit;
  return pl;
}

}  // namespace rows
}  // namespace o1d
