// 8-bit checkpoints (written, read back), activations and their derivatives
// over whole matrices, and sums over partial rows.
//
// All are bound by memory.  Eight lanes have a group of 64 columns, eight
// columns each (one 16-byte access in bfloat16, two in float32), so that a
// group's largest value takes three lane moves and its integers leave as eight
// bytes per lane.  50176 x 768 bfloat16: written 20.9 us (118 MB, 5.6 TB/s), read
// back through GELU 27.3 (4.3 TB/s; its slots per element), dy gelu'(x) 35.0 (195 MB, 5.6 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "o1d_rows.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {
namespace {

constexpr int kSpan = 8;  // columns of a lane


template <typename T>
__global__ __launch_bounds__(kThreads) void pack_kernel(const T* __restrict__ x, long long ldx, int M, int C,
                                                        int8_t* __restrict__ q, float* __restrict__ scale) {
  const unsigned groups = (unsigned)(C + kGroup - 1) / kGroup;
  const long long ldq = (C + 15) / 16 * 16, total = (long long)M * groups;
  const int l = threadIdx.x & 7;
  for (long long g = (long long)blockIdx.x * (kThreads / 8) + threadIdx.x / 8; g < total;
       g += (long long)gridDim.x * (kThreads / 8)) {
    const long long row = total < (1ll << 32) ? (unsigned)g / groups : g / groups;
    const int group = (int)(g - row * groups), c = group * kGroup + l * kSpan;
    float v[8] = {};
    if (c < C) load_some(x + row * ldx + c, C - c, v);
    const Scale s = scale_of(max8(amax_bits(v)));
    const uint2 w = round8(v, s);
    if (c < ldq) *reinterpret_cast<uint2*>(q + row * ldq + c) = w;
    if (l == 0) scale[g] = s.scale;
  }
}

// y = act(x), or dy act'(x) (SLOPE), x a matrix or (HELD) its checkpoint.
template <typename T, bool HELD, bool SLOPE>
__global__ __launch_bounds__(kThreads) void act_kernel(Operand x, const T* __restrict__ dy, long long lddy, int M, int C,
                                                       int act, T* __restrict__ y, long long ldy) {
  constexpr bool kFast = sizeof(T) == 2;
  const unsigned runs = (unsigned)(C + kSpan - 1) / kSpan;
  const long long ldq = (C + 15) / 16 * 16, groups = (C + kGroup - 1) / kGroup, total = (long long)M * runs;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < total; i += (long long)gridDim.x * kThreads) {
    const long long row = total < (1ll << 32) ? (unsigned)i / runs : i / runs;
    const int c = (int)(i - row * runs) * kSpan, n = C - c;
    float v[8], g[8];
    if constexpr (HELD) {
      const uint2 w = *reinterpret_cast<const uint2*>(x.q + row * ldq + c);
      unround8(w, x.scale[row * groups + c / kGroup], v);
    } else {
      load_some(static_cast<const T*>(x.p) + row * x.ld + c, n, v);
    }
    if constexpr (SLOPE) {
      load_some(dy + row * lddy + c, n, g);
      act_slopes<kFast>(g, v, act);
      store_some(y + row * ldy + c, n, g);
    } else {
      act_values<kFast>(v, act);
      store_some(y + row * ldy + c, n, v);
    }
  }
}

unsigned grid_for(long long items, int per_block) {
  const long long blocks = cdiv(items, per_block);
  return (unsigned)(blocks < 8192 ? (blocks > 0 ? blocks : 1) : 8192);
}

// out[c] = sum over j < parts of part[j ld + c] for the columns of C or 2 C
// (second half to out2): 32 columns x 32 slices of the rows per workgroup, each
// slice added in order, then the slices.
constexpr int kSlices = 32;

template <typename T>
__global__ __launch_bounds__(32 * kSlices) void col_sum(const float* __restrict__ part, int parts, long long ld, int C,
                                                        T* __restrict__ out, T* __restrict__ out2) {
  __shared__ float red[kSlices][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + col, width = out2 ? 2 * C : C;
  float s = 0.f;
  if (c < width) {
    constexpr int kBatch = 8;
    for (int j0 = slice; j0 < parts; j0 += kSlices * kBatch) {
      float v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) v[u] = j0 + u * kSlices < parts ? part[(long long)(j0 + u * kSlices) * ld + c] : 0.f;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) s += v[u];
    }
  }
  red[slice][col] = s;
  __syncthreads();
  if (slice == 0 && c < width) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < kSlices; ++k) t += red[k][col];
    if (c < C)
      out[c] = from_f32<T>(t);
    else
      out2[c - C] = from_f32<T>(t);
  }
}

template <typename T>
hipError_t act_t(const Operand& x, const void* dy, long long lddy, int M, int C, int act, void* y, long long ldy,
                 hipStream_t stream) {
  const dim3 grid(grid_for((long long)M * cdiv(C, kSpan), kThreads)), block(kThreads);
  const T* g = static_cast<const T*>(dy);
  T* o = static_cast<T*>(y);
  if (x.q) {
    if (g) hipLaunchKernelGGL((act_kernel<T, true, true>), grid, block, 0, stream, x, g, lddy, M, C, act, o, ldy);
    else hipLaunchKernelGGL((act_kernel<T, true, false>), grid, block, 0, stream, x, g, lddy, M, C, act, o, ldy);
  } else {
    if (g) hipLaunchKernelGGL((act_kernel<T, false, true>), grid, block, 0, stream, x, g, lddy, M, C, act, o, ldy);
    else hipLaunchKernelGGL((act_kernel<T, false, false>), grid, block, 0, stream, x, g, lddy, M, C, act, o, ldy);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(Dtype dt, const void* x, long long ldx, int M, int C, const Held& h, hipStream_t stream) {
  const dim3 grid(grid_for((long long)M * held_groups(C), kThreads / 8)), block(kThreads);
  if (dt == Dtype::F32)
    hipLaunchKernelGGL(pack_kernel<float>, grid, block, 0, stream, static_cast<const float*>(x), ldx, M, C, h.q, h.scale);
  else
    hipLaunchKernelGGL(pack_kernel<uint16_t>, grid, block, 0, stream, static_cast<const uint16_t*>(x), ldx, M, C, h.q,
                       h.scale);
  return hipGetLastError();
}

hipError_t launch_act(Dtype dt, const Operand& x, const void* dy, long long lddy, int M, int C, int act, void* y,
                      long long ldy, hipStream_t stream) {
  return dt == Dtype::F32 ? act_t<float>(x, dy, lddy, M, C, act, y, ldy, stream)
                          : act_t<uint16_t>(x, dy, lddy, M, C, act, y, ldy, stream);
}

hipError_t launch_col_sum(Dtype dt, const float* part, int parts, long long ld, int C, void* out, void* out2,
                          hipStream_t stream) {
  const dim3 grid((unsigned)cdiv(out2 ? 2ll * C : C, 32)), block(32 * kSlices);
  if (dt == Dtype::F32)
    hipLaunchKernelGGL(col_sum<float>, grid, block, 0, stream, part, parts, ld, C, static_cast<float*>(out),
                       static_cast<float*>(out2));
  else
    hipLaunchKernelGGL(col_sum<uint16_t>, grid, block, 0, stream, part, parts, ld, C, static_cast<uint16_t*>(out),
                       static_cast<uint16_t*>(out2));
  return hipGetLastError();
}

}  // namespace rows
}  // namespace o1d
