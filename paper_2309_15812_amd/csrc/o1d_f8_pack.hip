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
template <typename T, int COLS>
constexpr int kPackPitch = COLS + 4 / (int)sizeof(T);  // of the tile's rows: a word more than they hold

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

// Eight columns of a row from column c on, as they are in memory; zeros past the row's end.
template <typename T>
struct PackRun {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* row, int c, int C) {
    if (c + 8 <= C) {
      __builtin_memcpy(w, row + c, sizeof(w));
    } else {
      T t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = c + e < C ? row[c + e] : T(0);
      __builtin_memcpy(w, t, sizeof(w));
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    T t[8];
    __builtin_memcpy(t, w, sizeof(t));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f32(t[e]);
  }
};

// Sixteen lanes' eight columns each of a row: the group's exponent, and this lane's values.
template <int TYPE>
__device__ __forceinline__ int pack_group(const float (&v)[8], uint2& q) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, size_of(v[e]));
  const int e = exponent_of<TYPE>(max16(m));
  q = make_uint2(four8<TYPE>(v[0], v[1], v[2], v[3], e), four8<TYPE>(v[4], v[5], v[6], v[7], e));
  return e;
}

// By rows alone: 64 rows of a group of columns in a workgroup, four in a row of 16 lanes, all loads before the
// first group is made.  8192 x 8192 bfloat16 in 49 us, 4.1 TB/s; row after row in a lane 65.
constexpr int kRowsAtOnce = 4, kRowsPerGroup = kPackThreads / 16 * kRowsAtOnce;

template <typename T, int TYPE>
__global__ __launch_bounds__(kPackThreads) void f8_pack_rows(F8PackParams P) {
  const int lane16 = threadIdx.x & 15, c = blockIdx.y * kF8Group + 8 * lane16;
  const long long ldq = (P.C + kF8Group - 1) / kF8Group * (long long)kF8Group, lem = (P.M + 15) / 16 * 16;
  const int r0 = blockIdx.x * kRowsPerGroup + (int)(threadIdx.x >> 4);
  PackRun<T> run[kRowsAtOnce];
#pragma unroll
  for (int i = 0; i < kRowsAtOnce; ++i)
    run[i].load(static_cast<const T*>(P.x) + (long long)min(r0 + 16 * i, P.M - 1) * P.ldx, c, P.C);
#pragma unroll
  for (int i = 0; i < kRowsAtOnce; ++i) {
    const int r = r0 + 16 * i;
    float v[8];
    run[i].values(v);
    uint2 q;
    const int e = pack_group<TYPE>(v, q);
    if (r < P.M) *reinterpret_cast<uint2*>(P.q + (long long)r * ldq + c) = q;
    if (lane16 == 0 && r < lem) P.e[(long long)blockIdx.y * lem + r] = r < P.M ? (uint8_t)(e + 127) : 127;
  }
}

// Transposed, and by rows too where COLS is 128: a workgroup takes 128 rows x COLS columns.  COLS / 8 lanes hold a
// row's columns, which are packed by rows from there; the tile then lies in LDS, where two columns of some rows
// go to a lane, and the lanes' largest values are joined there.  (Of 64 columns alone, twice the workgroups:
// 50176 x 192 bfloat16 17.5 -> 11 us.)
template <typename T, int TYPE, int COLS>
__global__ __launch_bounds__(kPackThreads) void f8_pack(F8PackParams P) {
  constexpr int kLanes = COLS / 8, kRows = kPackThreads / kLanes, kPasses = kF8Group / kRows;  // lanes of a row, rows at a time
  constexpr int kPairs = COLS / 2, kStrips = kPackThreads / kPairs, kStrip = kF8Group / kStrips;  // a strip: a lane's rows
  constexpr int kSummed = 16;  // rows of a partial sum: sums have one order whatever COLS is
  __shared__ uint32_t most[kStrips][COLS];
  __shared__ float sums[kF8Group / kSummed][COLS];
  __shared__ uint8_t rexp[kF8Group];
  extern __shared__ __align__(16) char lds[];
  typedef T Row[kPackPitch<T, COLS>];
  Row* const tile = reinterpret_cast<Row*>(lds);
  const int r0 = blockIdx.x * kF8Group, c0 = blockIdx.y * COLS;
  const int in_row = threadIdx.x % kLanes, c = c0 + 8 * in_row;
  const long long ldq = (P.C + kF8Group - 1) / kF8Group * (long long)kF8Group, lem = (P.M + 15) / 16 * 16;
  PackRun<T> run[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i)
    run[i].load(static_cast<const T*>(P.x) + (long long)min(r0 + (int)(threadIdx.x / kLanes) + kRows * i, P.M - 1) * P.ldx, c, P.C);
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int row = (int)(threadIdx.x / kLanes) + kRows * i, r = r0 + row;
    float v[8];
    run[i].values(v);
    if (r >= P.M) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
    if constexpr (COLS == kF8Group) {
      if (P.q) {
        uint2 q;
        const int e = pack_group<TYPE>(v, q);
        if (r < P.M) *reinterpret_cast<uint2*>(P.q + (long long)r * ldq + c) = q;
        if (in_row == 0) rexp[row] = (uint8_t)(e + 127);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[row][8 * in_row + e] = from_f32<T>(v[e]);
  }
  __syncthreads();
  if (COLS == kF8Group && P.q && threadIdx.x < kF8Group && r0 + (int)threadIdx.x < lem)
    P.e[(long long)blockIdx.y * lem + r0 + threadIdx.x] = r0 + (int)threadIdx.x < P.M ? rexp[threadIdx.x] : 127;
  const int pair = threadIdx.x % kPairs, strip = threadIdx.x / kPairs;
  float v[2][kStrip];
  uint32_t m[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < kStrip; ++k)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v[j][k] = to_f32(tile[kStrip * strip + k][2 * pair + j]);
      m[j] = max(m[j], size_of(v[j][k]));
    }
#pragma unroll
  for (int j = 0; j < 2; ++j) most[strip][2 * pair + j] = m[j];
  if (P.part) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int h = 0; h < kStrip / kSummed; ++h) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kSummed; ++k) s += v[j][kSummed * h + k];
        sums[kStrip / kSummed * strip + h][2 * pair + j] = s;
      }
  }
  __syncthreads();
  if (P.part && threadIdx.x < COLS && c0 + (int)threadIdx.x < P.C) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kF8Group / kSummed; ++k) s += sums[k][threadIdx.x];
    P.part[(long long)blockIdx.x * P.C + c0 + threadIdx.x] = s;
  }
  const long long ldqt = (P.M + kF8Group - 1) / kF8Group * (long long)kF8Group, lec = (P.C + 15) / 16 * 16;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int col = 2 * pair + j;
    uint32_t a = most[0][col];
#pragma unroll
    for (int k = 1; k < kStrips; ++k) a = max(a, most[k][col]);
    const int e = exponent_of<TYPE>(a);
    if (c0 + col < P.C) {
      uint32_t w[kStrip / 4];
#pragma unroll
      for (int k = 0; k < kStrip / 4; ++k)
        w[k] = four8<TYPE>(v[j][4 * k], v[j][4 * k + 1], v[j][4 * k + 2], v[j][4 * k + 3], e);
      __builtin_memcpy(__builtin_assume_aligned(P.qt + (long long)(c0 + col) * ldqt + r0 + kStrip * strip, 16), w, kStrip);
    }
    if (strip == 0 && c0 + col < lec) P.et[(long long)blockIdx.x * lec + c0 + col] = c0 + col < P.C ? (uint8_t)(e + 127) : 127;
  }
}

template <typename T, int TYPE, int COLS>
hipError_t launch_pack_tiles(const F8PackParams& p, hipStream_t stream) {
  constexpr int kLds = kF8Group * kPackPitch<T, COLS> * (int)sizeof(T);
  static std::atomic<int> allowed{0};
  if (!allowed.load(std::memory_order_acquire)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f8_pack<T, TYPE, COLS>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    allowed.store(1, std::memory_order_release);
  }
  hipLaunchKernelGGL((f8_pack<T, TYPE, COLS>), dim3((unsigned)f8_groups(p.M), (unsigned)cdiv(p.C, COLS)),
                     dim3(kPackThreads), kLds, stream, p);
  return hipGetLastError();
}

template <typename T, int TYPE>
hipError_t launch_pack(const F8PackParams& p, hipStream_t stream) {
  if (p.qt) return p.q ? launch_pack_tiles<T, TYPE, 128>(p, stream) : launch_pack_tiles<T, TYPE, 64>(p, stream);
  hipLaunchKernelGGL((f8_pack_rows<T, TYPE>), dim3((unsigned)cdiv(p.M, kRowsPerGroup), (unsigned)f8_groups(p.C)),
                     dim3(kPackThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_pack(Dtype dt, const F8PackParams& p, hipStream_t stream) {
  if (dt == Dtype::F32) return p.type == kE4M3 ? launch_pack<float, kE4M3>(p, stream) : launch_pack<float, kE5M2>(p, stream);
  return p.type == kE4M3 ? launch_pack<uint16_t, kE4M3>(p, stream) : launch_pack<uint16_t, kE5M2>(p, stream);
}

namespace {

// Times in us, fitted to 70 products of 16 .. 60000 rows and 16 .. 8192 features and 24 weight gradients, each in every
// tile (the plans taken are within 10% of the best one measured): a workgroup's step of 128 k, alone on its CU
// and per workgroup where several share it, and its first loads and epilogue, likewise per workgroup.
struct F8Cost {
  double alone, shared, ends;
  int resident;
};
constexpr F8Cost kF8Costs[3][kF8_32x32] = {
    {{0., 0., 0., 0}, {0.9, 0.88, 2.0, 2}, {0.4, 0.37, 0.6, 4}},            // float32 results
    {{1.4, 1.98, 5.3, 1}, {0.52, 0.565, 1.7, 2}, {0.27, 0.225, 0.55, 4}},   // bfloat16
    {{0., 0., 0., 0}, {0.68, 0.43, 1.7, 2}, {0.45, 0.19, 0.55, 4}}};    // bfloat16 weight gradients, whose rows are far apart

double f8_time(const F8Cost& c, long long groups, long long steps) {
  auto round = [&](long long per_cu) {
    const double step = per_cu * c.shared > c.alone ? per_cu * c.shared : c.alone;
    return steps * step + c.ends * per_cu;
  };
  const long long slots = 256ll * c.resident, rest = groups % slots;
  return (double)(groups / slots) * round(c.resident) + (rest ? round(cdiv(rest, 256)) : 0.);
}

// Tiles of 32 x 32: a step's reads, of the rows that there are.
double f8_few_time(int M, int N, long long tiles, int steps) {
  return (double)cdiv(tiles, 256) * (0.28 + steps * 0.25 * ((M < 32 ? M : 32) + (N < 32 ? N : 32)) / 64.);
}

}  // namespace

F8Plan plan_f8(int kind, int M, int N, int K, int esize) {
  F8Plan pl{};
  MmParams& p = pl.p.mm;
  p.M = M;
  p.N = N;
  p.K = (int)f8_ld(K);
  p.steps = f8_groups(K);
  double best = -1.;
  for (int s = esize == 4 || kind == kWgrad ? kF8_128x128 : kF8_256x256; s < kF8ShapeCount; ++s) {
    const Shape& sh = kF8Shapes[s];
    const long long tm = cdiv(M, 32 * sh.tm * sh.wm), tn = cdiv(N, 32 * sh.tn * sh.wn);
    for (long long pieces = 1; pieces <= p.steps; pieces += 1 + pieces / 4) {
      const long long per = cdiv(p.steps, pieces), n = cdiv(p.steps, per);
      // (the pieces' sum: a launch, and each piece's results through memory)
      const double sum = n > 1 ? 3.5 + (double)n * M * N * 8 / 9.0e6 : 0.;
      const double t = s == kF8_32x32 ? f8_few_time(M, N, tm * tn, p.steps)
                                      : f8_time(kF8Costs[esize == 4 ? 0 : (kind == kWgrad ? 2 : 1)][s], tm * tn * n, per) + sum;
      if (best < 0. || t < best) {
        best = t;
        pl.shape = s;
        p.tm = (int)tm;
        p.tn = (int)tn;
        p.per = (int)per;
        p.nsplit = (int)n;
      }
      if (kind != kWgrad || s == kF8_32x32) break;
    }
  }
  p.nblocks = p.tm * p.tn * p.nsplit;
  pl.p.band = pl.shape == kF8_64x64 ? 8 : 4;  // (1, 4, 8, 16: 8192 x 8192 -> 8192 in 128 x 128 694, 605, 606, 622 us)
  return pl;
}

}  // namespace rows
}  // namespace o1d
