// Plan of the matrix products of rows, and the sum of the weight gradient's
// partial results.
#include <hip/hip_runtime.h>

#include "o1d_device.h"
#include "o1d_rows.h"

namespace o1d {
namespace rows {

namespace {

// Time of a product as rounds of resident workgroups, each with a time of its
// own and a time per step of 128 bytes of k (microseconds, measured over
// 784 .. 200704 rows and 96 .. 2048 features; they fit within about 15%).
struct Cost {
  float first, step;
  int resident;  // workgroups of a CU
};
constexpr Cost kCost[3][kShapeCount] = {
    // float32: 128 x 128, 64 x 256, 64 x 64, 128 x 96, 64 x 128, 128 x 64, 128 x 192
    {{5.f, 3.0f, 2}, {}, {5.f, 1.9f, 4}, {7.f, 1.9f, 2}, {}, {6.5f, 2.2f, 3}, {8.f, 4.f, 2}, {}},
    // bfloat16, whole runs
    {{3.7f, 0.90f, 2}, {}, {3.3f, 0.45f, 3}, {3.0f, 0.72f, 2}, {3.0f, 0.68f, 3}, {3.0f, 0.68f, 3}},
    // bfloat16, other runs
    {{10.f, 1.2f, 2}, {}, {6.f, 0.8f, 4}, {7.f, 0.9f, 2}, {10.f, 1.f, 3}, {10.f, 1.f, 3}}};

// Weight gradients run as many pieces as fill the GPU whatever the tile, so
// the tile that computes least past the output's edge is taken, weighted by
// the time of its products (float32: smaller tiles make more pieces per product).
constexpr float kArea[2][kShapeCount] = {{1.f, 1.02f, 1.5f, 1.15f, 1.3f, 1.3f, 1.1f}, {0.f, 0.f, 1.3f, 0.f, 1.f, 1.f}};
constexpr int kWgradBlocks = 512;

// Time of the kernels of few rows (microseconds, measured as above for 1 .. 2000
// rows): the waits of a workgroup's waves for their pieces of 32 k, of which
// a launch that fills the GPU once hides none, and the workgroups' own work.
constexpr int kFewMost = 1 << 16;
double few_cost(int M, int N, int K, int esize, bool groups) {
  const double pieces = (double)cdiv(K, 32), wgs = (double)cdiv(N, groups ? 64 : 16) * (double)cdiv(M, 64);
  const double share = M <= 16 ? 0.35 : (M <= 32 ? 0.6 : 1.), waves = groups ? 3. : 1.;
  return esize == 2 ? 3.3 + 0.14 * share * waves * pieces + wgs * share * (0.003 + 0.0005 * pieces)
                    : 3.5 + 0.33 * share * waves * pieces + wgs * share * (0.006 + 0.001 * pieces);
}
// A weight gradient's k in pieces of at least four steps.
void split_steps(MmParams& p, int blocks = kWgradBlocks) {
  const long long want = cdiv(blocks, (long long)p.tm * p.tn), most = p.steps / 4;
  const long long pieces = want < most ? want : most;
  p.per = (int)cdiv(p.steps, pieces > 1 ? pieces : 1);
  p.nsplit = (int)cdiv(p.steps, p.per);
  p.nblocks = p.tm * p.tn * p.nsplit;
}

}  // namespace

MmPlan plan_mm(int kind, int M, int N, int K, int esize, bool groups, bool whole) {
  MmPlan pl{};
  MmParams& p = pl.p;
  p.M = M;
  p.N = N;
  p.K = K;
  p.steps = (int)cdiv(K, kStepBytes / esize);
  const int type = esize == 2 ? 1 : 0;
  double best = -1.;
  for (int s = 0; s < kShapeCount; ++s) {
    const Shape& sh = kShapes[s];
    if ((groups && sh.tn % 2) || !shape_used(kind, esize, s)) continue;
    const int bm = 32 * sh.tm * sh.wm, bn = 32 * sh.tn * sh.wn;
    const long long tm = cdiv(M, bm), tn = cdiv(N, bn), tiles = tm * tn;
    double cost;
    if (kind == kWgrad) {
      const long long pieces = p.steps / 4 > 1 ? p.steps / 4 : 1, blocks = tiles * pieces;
      cost = (double)tiles * bm * bn * kArea[type][s] * (blocks < 256 ? 256. / (double)blocks : 1.);
    } else {
      const Cost& c = kCost[type && !whole ? 2 : type][s];
      // (a last round of fewer workgroups per CU has shorter steps)
      const long long slots = 256 * c.resident, rest = tiles % slots;
      cost = (double)(tiles / slots) * (c.first + c.step * p.steps);
      if (rest) cost += c.first + c.step * p.steps * (0.4 + 0.6 * (double)cdiv(rest, 256) / c.resident);
    }
    if (best < 0 || cost < best) {
      best = cost;
      pl.shape = s;
      p.tm = (int)tm;
      p.tn = (int)tn;
    }
  }
  pl.few = kind != kWgrad && M <= kFewMost && few_cost(M, N, K, esize, groups) < best;
  p.nsplit = 1;
  p.per = p.steps;
  if (kind == kWgrad) {
    split_steps(p);
  }
  p.nblocks = p.tm * p.tn * p.nsplit;
  return pl;
}

namespace {

// A workgroup's threads are kSumColumns outputs x kSumSlices slices of the
// pieces, each slice added in order, then the slices: with all pieces in one thread
// the sum waited for memory once per sixteen of them (28 pieces of 192 x 768 6.5 us).
constexpr int kSumColumns = 64, kSumSlices = kThreads / kSumColumns;

template <typename T>
__global__ __launch_bounds__(kThreads) void mm_sum(const float* __restrict__ part, int pieces, long long MN, int M,
                                                   T* __restrict__ dw, T* __restrict__ db) {
  __shared__ float red[kSumSlices][kSumColumns];
  const long long width = MN + M;
  const int col = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
  const long long i = (long long)blockIdx.x * kSumColumns + col;
  const bool in = i < (db ? width : MN);
  constexpr int kBatch = 8;
  float s = 0.f;
  if (in) {
    for (int j0 = slice; j0 < pieces; j0 += kSumSlices * kBatch) {
      float v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        v[u] = j0 + u * kSumSlices < pieces ? part[(long long)(j0 + u * kSumSlices) * width + i] : 0.f;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) s += v[u];
    }
  }
  red[slice][col] = s;
  __syncthreads();
  if (slice || !in) return;
#pragma unroll
  for (int k = 1; k < kSumSlices; ++k) s += red[k][col];
  if (i < MN)
    dw[i] = from_f32<T>(s);
  else
    db[i - MN] = from_f32<T>(s);
}

}  // namespace

bool make_operand(MmPlan& pl, int act, bool held, int esize) {
  // Picoseconds per element: of the product that makes it (none, relu, gelu,
  // gelu_tanh, silu), above the plain product's; and of writing it and reading it
  // back.  50176 x 768 -> 192 bfloat16 from a checkpoint with GELU: 58 us against
  // 68 with a pass of its own, 200704 x 384 -> 96 96 against 93.
  constexpr double kMade[2][kActs] = {{1.2, 1.2, 3.5, 3.0, 3.0}, {0.9, 0.95, 1.05, 1.05, 1.0}};
  constexpr double kLaunch = 3e6;
  MmParams& p = pl.p;
  const double elements = (double)p.K * p.N, wide = (double)cdiv(p.M, 192), narrow = (double)cdiv(p.M, 64);
  const double per = kMade[esize == 2 ? 1 : 0][act], apart = elements * ((held ? 1. : esize) + 2. * esize) / 5. + kLaunch;
  const bool small = elements * narrow * per < kLaunch;
  if (!small && elements * wide * per > apart) return false;
  // 64 x 64 tiles where there are few, else those that make an element least often
  const int shape = small && cdiv(p.M, 192) * cdiv(p.N, 64) * (p.steps / 4) < 256 ? k64x64 : k192x64;
  const Shape& sh = kShapes[shape];
  pl.shape = shape;
  p.tm = (int)cdiv(p.M, 32 * sh.tm * sh.wm);
  p.tn = (int)cdiv(p.N, 32 * sh.tn * sh.wn);
  split_steps(p, 768);  // (three resident workgroups per CU)
  return true;
}

hipError_t launch_mm(Dtype dt, int kind, const MmPlan& pl, hipStream_t stream) {
  if (pl.few) return dt == Dtype::F32 ? launch_few_f32(kind, pl.p, stream) : launch_few_bf16(kind, pl.p, stream);
  if (dt == Dtype::BF16 && !pl.p.made && whole_runs(kind, pl.p.M, pl.p.N, pl.p.K, pl.p.a, pl.p.lda, pl.p.b, pl.p.ldb, 2)) {
    return kind == kFwd ? launch_mmf_fwd_bf16(pl, stream)
                        : (kind == kDgrad ? launch_mmf_dgrad_bf16(pl, stream) : launch_mmf_wgrad_bf16(pl, stream));
  }
  if (dt == Dtype::F32)
    return kind == kFwd ? launch_mm_fwd_f32(pl, stream)
                        : (kind == kDgrad ? launch_mm_dgrad_f32(pl, stream) : launch_mm_wgrad_f32(pl, stream));
  return kind == kFwd ? launch_mm_fwd_bf16(pl, stream)
                      : (kind == kDgrad ? launch_mm_dgrad_bf16(pl, stream) : launch_mm_wgrad_bf16(pl, stream));
}

hipError_t launch_mm_sum(Dtype dt, const MmPlan& pl, void* dw, void* db, hipStream_t stream) {
  const long long MN = (long long)pl.p.M * pl.p.N, width = MN + (db ? pl.p.M : 0);
  const dim3 grid((unsigned)cdiv(width, kSumColumns)), block(kThreads);
  if (dt == Dtype::F32)
    hipLaunchKernelGGL(mm_sum<float>, grid, block, 0, stream, pl.p.part, pl.p.nsplit, MN, pl.p.M, static_cast<float*>(dw),
                       static_cast<float*>(db));
  else
    hipLaunchKernelGGL(mm_sum<uint16_t>, grid, block, 0, stream, pl.p.part, pl.p.nsplit, MN, pl.p.M,
                       static_cast<uint16_t*>(dw), static_cast<uint16_t*>(db));
  return hipGetLastError();
}

}  // namespace rows
}  // namespace o1d
