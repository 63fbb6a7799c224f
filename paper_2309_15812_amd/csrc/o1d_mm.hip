// Plan of the matrix products of rows, and the sum of the weight gradient's
// partial results.
#include <hip/hip_runtime.h>

#include "o1d_device.h"
#include "o1d_rows.h"
#include "o1d_rows_device.h"

namespace o1d {
namespace rows {

namespace {

// Time of a product as rounds of resident workgroups, each with a time of its
// own and a time per step of 128 bytes of k (microseconds).  Forward products and input
// gradients: measured at 3400 sizes of 16 .. 200704 rows and 16 .. 2048 features with
// each tile; the model fits within 16 to 19%, the plan it takes is 2 to 3% from
// the best measured one.
struct Cost {
  float first, step;
  int resident;  // workgroups of a CU
};
constexpr double kLaunch = 2.3, kAlone = 0.25;  // (the time of a CU's only workgroup, as a share)
constexpr Cost kCost[3][kShapeCount] = {
    // float32: 128 x 128, 64 x 64, 128 x 96, 64 x 128, 128 x 64, 128 x 192, 128 x 32, 32 x 128
    {{12.8f, 3.05f, 2}, {5.2f, 2.15f, 4}, {9.0f, 2.55f, 2}, {}, {8.4f, 2.7f, 3}, {23.f, 3.9f, 2}, {4.4f, 2.15f, 3}},
    // bfloat16, whole runs
    {{7.7f, 1.08f, 2}, {2.85f, 0.66f, 3}, {5.8f, 0.93f, 2}, {5.6f, 0.94f, 3}, {5.6f, 1.03f, 3}, {}, {3.2f, 0.86f, 3}},
    // bfloat16, other runs
    {{9.5f, 1.6f, 2}, {4.5f, 1.1f, 4}, {6.5f, 1.44f, 2}, {6.7f, 1.43f, 3}, {7.2f, 1.44f, 3}, {}, {4.7f, 1.46f, 4}}};

// Weight gradients in the same terms, measured at 1100 sizes of 300 .. 200704
// rows with 2 to 12 numbers of pieces for each tile (the model fits within 7 to
// 12%; the plan it takes is 3 to 5% from the best measured one.  As many pieces
// as make about 512 workgroups, and the tile by its area alone, was 11 to 14%).
constexpr Cost kWgradCost[3][kShapeCount] = {
    {{1.f, 3.1f, 2}, {0.f, 2.1f, 4}, {0.f, 2.6f, 2}, {0.f, 2.8f, 3}, {0.f, 2.65f, 3}, {2.7f, 4.5f, 2}, {0.f, 2.13f, 3},
     {0.f, 2.08f, 3}},
    {{0.f, 1.04f, 2}, {0.f, 0.62f, 3}, {}, {0.f, 0.92f, 3}, {0.f, 0.91f, 3}},
    {{0.f, 1.64f, 2}, {0.f, 1.19f, 4}, {}, {0.f, 1.42f, 3}, {0.f, 1.41f, 3}}};
// Those that make their operand, 64 x 64 and 192 x 64: a step's time by activation
// (none, relu, gelu, gelu_tanh, silu).  50176 x 768 -> 192 bfloat16 from a checkpoint
// with GELU: 55 to 58 us against 68 with a pass of its own.
constexpr int kMadeShapes[2] = {k64x64, k192x64}, kMadeResident[2][2] = {{4, 2}, {4, 3}};
constexpr float kMadeStep[2][2][kActs] = {{{2.5f, 2.5f, 3.6f, 3.4f, 3.35f}, {3.5f, 3.5f, 4.4f, 4.3f, 4.0f}},
                                          {{1.6f, 1.75f, 2.3f, 2.1f, 1.95f}, {2.75f, 3.0f, 3.25f, 3.15f, 3.05f}}};
constexpr double kWgradLaunch = 3.5, kWgradAlone = 0.4;
constexpr double kSumEach = 0.02, kSumElement = 1.3e-6;  // the sum of the pieces: per piece, per element
constexpr double kPassBytes = 4e6;                       // a pass of its own: bytes per microsecond

double rounds(const Cost& c, long long blocks, double steps, double alone) {
  // (a last round of fewer workgroups per CU is shorter)
  const long long slots = 256 * c.resident, rest = blocks % slots;
  double t = (double)(blocks / slots) * (c.first + c.step * steps);
  if (rest) t += (c.first + c.step * steps) * (alone + (1. - alone) * (double)cdiv(rest, 256) / c.resident);
  return t;
}

// Time of the kernels of few rows (measured at the same sizes): a launch, the
// waits of a workgroup's waves for their pieces of 32 k, of which a launch that
// fills the GPU once hides none, and the workgroups' own work.
struct FewCost {
  double launch, piece, each, work;
};
constexpr FewCost kFewCost[3][2] = {{{3.4, 0.27, 0.0072, 0.00093}, {4.0, 0.75, 0.012, 0.00325}},   // float32; with a checkpoint
                                    {{3.3, 0.09, 0.0047, 0.00035}, {3.5, 0.29, 0.009, 0.00078}},  // bfloat16, whole runs
                                    {{3.4, 0.31, 0.006, 0.0004}, {3.5, 1.0, 0.011, 0.001}}};
constexpr int kFewMost = 1 << 16;
double few_cost(int M, int N, int K, int type, bool groups) {
  const FewCost& c = kFewCost[type][groups];
  const double pieces = (double)cdiv(K, 32), wgs = (double)cdiv(N, groups ? 64 : 16) * (double)cdiv(M, 64);
  const double share = M <= 16 ? 0.35 : (M <= 32 ? 0.6 : 1.);
  return c.launch + c.piece * share * pieces + wgs * share * (c.each + c.work * pieces);
}

// Takes the tile for a weight gradient, with its k in the pieces that cost least
// (numbers that just fill the GPU, of at least three steps), if it costs less than `best`.
void try_wgrad(MmPlan& pl, int shape, const Cost& c, double& best) {
  MmParams& p = pl.p;
  const Shape& sh = kShapes[shape];
  const long long tm = cdiv(p.M, 32 * sh.tm * sh.wm), tn = cdiv(p.N, 32 * sh.tn * sh.wn), tiles = tm * tn;
  const long long most = p.steps >= 8 ? p.steps / 3 : 1;
  for (int fill = 1; fill <= 2 * c.resident; ++fill) {
    long long pieces = 256 * fill / tiles;
    pieces = pieces > most ? most : (pieces < 1 ? 1 : pieces);
    const long long per = cdiv(p.steps, pieces);
    pieces = cdiv(p.steps, per);
    const double sum = pieces > 1 ? kWgradLaunch + (double)pieces * (kSumEach + kSumElement * p.M * p.N) : 0.;
    const double cost = kWgradLaunch + rounds(c, tiles * pieces, (double)per, kWgradAlone) + sum;
    if (best >= 0 && cost >= best) continue;
    best = cost;
    pl.shape = shape;
    p.tm = (int)tm;
    p.tn = (int)tn;
    p.per = (int)per;
    p.nsplit = (int)pieces;
    p.nblocks = (int)(tiles * pieces);
  }
}

}  // namespace

MmPlan plan_mm(int kind, int M, int N, int K, int esize, bool groups, bool whole) {
  MmPlan pl{};
  MmParams& p = pl.p;
  p.M = M;
  p.N = N;
  p.K = K;
  p.steps = (int)cdiv(K, kStepBytes / esize);
  p.nsplit = 1;
  p.per = p.steps;
  const int type = esize == 4 ? 0 : (whole ? 1 : 2);
  double best = -1.;
  for (int s = 0; s < kShapeCount; ++s) {
    const Shape& sh = kShapes[s];
    if ((groups && sh.tn % 2) || !shape_used(kind, esize, s)) continue;
    const long long tm = cdiv(M, 32 * sh.tm * sh.wm), tn = cdiv(N, 32 * sh.tn * sh.wn);
    const double cost = kLaunch + rounds(kCost[type][s], tm * tn, (double)p.steps, kAlone);
    if (best >= 0 && cost >= best) continue;
    best = cost;
    pl.shape = s;
    p.tm = (int)tm;
    p.tn = (int)tn;
  }
  pl.few = M <= kFewMost && few_cost(M, N, K, type, groups) < best;
  p.nblocks = p.tm * p.tn;
  return pl;
}

MmPlan plan_wgrad(int M, int N, int K, int esize, bool held, int act, bool& made) {
  MmPlan pl{};
  MmParams& p = pl.p;
  p.M = M;
  p.N = N;
  p.K = K;
  p.steps = (int)cdiv(K, kStepBytes / esize);
  const bool whole = M % (16 / esize) == 0 && N % (16 / esize) == 0;
  double best = -1.;
  for (int s = 0; s < kShapeCount; ++s)
    if (shape_used(kWgrad, esize, s)) try_wgrad(pl, s, kWgradCost[esize == 4 ? 0 : (whole ? 1 : 2)][s], best);
  made = false;
  if (!held && act == kNone) return pl;
  // act(x) from a pass of its own (its launch, x read, act(x) written), or made
  const double before = best += kWgradLaunch + (double)K * N * ((held ? 1 : esize) + esize) / kPassBytes;
  for (int i = 0; i < 2; ++i) {
    const int type = esize == 2;
    try_wgrad(pl, kMadeShapes[i], {0.f, kMadeStep[type][i][act], kMadeResident[type][i]}, best);
  }
  made = best < before;
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

// The same where every thread has pieces enough to wait for at once, or there are
// outputs enough to fill the GPU: four columns per thread, all pieces.
// 2048 x 2048 in two pieces: 28 us above, 7.4 (float32 8.7) here.
constexpr int kWideColumns = 4;

template <typename T>
__global__ __launch_bounds__(kThreads) void mm_sum_wide(const float* __restrict__ part, int pieces, long long MN, int M,
                                                        T* __restrict__ dw, T* __restrict__ db) {
  const long long width = MN + M, i = ((long long)blockIdx.x * kThreads + threadIdx.x) * kWideColumns;
  const long long left = (db ? width : MN) - i;
  if (left <= 0) return;
  const int n = left < kWideColumns ? (int)left : kWideColumns;
  constexpr int kBatch = 4;
  float s[kWideColumns] = {};
  for (int j0 = 0; j0 < pieces; j0 += kBatch) {
    float v[kBatch][kWideColumns] = {};
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (j0 + u < pieces) load_some(part + (long long)(j0 + u) * width + i, n, v[u]);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int e = 0; e < kWideColumns; ++e) s[e] += v[u][e];
  }
  if (i + n <= MN) {
    store_some(dw + i, n, s);
  } else {
#pragma unroll
    for (int e = 0; e < kWideColumns; ++e) {
      if (e >= n) break;
      if (i + e < MN)
        dw[i + e] = from_f32<T>(s[e]);
      else
        db[i + e - MN] = from_f32<T>(s[e]);
    }
  }
}

template <typename T>
void launch_sum(const MmPlan& pl, T* dw, T* db, hipStream_t stream) {
  const long long MN = (long long)pl.p.M * pl.p.N, outputs = MN + (db ? pl.p.M : 0);
  if (wide_sum(pl.p.nsplit, outputs))
    hipLaunchKernelGGL(mm_sum_wide<T>, dim3((unsigned)cdiv(outputs, kThreads * kWideColumns)), dim3(kThreads), 0, stream,
                       pl.p.part, pl.p.nsplit, MN, pl.p.M, dw, db);
  else
    hipLaunchKernelGGL(mm_sum<T>, dim3((unsigned)cdiv(outputs, kSumColumns)), dim3(kThreads), 0, stream, pl.p.part,
                       pl.p.nsplit, MN, pl.p.M, dw, db);
}

}  // namespace

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
  if (dt == Dtype::F32)
    launch_sum(pl, static_cast<float*>(dw), static_cast<float*>(db), stream);
  else
    launch_sum(pl, static_cast<uint16_t*>(dw), static_cast<uint16_t*>(db), stream);
  return hipGetLastError();
}

}  // namespace rows
}  // namespace o1d
