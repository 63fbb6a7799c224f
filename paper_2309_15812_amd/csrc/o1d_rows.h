// Host-side plans and launchers of the row operators: layer norm, the matrix
// product with an epilogue and its gradients, and 8-bit checkpoints.  All act on
// matrices of M rows (pixels or tokens, channels last) whose features are
// contiguous; rows are `ld` elements apart.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "o1d_launch.h"

namespace o1d {
namespace rows {

inline long long cdiv(long long a, long long b) { return (a + b - 1) / b; }

// ---- 8-bit checkpoints: groups of 64 columns of a row share a scale; the
// integers' rows are padded to 16 bytes.
constexpr int kGroup = 64;
inline long long held_ld(int C) { return cdiv(C, 16) * 16; }
inline int held_groups(int C) { return (int)cdiv(C, kGroup); }

struct Held {
  int8_t* q;
  float* scale;
};

// A matrix operand: its elements (rows ld apart), or its 8-bit checkpoint.
struct Operand {
  const void* p;
  long long ld;
  const int8_t* q;  // not NULL: the checkpoint
  const float* scale;
};

enum Act { kNone = 0, kRelu = 1, kGelu = 2, kGeluTanh = 3, kSilu = 4, kActs = 5 };

// ---- layer norm

struct LnParams {
  int M, C;
  long long ldx, ldy, lddx;  // ldy: y's (forward) or dy's (backward)
  float eps;
  const void *x, *w, *b, *dy;
  const int8_t* xq;
  const float* xscale;
  void *y, *dx, *dw, *db;
  float *mean, *rstd;         // written by the forward, read by the backward
  float* part;                // backward: partial sums, blocks x 2 x C
  int blocks;
};

// Layouts of a row: `lanes` lanes with `runs` 16-byte runs each (lanes 0: too
// long for a wave).  The forward's: the fewest lanes that hold it in four
// runs each, up to a wave with eight.
struct LnMap {
  int lanes, runs;
};
inline LnMap ln_fwd_map(int C, int esize) {
  const long long total = cdiv(C, 16 / esize);
  int lanes = 4;
  while (lanes < 64 && total > 4 * lanes) lanes *= 2;
  const int runs = (int)cdiv(total, lanes);
  return runs <= 8 ? LnMap{lanes, runs} : LnMap{0, 0};
}

// The backward's: `lanes` lanes with `runs` 16-byte runs each
// (lanes 0: too long for a wave).  Few runs per lane leave registers for more
// waves and make the sums over a workgroup's rows short; lanes past the row's
// end do nothing.  33333 x 211 bfloat16: 8 lanes x 4 runs 24 us, 32 x 1 15 us.
inline LnMap ln_bwd_map(int C, int esize) {
  const long long total = cdiv(C, 16 / esize);
  LnMap best{0, 0};
  float score = 0.f;
  for (int lanes = 4; lanes <= 64; lanes *= 2) {
    const long long runs = cdiv(total, lanes);
    if (runs > (lanes == 64 ? 8 : 3)) continue;
    const float s = (float)total / (float)(lanes * runs) * (runs == 1 ? 1.f : (runs == 2 ? 0.95f : 0.85f));
    if (s >= score) {
      score = s;
      best = {lanes, (int)runs};
    }
  }
  return best;
}
constexpr int ln_bwd_waves(int runs) { return runs <= 2 ? 8 : 4; }

// Workgroups of the backward, each of which leaves one partial row of dw and db:
// two per CU at most, with about the same number of rows each.
constexpr int kLnMostBlocks = 512;  // (1024: 33333 x 211 bfloat16 1.15 times, 50176 x 192 1.28 times the time)
inline int ln_bwd_blocks(int M, int C, int esize) {
  const LnMap m = ln_bwd_map(C, esize);
  if (!m.lanes) return M < 2 ? 2 : (M < 256 ? M : 256);
  const long long blocks = cdiv(M, 64 / m.lanes * ln_bwd_waves(m.runs));
  if (blocks <= 4) return 1;  // one workgroup, whose sums are dw and db: no second launch
  if (blocks <= kLnMostBlocks) return (int)blocks;
  return (int)cdiv(blocks, cdiv(blocks, kLnMostBlocks));
}

hipError_t launch_ln_fwd_f32(const LnParams& p, hipStream_t stream);
hipError_t launch_ln_fwd_bf16(const LnParams& p, hipStream_t stream);
hipError_t launch_ln_bwd_f32(const LnParams& p, hipStream_t stream);
hipError_t launch_ln_bwd_bf16(const LnParams& p, hipStream_t stream);

// out[c] = sum over j < parts of part[j ld + c], c < C, in a fixed order; two
// such sums side by side (the second at part + C) where out2 is given.
hipError_t launch_col_sum(Dtype dt, const float* part, int parts, long long ld, int C, void* out, void* out2,
                          hipStream_t stream);

// ---- checkpoints

hipError_t launch_pack(Dtype dt, const void* x, long long ldx, int M, int C, const Held& h, hipStream_t stream);
// y = act(x) (dy NULL) or dy act'(x)
hipError_t launch_act(Dtype dt, const Operand& x, const void* dy, long long lddy, int M, int C, int act, void* y,
                      long long ldy, hipStream_t stream);

// ---- products  C[m][n] = sum_k A[m][k] B[n][k]
//
//   kFwd    y  = x W^T     m rows of x,  n = output feature, k = input feature
//   kDgrad  dx = dy W      m rows of dy, n = input feature,  k = output feature
//   kWgrad  dW = dy^T x    m = output feature, n = input feature, k = row
enum Kind { kFwd = 0, kDgrad = 1, kWgrad = 2 };

struct MmParams {
  int M, N, K;
  const void *a, *b;
  long long lda, ldb;
  int tm, tn;           // tiles along m and n
  int steps, per;       // k steps in all and per piece
  int nsplit;           // weight gradient: pieces of k
  int nblocks;
  // epilogues
  int act;                              // (weight gradient: of b, with made)
  const int8_t* bq;                     // weight gradient: b's checkpoint
  int made;                             // weight gradient: b is act(x) of a tensor or a checkpoint, made as it is staged
  const void* bias;                     // forward
  const void* res; long long ldres;     // forward
  void* out; long long ldo;             // forward, input gradient
  void* pre; long long ldpre;           // forward: written; input gradient: read
  int8_t* q; float* scale;              // the same in 8 bits
  long long ldq; int groups;
  float* part;                          // weight gradient: nsplit x (M N + M), or (one piece) out and
  void* db;
  int want_db;
};

// Workgroup tiles: wm x wn waves, each 32 tm x 32 tn.
struct Shape {
  int wm, wn, tm, tn;
};

struct MmPlan {
  bool few;   // the kernels of few rows; else
  int shape;  // index into kShapes
  MmParams p;
};

enum ShapeId { k128x128, k64x64, k128x96, k64x128, k128x64, k128x192, k128x32, k32x128, k192x64, kShapeCount };
constexpr Shape kShapes[kShapeCount] = {{2, 2, 2, 2}, {2, 2, 1, 1}, {4, 1, 1, 3}, {2, 2, 1, 2},
                                         {4, 1, 1, 2}, {2, 2, 2, 3}, {4, 1, 1, 1}, {1, 4, 1, 1}, {2, 2, 3, 1}};
// Tiles that are planned, by what they measured: 128 x 192 for float32 alone, 128 x
// 96 not for bfloat16 weight gradients, of which narrow ones gain nothing from 128 x
// 32 and 32 x 128 either; 192 x 64 for weight gradients that make
// their operand.
constexpr bool shape_used(int kind, int esize, int shape) {
  switch (shape) {
    case k128x96: return kind != kWgrad || esize == 4;
    case k128x128:
    case k64x64:
    case k128x64: return true;
    case k128x32: return kind != kWgrad || esize == 4;
    case k32x128: return kind == kWgrad && esize == 4;
    case k64x128: return kind == kWgrad || esize == 2;
    case k128x192: return esize == 4;
    default: return false;
  }
}
constexpr int kStepBytes = 128;  // k per step: 32 float32 or 64 bfloat16

// Whole 16-byte runs: along k where an operand is contiguous along it, else along its rows.
inline bool whole_runs(int kind, int M, int N, int K, const void* a, long long lda, const void* b, long long ldb, int esize) {
  const int v = 16 / esize;
  auto aligned = [&](const void* t, long long ld) { return (uintptr_t)t % 16 == 0 && ld % v == 0; };
  return (kind == kWgrad ? M : K) % v == 0 && (kind == kFwd ? K : N) % v == 0 && aligned(a, lda) && aligned(b, ldb);
}

// A forward product's or input gradient's plan.  `groups`: an 8-bit checkpoint is
// written (waves with 64 columns).  `whole`: whole_runs.
MmPlan plan_mm(int kind, int M, int N, int K, int esize, bool groups, bool whole);

// A weight gradient's plan, which sizes its workspace (and does not go by the
// addresses).  `made`: the product makes act(x), of a tensor or a checkpoint
// (`held`), itself as it stages it, once per tile along m, instead of reading it
// from a pass of its own (a launch, and act(x) through memory).
MmPlan plan_wgrad(int M, int N, int K, int esize, bool held, int act, bool& made);

#define O1D_MM_DECL(T)                                                                    \
  hipError_t launch_mm_fwd_##T(const MmPlan& pl, hipStream_t stream);                     \
  hipError_t launch_mm_dgrad_##T(const MmPlan& pl, hipStream_t stream);                   \
  hipError_t launch_mm_wgrad_##T(const MmPlan& pl, hipStream_t stream);
O1D_MM_DECL(f32)
O1D_MM_DECL(bf16)
#undef O1D_MM_DECL
hipError_t launch_mmf_fwd_bf16(const MmPlan& pl, hipStream_t stream);
hipError_t launch_mmf_dgrad_bf16(const MmPlan& pl, hipStream_t stream);
hipError_t launch_mmf_wgrad_bf16(const MmPlan& pl, hipStream_t stream);

hipError_t launch_few_f32(int kind, const MmParams& p, hipStream_t stream);
hipError_t launch_few_bf16(int kind, const MmParams& p, hipStream_t stream);

// The product's kernel: of whole aligned runs where the operands have those.
hipError_t launch_mm(Dtype dt, int kind, const MmPlan& pl, hipStream_t stream);

// dw[i] = sum of the pieces' partials (i < M N), db[o] likewise behind them.
// (wide_sum: of four columns per thread)
inline bool wide_sum(int pieces, long long outputs) { return pieces <= 4 || outputs >= (1 << 18); }
hipError_t launch_mm_sum(Dtype dt, const MmPlan& pl, void* dw, void* db, hipStream_t stream);

}  // namespace rows
}  // namespace o1d
