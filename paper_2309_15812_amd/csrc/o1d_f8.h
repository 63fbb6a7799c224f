// Host-side plans and launchers of the products of 8-bit floating point operands
// with a power-of-two scale for each 128 values of a row, and of their packing.
#pragma once

#include "o1d_rows.h"

namespace o1d {
namespace rows {

// An operand of R rows of K values: q[R][f8_ld(K)] (zeros behind a row's end) and
// exponents e[f8_groups(K)][f8_le(R)] (127 behind the last row); value k of row r
// stands for q[r][k] 2^(e[k / 128][r] - 127).
constexpr int kF8Group = 128;
inline int f8_groups(int K) { return (int)cdiv(K, kF8Group); }
inline long long f8_ld(int K) { return cdiv(K, kF8Group) * kF8Group; }
inline long long f8_le(int R) { return cdiv(R, 16) * 16; }

enum F8Type { kE4M3 = 0, kE5M2 = 1 };

struct F8PackParams {
  const void* x;  // M rows of C values, ldx apart
  long long ldx;
  int M, C, type;
  uint8_t *q, *e;    // by rows (or NULL): groups along the columns
  uint8_t *qt, *et;  // transposed (or NULL): C rows of M values, groups along x's rows
  float* part;       // (or NULL) column sums of each 128 rows of x
};
hipError_t launch_f8_pack(Dtype dt, const F8PackParams& p, hipStream_t stream);

// C[m][n] = sum_k A[m][k] B[n][k], both operands in 8 bits along k.  `mm` as
// for the other products (a, b, lda and ldb are the operands' q).
struct F8MmParams {
  MmParams mm;
  const uint8_t *ea, *eb;
  long long lea, leb;
  int band;  // rows of tiles that are taken together
};
enum F8ShapeId { kF8_256x256, kF8_128x128, kF8_64x64, kF8_32x32, kF8ShapeCount };
constexpr Shape kF8Shapes[kF8ShapeCount] = {{2, 4, 4, 2}, {2, 2, 2, 2}, {2, 2, 1, 1}, {1, 1, 1, 1}};
// (Tiles of 32 x 32 are of another kernel, whose waves each take steps of their own.)

struct F8Plan {
  int shape, atype;
  F8MmParams p;
};
// kFwd or kDgrad (which differ in their epilogue), or kWgrad (pieces of k; no tiles of 256 x 256, whose rows far apart it reads no
// faster).
F8Plan plan_f8(int kind, int M, int N, int K, int esize);

#define O1D_F8_DECL(T)                                                   \
  hipError_t launch_f8_fwd_##T(const F8Plan& pl, hipStream_t stream);    \
  hipError_t launch_f8_dgrad_##T(const F8Plan& pl, hipStream_t stream);  \
  hipError_t launch_f8_wgrad_##T(const F8Plan& pl, hipStream_t stream);
O1D_F8_DECL(f32)
O1D_F8_DECL(bf16)
#undef O1D_F8_DECL

}  // namespace rows
}  // namespace o1d
