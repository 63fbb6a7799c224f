// Host-side plan and launchers of group norm with an activation on channels-last activations.
#pragma once

#include "o1d_rows.h"

namespace o1d {
namespace rows {

struct GnParams {
  int N, P, C, G, D;        // samples, pixels of one, channels = G groups of D
  uint32_t over_d;          // 2^32 / D rounded up (D > 1)
  long long ldx, ldy, ldd;  // rows apart: of x, of y (forward) or dx, of dy
  float eps;
  int act;
  const void *x, *w, *b, *dy;
  void* out;                // y or dx
  float *mean, *rstd;       // N x G: written by the forward, read by the backward
  float* part;              // partial results (below)
  void *dw, *db;
  int gb, bundles;          // groups of a workgroup's channels, and how many such pieces
  int chunks, rows;         // not held: pieces of a sample's pixels, and their rows (the last may have fewer)
};

// A workgroup's channels are the `gb` groups of a bundle.  Held: it holds all
// pixels of a sample in registers (`runs` 16-byte runs of `threads` threads) and memory is
// passed once.  Else a first pass leaves partial statistics of each chunk of
// pixels, and a second reads the chunk again.
struct GnPlan {
  bool held;
  int threads, runs;
  int gb, bundles, chunks, rows;
};
constexpr int kGnMostChannels = 1024;  // of a group
constexpr int kGnMostChunks = 512;     // of a sample
constexpr int kGnThreads = 256, kGnBatch = 8;  // in chunks: threads of a workgroup, most rows that a thread takes at a time
// A row of a sample in chunks.  A thread's next rows are worked out before they are compared with the chunk's end, up to
// kGnThreads kGnBatch = 2048 behind it; an int has room for 1024 behind the longest sample, and kept to that
// only by how the plan divides one (the furthest row was 2^31 - 364).
using GnRow = uint32_t;
// The k-th of a thread's next rows from r on, `slots` apart, or the chunk's last one.
__host__ __device__ __forceinline__ GnRow gn_row(GnRow r, int k, int slots, GnRow end) {
  const GnRow at = r + (GnRow)(k * slots);
  return at < end ? at : end - 1;
}
// Threads of the larger workgroups and most runs of a held sample: in bfloat16 the backward unpacks its
// registers twice and needs 256 of them per thread.
constexpr int gn_big(bool backward, int esize) { return backward && esize == 2 ? 512 : 1024; }
constexpr int gn_most_runs(bool backward, int esize) { return backward ? (esize == 2 ? 6 : 8) : 10; }
// The runs (even) that a workgroup's threads may have.  (Two of 512 threads are five of 256 at most.)
constexpr bool gn_takes(bool backward, int esize, int threads, int runs) {
  return runs <= (threads == 64 ? 4 : gn_most_runs(backward, esize)) && !(threads == 512 && runs == 2);
}
// Between the passes a wave joins a sample's group, and the groups behind the grid's last one in turn: all of them would
// be more than the fewer than 2^32 threads that a grid has (65536 samples of 1024 groups are 2^32).
constexpr int kGnMostJoins = 1 << 16;  // workgroups
constexpr int kGnCloseWaves = 16, kGnCloseCols = 32;  // backward: waves of one, and columns of a gradients' sum in one
inline unsigned gn_join_blocks(int N, int G, int waves) {
  const long long blocks = cdiv((long long)N * G, waves);
  return (unsigned)(blocks < kGnMostJoins ? blocks : kGnMostJoins);
}
inline int gn_close_columns(int C) { return (int)cdiv(2ll * C, kGnCloseCols); }  // workgroups of the gradients' sums, before those
GnPlan plan_gn(bool backward, int N, int P, int C, int G, int esize);

// Floats of workspace: the forward's, not held: (mean, sum of squares) of each sample, group and
// chunk.  The backward's: dw and db of each sample and chunk (2 C each), then, not held, the two sums
// over each group of each chunk, a group's chunks side by side, and of the sample.
inline long long gn_parts(const GnPlan& pl, int N) { return (long long)N * (pl.held ? 1 : pl.chunks); }
inline long long gn_fwd_floats(const GnPlan& pl, int N, int G) { return pl.held ? 0 : gn_parts(pl, N) * G * 2; }
inline long long gn_bwd_floats(const GnPlan& pl, int N, int C, int G) {
  return gn_parts(pl, N) * (2ll * C + (pl.held ? 0 : 2ll * G)) + (pl.held ? 0 : 2ll * N * G);
}

hipError_t launch_gn_fwd_f32(const GnPlan& pl, const GnParams& p, hipStream_t stream);
hipError_t launch_gn_fwd_bf16(const GnPlan& pl, const GnParams& p, hipStream_t stream);
hipError_t launch_gn_bwd_f32(const GnPlan& pl, const GnParams& p, hipStream_t stream);
hipError_t launch_gn_bwd_bf16(const GnPlan& pl, const GnParams& p, hipStream_t stream);

}  // namespace rows
}  // namespace o1d
