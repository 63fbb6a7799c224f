// The plan of group norm.
#include "o1d_gn.h"

namespace o1d {
namespace rows {

GnPlan plan_gn(bool backward, int N, int P, int C, int G, int esize) {
  const int D = C / G, V = 16 / esize, big = gn_big(backward, esize);
  GnPlan best{};
  best.held = false;
  // Held: the largest bundles that a workgroup holds and that still give every CU one
  double cost = -1.;
  for (int bundles = 1; bundles <= G; ++bundles) {
    const int gb = (int)cdiv(G, bundles), CB = gb * D;
    if (bundles > 1 && (int)cdiv(G, bundles - 1) == gb) continue;  // (the same with fewer)
    if (CB > kGnMostChannels) continue;
    if ((C >= V && CB < V) || (C < V && bundles > 1)) break;
    const int real = (int)cdiv(G, gb);
    for (int threads : {64, 256, big}) {
      const int run = (int)cdiv(CB, V);
      if (run > threads) continue;
      const long long rows = threads / run, need = cdiv(P, rows);
      const int runs = need <= 2 ? 2 : (int)cdiv(need, 2) * 2;
      if (!gn_takes(backward, esize, threads, runs)) continue;
      // A measure of time that orders the held plans, and them against two passes; as a time it is short, by half for one large
      // workgroup per CU (64 x 3136 x 96 bfloat16 13.5 of 25 us, two passes 18.3): what a CU moves, at the rate that it has among the
      // others, and the two reductions, which small workgroups on a CU have at the same time (65536 samples of 1 x 64 bfloat16 in workgroups of 64 threads 125 us, in two passes 580);
      // rows of fewer channels than a run are loaded one by one (6 x 183 x 7 bfloat16 in two runs 7 us, in four 10)
      const double bytes = (double)P * CB * esize, piece = CB * esize;
      const long long groups = (long long)N * real, rounds = cdiv(groups, 256);
      const double per_cu = groups >= 256 ? 20e3 : (groups > 102 ? 5.12e6 / groups : 50e3);  // bytes per us
      const double sums = threads == 64 ? 1.2 * cdiv(groups, backward ? 2048 : 4096)
                                        : (threads == 256 ? 1.5 * cdiv(groups, backward ? 512 : 1024) : 3. * rounds);
      const double t = rounds * (bytes / per_cu * (piece < 64 ? 64 / piece : 1.)) + sums + (C < V ? 0.8 : 0.05) * runs;
      if (cost >= 0. && t >= cost) continue;
      cost = t;
      best = {true, threads, runs, gb, real, 1, P};
    }
  }
  const double twice = 6. + (double)N * P * C * esize * 1.6 / 5.0e6 + 3. * (N / 1024);
  if (best.held && cost <= twice) return best;
  // In chunks: bundles as wide as a workgroup takes, pieces enough to fill the GPU
  GnPlan pl{};
  pl.gb = kGnMostChannels / D < G ? kGnMostChannels / D : G;
  pl.bundles = (int)cdiv(G, pl.gb);
  pl.gb = (int)cdiv(G, pl.bundles);
  pl.bundles = (int)cdiv(G, pl.gb);
  const int rows = 256 / (int)cdiv((long long)pl.gb * D, V);  // at a time
  // (three of a CU, all there at once: 3 x 12707 x 203 bfloat16 in 384, 768 and 1536 pieces forward 31, 28 and 33 us, backward
  // 44, 38 and 46; at least two rows of a thread: 2 x 4880 x 6 backward with four 18 us, with two 16)
  long long chunks = cdiv(768, (long long)N * pl.bundles);
  const long long least = cdiv(P, 2ll * (rows > 0 ? rows : 1));
  if (chunks > least) chunks = least;
  if (chunks > kGnMostChunks) chunks = kGnMostChunks;
  if (chunks < 1) chunks = 1;
  pl.rows = (int)cdiv(P, chunks);
  pl.chunks = (int)cdiv(P, pl.rows);
  return pl;
}

}  // namespace rows
}  // namespace o1d
