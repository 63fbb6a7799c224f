"""Group norm's plan on the host: what its kernels make of the sizes that its entry points take.

Small C++ programs take plan_gn's plans and go over a chunk's rows as the kernels' threads do.
"""
import os
import subprocess

import pytest

from paper_2309_15812_amd import build

HEAD = r"""
#include <stdio.h>
#include "o1d_gn_plan.hip"
using namespace o1d::rows;
const long long kMostRows = 0x7fffffff - 1024;  // samples x pixels of a call
"""

ROWS = HEAD + r"""
// Every row of a sample's first and last chunks is taken once, and no thread reads another one, also of the longest samples.
int main() {
  const int sizes[][2] = {{1, 1}, {4, 1}, {8, 8}, {7, 7}, {96, 32}, {203, 7}, {1100, 11}};
  long long taken = 0;
  for (int backward : {0, 1})
    for (int es : {2, 4})
      for (auto& c : sizes)
        for (int N : {1, 2, 3, 7, 767, 768})
          for (long long all : {kMostRows, kMostRows - 1021, kMostRows / 3, 1000000ll, 12707ll}) {
            const int P = (int)(all / N);
            if (P < 1) continue;
            const GnPlan pl = plan_gn(backward, N, P, c[0], c[1], es);
            if (pl.held) continue;
            const int CB = pl.gb * (c[0] / c[1]), V = 16 / es, slots = kGnThreads / (int)cdiv(CB, V);
            if (pl.chunks > kGnMostChunks || (long long)pl.chunks * pl.rows < P || (pl.chunks - 1ll) * pl.rows >= P) {
              printf("N=%d P=%d C=%d: %d chunks of %d\n", N, P, c[0], pl.chunks, pl.rows);
              return 1;
            }
            for (int batch : {kGnBatch, kGnBatch / 2})
              for (int chunk : {0, pl.chunks - 1}) {
                const GnRow r0 = (GnRow)chunk * (GnRow)pl.rows, past = r0 + (GnRow)pl.rows, r1 = past < (GnRow)P ? past : (GnRow)P;
                long long seen = 0;
                for (int slot : {0, slots / 2, slots - 1}) {
                  long long mine = 0;
                  const long long most = cdiv((long long)r1 - r0, (long long)batch * slots) + 1;
                  long long round = 0;
                  for (GnRow r = r0 + slot; r < r1; r += batch * slots) {
                    if (++round > most) {
                      printf("N=%d P=%d C=%d chunk %d: a thread goes on behind row %lld\n", N, P, c[0], chunk, (long long)r1);
                      return 1;
                    }
                    for (int k = 0; k < batch; ++k) {
                      const long long at = (long long)gn_row(r, k, slots, r1), want = (long long)r + (long long)k * slots;
                      if (at < (long long)r0 || at >= (long long)r1 || (want < (long long)r1 ? at != want : at != (long long)r1 - 1)) {
                        printf("N=%d P=%d C=%d chunk %d: row %lld of %lld .. %lld\n", N, P, c[0], chunk, at, (long long)r0, (long long)r1);
                        return 1;
                      }
                      mine += want < (long long)r1;
                    }
                  }
                  const long long rest = (long long)r1 - r0 - slot;
                  if (mine != (rest > 0 ? cdiv(rest, slots) : 0)) {
                    printf("N=%d P=%d C=%d chunk %d: %lld rows of slot %d\n", N, P, c[0], chunk, mine, slot);
                    return 1;
                  }
                  seen += mine;
                }
                taken += seen;
              }
          }
  printf("%lld rows\n", taken);
  return taken > 0 ? 0 : 1;
}
"""

GRIDS = HEAD + r"""
// All samples' groups are joined whatever their number, by grids of fewer than 2^32 threads.
int main() {
  long long most = 0;
  const int sizes[][3] = {{65536, 2048, 1024}, {65536, 7168, 1024}, {1, 1, 1}, {300, 64, 2}, {1 << 17, 512, 512}, {1 << 16, 1024, 1024},
                          {(1 << 16) + 1, 1024, 1024}, {0x7fffffff - 1024, 1 << 20, 1 << 20}, {1 << 20, 1 << 10, 1 << 10}, {3, 203, 7}};
  for (auto& s : sizes) {
    const long long N = s[0], C = s[1], G = s[2], groups = N * G;
    const long long join = gn_join_blocks((int)N, (int)G, kGnThreads / 64), close = gn_join_blocks((int)N, (int)G, kGnCloseWaves);
    const long long columns = gn_close_columns((int)C);
    if (join < 1 || close < 1 || join * kGnThreads >= 1ll << 32 || (columns + close) * 64 * kGnCloseWaves >= 1ll << 32 ||
        columns * kGnCloseCols < 2 * C) {
      printf("%lld samples of %lld groups: %lld and %lld + %lld workgroups\n", N, G, join, columns, close);
      return 1;
    }
    // (a grid that is not cut has a wave for each group)
    if ((join < kGnMostJoins && join * (kGnThreads / 64) < groups) || (close < kGnMostJoins && close * kGnCloseWaves < groups)) {
      printf("%lld samples of %lld groups: %lld and %lld workgroups leave groups out\n", N, G, join, close);
      return 1;
    }
    most = join > most ? join : most;
  }
  return most == kGnMostJoins ? 0 : 1;
}
"""


@pytest.fixture(scope="module")
def compile_run(tmp_path_factory):
    def go(source):
        d = tmp_path_factory.mktemp("gn")
        src, exe = d / "t.cpp", d / "t"
        src.write_text(source)
        rocm = os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC)))
        subprocess.run(["g++", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", build.CSRC,
                        "-I", os.path.join(rocm, "include"), str(src), "-o", str(exe)], check=True)
        return subprocess.run([str(exe)], capture_output=True, text=True)
    return go


def test_rows_of_a_chunk_stay_in_it(compile_run):
    r = compile_run(ROWS)
    assert r.returncode == 0, r.stdout


def test_grids_between_the_passes(compile_run):
    r = compile_run(GRIDS)
    assert r.returncode == 0, r.stdout
