// Matrix products of rows whose runs are whole and aligned (included by
// o1d_mmf_*.hip): the products of o1d_mm_kernels.h with memory moved straight
// into LDS, several steps ahead.
//
// A step is 128 bytes of k (a cache line).  Its 16-byte runs go from memory to LDS without
// passing registers (one instruction moves 64 runs to 1 KB of LDS in lane
// order); which run a lane fetches is chosen so that the fragments' reads do
// not conflict.  kStages buffers are filled ahead of the products, one barrier
// per step.  A workgroup takes tile after tile: the next tile's first steps are
// on their way while the epilogue of the last one, which needs registers only,
// runs, which hides most of the first loads (1.7 us per tile).
//
// Bound by the CU's loads from L2: a step of 128 x 128 brings 32 KB, about 26 bytes a
// clock and CU, while its products take two fifths of that time; 8192 x 2048 -> 2048
// 66 to 77 us (0.9 to 1.04 PFLOP/s).  With few steps per tile the epilogue's vector
// instructions come next to that: 12544 x 384 -> 1536 with GELU and checkpoint 37 to 40 us.
//
// Runs past K are fetched from a zeroed run, rows past the end from the last row.
#pragma once

#include "o1d_mm_kernels.h"

namespace o1d {
namespace rows {
namespace {

constexpr int kFastStep = kStepBytes;  // bytes of k: whole cache lines

__device__ const u32x4 g_zero_run = {0u, 0u, 0u, 0u};

// 64 lanes' 16-byte runs to 1 KB of LDS at `lds` (the same in all lanes), in
// lane order.  The instruction is invisible to the compiler's wait counts: the
// caller waits (wait_loads) before a barrier that precedes the reads.
// (m0 is no register that values are given to, which the compiler warns of where it is named.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void fetch(const char* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void fetch(const char* base, uint32_t off, uint32_t stage, uint32_t block) {
  asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(stage), "s"(block)
               : "memory", "scc", "m0");
}
#pragma clang diagnostic pop

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// (the reads of the last step's fragments are done in every wave)
__device__ __forceinline__ void step_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One operand's tile in LDS: R rows x 128 bytes of k.  KC: contiguous along k in
// memory (and LDS rows of 128 bytes), else along the rows (LDS rows of R elements).
template <typename T, int R, bool KC>
struct FastTile {
  static constexpr int V = 16 / (int)sizeof(T), BK = kFastStep / (int)sizeof(T);
  static constexpr int kBlocks = R / 8;            // KB of LDS
  static constexpr int kBytes = R * kFastStep;
  static constexpr int kRuns = KC ? 8 : R / V;     // runs of an LDS row

  // the run of LDS row `row` that lies at place `slot`
  static __device__ __forceinline__ int run_at(int row, int slot) {
    // LDS has 64 banks: sixteen 16-byte reads (KC: of consecutive rows) or 32
    // 8-byte ones (the transposing reads: two 32-byte pieces of four k) at a time
    if constexpr (KC) return slot ^ ((row >> 1) & 7);
    if constexpr (R % 64 != 0) return slot;  // (rows of 96: 192 bytes apart)
    if constexpr (R == 64) return slot ^ (2 * (row & 2));
    return slot ^ (4 * (row & 3));
  }

  // Where lane l of block b fetches from for step 0: offset in bytes from row
  // r0 (KC) or column r0 of the operand; and that run's k in elements.
  static __device__ __forceinline__ uint32_t source(int b, int l, long long ld, int r0, int rows) {
    const int at = 64 * b + l, row = at / kRuns, run = run_at(row, at % kRuns);
    if constexpr (KC)
      return ((uint32_t)min(row, rows - 1 - r0) * (uint32_t)ld + run * V) * (uint32_t)sizeof(T);
    else
      return ((uint32_t)row * (uint32_t)ld + min(run * V, rows - V - r0)) * (uint32_t)sizeof(T);
  }
  static __device__ __forceinline__ int k_at(int b, int l) {
    const int at = 64 * b + l, row = at / kRuns;
    return KC ? run_at(row, at % kRuns) * V : row;
  }
  static __device__ __forceinline__ const char* origin(const void* p, long long ld, int r0, int s0) {
    const long long at = KC ? (long long)r0 * ld + (long long)s0 * BK : (long long)s0 * BK * ld + r0;
    return static_cast<const char*>(p) + at * (long long)sizeof(T);
  }

  // Fragment j (0 .. 3: a quarter of the step) of the 32 rows from `row` on; k as in Tile::frag.
  static __device__ __forceinline__ Frag<T> frag(const char* lds, int row, int j) {
    Frag<T> f;
    const int l = threadIdx.x & 63;
    if constexpr (KC) {
      const int r = row + (l & 31);
      f.p[0] = *reinterpret_cast<const u32x4*>(lds + r * kFastStep + run_at(r, 2 * j + (l >> 5)) * 16);
    } else {
      const int g = l >> 4, i = l & 15;
      const int k = 8 * (2 * j + (g >> 1)) + (i >> 2), r = row + 16 * (g & 1) + 4 * (i & 3);
      // (k and k + 4 have their runs in the same order)
      const char* at = lds + k * R * 2 + run_at(k, r / 8) * 16 + r % 8 * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * R * 2));
      __builtin_memcpy(&f.p[0], &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&f.p[0]) + 8, &hi, 8);
    }
    return f;
  }
};

template <typename T, int KIND, int SHAPE>
struct FastGeo {
  static constexpr Shape S = kShapes[SHAPE];
  static constexpr int BM = 32 * S.tm * S.wm, BN = 32 * S.tn * S.wn;
  using TA = FastTile<T, BM, KIND != kWgrad>;
  using TB = FastTile<T, BN, KIND == kFwd>;
  static constexpr int kBlocks = TA::kBlocks + TB::kBlocks;
  static constexpr int kFetches = (kBlocks + 3) / 4;  // of a wave, per step
  static constexpr int kStage = TA::kBytes + TB::kBytes;
  static constexpr int kStages = kStage * 3 <= 64 * 1024 ? 3 : 2;
  static constexpr int kLds = kStage * kStages;
  static constexpr int kWaves = S.tm * S.tn <= 2 ? 3 : 2;  // per SIMD
};

template <typename T, int KIND, int SHAPE>
__global__ __launch_bounds__(kMmThreads, (FastGeo<T, KIND, SHAPE>::kWaves)) void mmf(MmParams P) {
  using G = FastGeo<T, KIND, SHAPE>;
  constexpr int TM = G::S.tm, TN = G::S.tn, BK = kFastStep / (int)sizeof(T), S = G::kStages, NF = G::kFetches;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / G::S.wn * 32 * TM, wn = wave % G::S.wn * 32 * TN;
  // consecutive tiles, which share rows of A (weight gradient: the piece of
  // k), on one XCD; this workgroup's: id, id + stride, ..
  const int per_xcd = (P.nblocks + 7) / 8, stride = (int)gridDim.x / 8;
  const int last = min(P.nblocks, ((int)blockIdx.x % 8 + 1) * per_xcd);
  int id = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (id >= last) return;

  struct At {
    int m0, n0, split, s0, s1;
  };
  auto tile_of = [&](int t) __attribute__((always_inline)) {
    const int nt = t % P.tn, rest = t / P.tn;
    auto scalar = [](int v) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(v); };
    At a;
    a.m0 = scalar(rest % P.tm * G::BM);
    a.n0 = scalar(nt * G::BN);
    a.split = scalar(rest / P.tm);
    a.s0 = a.split * P.per;
    a.s1 = min(P.steps, a.s0 + P.per);
    return a;
  };

  // ---- the loads, kStages - 1 steps ahead of the products: a lane's offsets
  // stay for a tile, the operands' (scalar) addresses go from step to step
  static_assert(G::TA::kBlocks % 4 == 0, "a wave's first fetches are A's");
  uint32_t off[NF], block[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) block[f] = (uint32_t)min(wave + 4 * f, G::kBlocks - 1) * 1024;
  const char *base_a, *base_b;
  int ahead_id = id, ahead_left = 0;  // the tile that is loaded and its steps to come
  int ahead_k = 0;                    // k from the next step on
  uint32_t ahead_stage = 0;
  const long long step_a = KIND != kWgrad ? kFastStep : (long long)BK * P.lda * (long long)sizeof(T);
  const long long step_b = KIND == kFwd ? kFastStep : (long long)BK * P.ldb * (long long)sizeof(T);
  auto is_a = [](int f) __attribute__((always_inline)) { return 4 * f < G::TA::kBlocks; };
  auto aim = [&]() __attribute__((always_inline)) {  // at the first step of tile ahead_id
    const At a = tile_of(ahead_id);
    ahead_left = a.s1 - a.s0;
    ahead_k = P.K - a.s0 * BK;
    base_a = G::TA::origin(P.a, P.lda, a.m0, a.s0);
    base_b = G::TB::origin(P.b, P.ldb, a.n0, a.s0);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int b = (int)(block[f] / 1024);
      if (is_a(f))
        off[f] = G::TA::source(b, lane, P.lda, a.m0, P.M);
      else
        off[f] = G::TB::source(b - G::TA::kBlocks, lane, P.ldb, a.n0, P.N);
    }
  };
  // The next step's loads, a whole one inside the tile.
  auto issue_whole = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int f = 0; f < NF; ++f) fetch(is_a(f) ? base_a : base_b, off[f], ahead_stage, block[f]);
    ahead_stage = ahead_stage == (S - 1) * G::kStage ? 0 : ahead_stage + G::kStage;
    --ahead_left;
    ahead_k -= BK;
    base_a += step_a;
    base_b += step_b;
  };
  // The next step's loads, whatever it is (nothing to load: zeros that are never read).
  auto issue = [&]() __attribute__((always_inline)) {
    if (ahead_left == 0 && ahead_id + stride < last) {
      ahead_id += stride;
      aim();
    }
    if (ahead_left > 0 && ahead_k >= BK) {
      issue_whole();
    } else {
      const bool any = ahead_left > 0;
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const int b = (int)(block[f] / 1024);
        const int k = is_a(f) ? G::TA::k_at(b, lane) : G::TB::k_at(b - G::TA::kBlocks, lane);
        const char* p = (is_a(f) ? base_a : base_b) + off[f];
        fetch(any && k < ahead_k ? p : reinterpret_cast<const char*>(&g_zero_run), ahead_stage + block[f]);
      }
      ahead_stage = ahead_stage == (S - 1) * G::kStage ? 0 : ahead_stage + G::kStage;
      if (any) --ahead_left;
    }
  };

  aim();
#pragma unroll
  for (int s = 0; s < S - 1; ++s) issue();

  uint32_t stage = 0;
  int landed = 0;
  for (; id < last; id += stride) {
    const At at = tile_of(id);
    f32x16 acc[TM][TN];
    float dbs[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      dbs[i] = 0.f;
#pragma unroll
      for (int k = 0; k < TN; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][k][e] = 0.f;
    }
    const bool sum_a = KIND == kWgrad && P.want_db && at.n0 == 0 && wn == 0;
    auto step = [&](auto&& loads) __attribute__((always_inline)) {
      if (landed > 0)
        --landed;
      else
        wait_loads<(S - 2) * NF>();
      step_barrier();
      const char *la = lds + stage, *lb = la + G::TA::kBytes;
      stage = stage == (S - 1) * G::kStage ? 0 : stage + G::kStage;
      Frag<T> fm[4][TM], fn[4][TN];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < TM; ++i) fm[j][i] = G::TA::frag(la, wm + 32 * i, j);
#pragma unroll
        for (int i = 0; i < TN; ++i) fn[j][i] = G::TB::frag(lb, wn + 32 * i, j);
      }
      loads();
      __builtin_amdgcn_sched_barrier(0);  // the reads before the products
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (sum_a) {
#pragma unroll
          for (int i = 0; i < TM; ++i) dbs[i] = add_frag<T>(fm[j][i], dbs[i]);
        }
        products<T>(fn[j], fm[j], acc);
      }
    };
    // steps whose load ahead is a whole one of this tile, then the others
    const int steps = at.s1 - at.s0;
    const int whole = ahead_id == id ? min(ahead_left, ahead_k / BK) : 0;
    int s = 0;
    for (; s < whole; ++s) step(issue_whole);
    for (; s < steps; ++s) step(issue);
    // the stages on their way are waited for before the first store, not
    // behind the stores
    auto first = [&]() __attribute__((always_inline)) {
      wait_loads<0>();
      landed = S - 1;
    };
    if constexpr (KIND == kWgrad) {
      first();
      if (sum_a) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const float s = dbs[i] + __shfl_xor(dbs[i], 32, 64);
          const int m = at.m0 + wm + 32 * i + (lane & 31);
          if (lane < 32 && m < P.M) put_db<T>(P, at.split, m, s);
        }
      }
    }
    if (at.m0 + G::BM <= P.M && at.n0 + G::BN <= P.N)
      epilogue<T, KIND, true>(P, at.m0 + wm, at.n0 + wn, at.split, acc, first);
    else
      epilogue<T, KIND, false>(P, at.m0 + wm, at.n0 + wn, at.split, acc, first);
  }
  wait_loads<0>();  // nothing is on its way to LDS when the workgroup ends
}

template <typename T, int KIND, int SHAPE>
hipError_t launch_fast_shape(const MmPlan& pl, hipStream_t stream) {
  using G = FastGeo<T, KIND, SHAPE>;
  static std::atomic<int> allowed{0};
  static std::atomic<int> resident{0};
  if (!allowed.load(std::memory_order_acquire)) {
    const void* f = reinterpret_cast<const void*>(mmf<T, KIND, SHAPE>);
    hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds);
    if (e != hipSuccess) return e;
    int per_cu = 0;
    e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, f, kMmThreads, G::kLds);
    if (e != hipSuccess) return e;
    resident.store(per_cu > 0 ? per_cu : 1);
    allowed.store(1, std::memory_order_release);
  }
  const int most = 256 * resident.load(), blocks = (pl.p.nblocks + 7) / 8 * 8;
  hipLaunchKernelGGL((mmf<T, KIND, SHAPE>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(kMmThreads), G::kLds,
                     stream, pl.p);
  return hipGetLastError();
}

template <typename T, int KIND, int SHAPE>
hipError_t launch_fast_planned(const MmPlan& pl, hipStream_t stream) {
  if constexpr (shape_used(KIND, (int)sizeof(T), SHAPE)) return launch_fast_shape<T, KIND, SHAPE>(pl, stream);
  return hipErrorInvalidValue;  // (no plan has it)
}

template <typename T, int KIND>
hipError_t launch_fast_kind(const MmPlan& pl, hipStream_t stream) {
  switch (pl.shape) {
    case k128x128: return launch_fast_planned<T, KIND, k128x128>(pl, stream);
    case k64x64: return launch_fast_planned<T, KIND, k64x64>(pl, stream);
    case k128x96: return launch_fast_planned<T, KIND, k128x96>(pl, stream);
    case k64x128: return launch_fast_planned<T, KIND, k64x128>(pl, stream);
    case k128x64: return launch_fast_planned<T, KIND, k128x64>(pl, stream);
    case k128x32: return launch_fast_planned<T, KIND, k128x32>(pl, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace
}  // namespace rows
}  // namespace o1d
