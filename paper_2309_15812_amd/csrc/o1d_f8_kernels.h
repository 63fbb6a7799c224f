// Matrix products of 8-bit floating point operands with a power-of-two scale for
// each 128 values of a row (included by o1d_f8_*.hip).
//
//   C[m][n] = sum over groups g of 128 k:  2^(ea[g][m] + eb[g][n] - 254) sum_{k in g} qa[m][k] qb[n][k]
//
// Results of bfloat16: the matrix instruction takes both operands' exponents with the fragments and adds the
// scaled products to the float32 sum: nothing is multiplied per group in vector registers.
// It adds eight products at a time (a lane's eight bytes) in fixed point, to 2^-13 of the power of two below the
// largest of them, and those sums in float32: measured, results are 1.5e-5 from 64 bits, a hundredth of their own rounding.  (A product that is less
// than 2^-13 of another one among its eight is lost, also where that one cancels.  Summed in float32, as below, 8192 x 8192 -> 8192 takes
// 930 us against 490 in the same run, 4096 x 4096 -> 4096 145 against 69.)
//
// Results of float32: fragments are widened to bfloat16, with their scales, which loses nothing (eight significant bits hold
// either type's values; below 2^-126 bfloat16 has fewer), and multiplied by the bfloat16 instruction, whose sums keep
// float32's bits: 4e-8 from 64 bits, at half the rate at best.
//
// 8192 x 8192 -> 8192 takes 452 to 474 us (422 at least), 2.4 PFLOP/s, in tiles of 256 x 256 by eight waves, two operands' steps of 128 k in LDS (64 KB
// each): bound by the matrix instructions.  The other tiles there: 128 x 128 605 us (each operand is read from the L2 twice as
// often), 256 x 256 by four waves 544 (a wave's sums are 256 registers, and fragments have too few left to be read ahead).
// 12544 x 384 -> 1536 with gelu and its argument kept takes 30 us, 82 MB: three steps of products, so its epilogue's
// 77 MB of stores are not covered by them.
#pragma once

#include "o1d_f8.h"
#include "o1d_mmf_kernels.h"
#include "o1d_wave.h"

namespace o1d {
namespace rows {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// As fetch, of the lanes in `mask` (all or none: no branch parts the products); and 64 lanes' words to
// 256 bytes of LDS at `lds`.  All lanes are active before and after.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void fetch_if(uint64_t mask, const char* base, uint32_t off, uint32_t stage, uint32_t block) {
  asm volatile("s_add_u32 m0, %2, %3\n\ts_mov_b64 exec, %4\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(off),
               "s"(base), "s"(stage), "s"(block), "s"(mask)
               : "memory", "scc", "m0");
}
__device__ __forceinline__ void fetch_words_if(uint64_t mask, const char* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 exec, %2\n\tglobal_load_lds_dword %0, off\n\ts_mov_b64 exec, -1" ::"v"(from),
               "s"(lds), "s"(mask)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// acc[k] += m fragment times n fragment k, 64 of k: fragments of two runs, the same two
// for both operands, and their rows' exponents.  between(): called after each product.
template <int ATYPE, int TN, class F>
__device__ __forceinline__ void f8_products(const u32x4 (&n)[TN][2], const u32x4 (&m)[2], const uint32_t (&sn)[TN],
                                            uint32_t sm, f32x16 (&acc)[TN], F&& between) {
  auto whole = [](const u32x4(&f)[2]) __attribute__((always_inline)) {
    i32x8 r;
    __builtin_memcpy(&r, f, 32);
    return r;
  };
  wave::static_for<TN>([&](auto kc) __attribute__((always_inline)) {
    constexpr int k = decltype(kc)::value;
    acc[k] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(n[k]), whole(m), acc[k], kE4M3, ATYPE, 0, (int)sn[k], 0,
                                                             (int)sm);
    between(kc);
  });
}

// Eight values of a run, two words, widened.
template <int TYPE>
__device__ __forceinline__ bf16x8 widened(uint32_t lo, uint32_t hi, uint32_t exponent) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float scale = __uint_as_float(exponent << 23);  // (its exponent is what is read)
  bf16x2 p[4];
  if constexpr (TYPE == kE4M3) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
  }
  bf16x8 r;
  __builtin_memcpy(&r, p, 16);
  return r;
}
template <int ATYPE, int TN, class F>
__device__ __forceinline__ void wide_products(const u32x4 (&n)[TN][2], const u32x4 (&m)[2], const uint32_t (&sn)[TN],
                                              uint32_t sm, f32x16 (&acc)[TN], F&& between) {
  wave::static_for<TN>(between);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x8 wm = widened<ATYPE>(m[j / 2][j % 2 * 2], m[j / 2][j % 2 * 2 + 1], sm);
#pragma unroll
    for (int k = 0; k < TN; ++k)
      acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened<kE4M3>(n[k][j / 2][j % 2 * 2], n[k][j / 2][j % 2 * 2 + 1], sn[k]),
                                                       wm, acc[k], 0, 0, 0);
  }
}

// The wave's tile, a block of 32 rows x 64 columns (32 of a tile that narrow) after the other, by way of LDS (`mine`,
// 8 or 4 KB): from the products' layout, 32 rows in a store of 32 bytes each, to whole cache lines of
// eight rows; what the block's epilogue reads comes the same way.  (Straight from the products' layout, rows 16 KB
// apart, the epilogue of a tile of 256 x 256 took 21 us.)  ACT: the activation (kActs: P.act, whatever it is);
// one choice for the tile, not one for every run.
template <typename T, int KIND, bool WHOLE, int ACT, int TM, int TN>
__device__ __forceinline__ void f8_blocks(const MmParams& Q, int m0, int n0, int split, const f32x16 (&acc)[TM][TN],
                                          char* mine) {
  constexpr int NB = TN % 2 ? 1 : 2, kCols = 32 * NB, kRuns = kCols / 4, kSame = kCols / 8, kRows = 64 / kSame;
  constexpr int kSets = 32 / kRows, kBlocks = TM * TN / NB;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // (what follows from it is not computed before the products, for registers)
  const int half = lane >> 5, row = lane & 31;
  MmParams P = Q;
  if constexpr (ACT != kActs) P.act = ACT;
  const int r = lane / kSame, c = lane % kSame;  // this lane's row (of every kRows) and run of eight columns
  // runs of four columns lie in an order of their row's own, so that neither side has bank conflicts
  float* const to = reinterpret_cast<float*>(mine) + row * kCols;
  const float* const from = reinterpret_cast<const float*>(mine) + r * kCols;
  static_assert(kRows % 8 == 0 && kRuns % 8 == 0, "the order repeats");
  wave::static_for<kBlocks>([&](auto bc) __attribute__((always_inline)) {
    constexpr int b = decltype(bc)::value, i = b % TM, k = b / TM;
    const int m = m0 + 32 * i + r, n = n0 + kCols * k + 8 * c;
    Ahead<T, KIND, WHOLE> ahead[kSets];
    if constexpr (KIND != kWgrad) {
#pragma unroll
      for (int q = 0; q < kSets; ++q) ahead[q].load(P, m + kRows * q, n);
    }
    T bias[8];
    const bool biased = KIND == kFwd && P.bias;
    if (biased) {
      const T* p = static_cast<const T*>(P.bias) + n;
      if (WHOLE || n + 8 <= P.N) {
        __builtin_memcpy(bias, p, sizeof(bias));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = n + e < P.N ? p[e] : T(0);
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[i][NB * k + j][4 * g], acc[i][NB * k + j][4 * g + 1], acc[i][NB * k + j][4 * g + 2],
                            acc[i][NB * k + j][4 * g + 3]};
        __builtin_memcpy(__builtin_assume_aligned(to + 4 * ((8 * j + 2 * g + half) ^ (row & (kRuns - 1))), 16), v, 16);
      }
    asm volatile("" ::: "memory");  // (a wave's accesses of LDS keep their order)
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < kSets; ++q) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        __builtin_memcpy(v + 4 * j,
                         __builtin_assume_aligned(from + kRows * q * kCols + 4 * ((2 * c + j) ^ ((r + kRows * q) & (kRuns - 1))), 16),
                         16);
      if (biased) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += to_f32(bias[e]);
      }
      const int mq = m + kRows * q;
      if constexpr (KIND == kWgrad) {
        if (WHOLE || (mq < P.M && n < P.N)) {
          if (P.nsplit == 1)
            put<T, WHOLE>(static_cast<T*>(P.out) + (long long)mq * P.N + n, P.N - n, v);
          else
            put<float, WHOLE>(P.part + (long long)split * ((long long)P.M * P.N + P.M) + (long long)mq * P.N + n, P.N - n, v);
        }
      } else {
        finish<T, KIND, WHOLE>(P, mq, n, ahead[q], v);
      }
      if constexpr (TM * TN > 4) __builtin_amdgcn_sched_barrier(0);  // (registers)
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_sched_barrier(0);
  });
}

template <typename T, int KIND, int TM, int TN>
__device__ __forceinline__ void f8_epilogue(const MmParams& P, bool whole, int m0, int n0, int split,
                                            const f32x16 (&acc)[TM][TN], char* mine) {
  if (!whole) return f8_blocks<T, KIND, false, kActs>(P, m0, n0, split, acc, mine);
  if constexpr (KIND == kWgrad) return f8_blocks<T, KIND, true, kNone>(P, m0, n0, split, acc, mine);
  switch (P.act) {
    case kRelu: return f8_blocks<T, KIND, true, kRelu>(P, m0, n0, split, acc, mine);
    case kGelu: return f8_blocks<T, KIND, true, kGelu>(P, m0, n0, split, acc, mine);
    case kGeluTanh: return f8_blocks<T, KIND, true, kGeluTanh>(P, m0, n0, split, acc, mine);
    case kSilu: return f8_blocks<T, KIND, true, kSilu>(P, m0, n0, split, acc, mine);
    default: return f8_blocks<T, KIND, true, kNone>(P, m0, n0, split, acc, mine);
  }
}

template <int SHAPE>
struct F8Geo {
  static constexpr Shape S = kF8Shapes[SHAPE];
  static constexpr int kCount = S.wm * S.wn, kThreads = 64 * kCount;  // waves and threads of a workgroup
  static constexpr int BM = 32 * S.tm * S.wm, BN = 32 * S.tn * S.wn;
  using TA = FastTile<uint8_t, BM, true>;
  using TB = FastTile<uint8_t, BN, true>;
  static constexpr int kBlocks = TA::kBlocks + TB::kBlocks, kFetches = kBlocks / kCount;  // KB, and a wave's, of a step
  static_assert(kBlocks % kCount == 0 && TA::kBlocks % kCount == 0, "a wave's first fetches are A's");
  static constexpr int kScales = kBlocks * 1024;  // where the exponents of a step lie, A's then B's
  static constexpr int kStage = kScales + 256 * kCount;
  static_assert(BM + BN <= 256 * kCount, "a word of exponents for each thread");
  static constexpr int kLds = kStage * 2;
  static constexpr int kMine = 32 * (S.tn % 2 ? 32 : 64) * 4;  // of a wave, for the epilogue, in a stage
  static_assert(kMine * kCount <= kStage, "a block of sums for each wave");
  static constexpr int kWaves = SHAPE == kF8_64x64 ? 4 : 2;  // per SIMD
};

// Two stages of LDS.  A step's products go by 32 rows of m and 64 of k at a time (a part), whose fragments
// are read kAhead parts before.  When a step's last fragments are on their way to registers and the next step has
// landed, its stage is free: the loads of the step after the next go there, and the next step's first fragments are
// read during the products that are left.  One barrier per step; the loads have a whole step to arrive.
template <typename T, int KIND, int SHAPE, int ATYPE>
__global__ __launch_bounds__(F8Geo<SHAPE>::kThreads, F8Geo<SHAPE>::kWaves) void f8mm(F8MmParams Q) {
  using G = F8Geo<SHAPE>;
  const MmParams& P = Q.mm;
  constexpr int TM = G::S.tm, TN = G::S.tn, BK = kF8Group, NF = G::kFetches;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / G::S.wn * 32 * TM, wn = wave % G::S.wn * 32 * TN;
  const int per_xcd = (P.nblocks + 7) / 8, stride = (int)gridDim.x / 8;
  const int last = min(P.nblocks, ((int)blockIdx.x % 8 + 1) * per_xcd);
  int id = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (id >= last) return;

  struct At {
    int m0, n0, split, s0, s1;
  };
  // Tiles in bands of `band` rows of tiles, column after column: those at work at a time share both operands.
  auto tile_of = [&](int t) __attribute__((always_inline)) {
    auto scalar = [](int v) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(v); };
    const int per = P.tm * P.tn, split = t / per, in = t - split * per;
    const int band = in / (Q.band * P.tn), first = band * Q.band, rows = min(Q.band, P.tm - first);
    const int rest = in - first * P.tn;
    At a;
    a.m0 = scalar((first + rest % rows) * G::BM);
    a.n0 = scalar(rest / rows * G::BN);
    a.split = scalar(split);
    a.s0 = a.split * P.per;
    a.s1 = min(P.steps, a.s0 + P.per);
    return a;
  };

  // ---- the loads, two steps ahead of the products: a lane's offsets stay for a tile, the operands'
  // (scalar) addresses go from step to step
  uint32_t off[NF], block[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) block[f] = (uint32_t)(wave + G::kCount * f) * 1024;
  const char *base_a = nullptr, *base_b = nullptr, *exps = nullptr;
  long long exps_by = 0;
  int ahead_id = id, ahead_left = 0;
  uint32_t ahead_stage = 0;
  auto is_a = [](int f) __attribute__((always_inline)) { return G::kCount * f < G::TA::kBlocks; };
  auto aim = [&]() __attribute__((always_inline)) {
    const At a = tile_of(ahead_id);
    ahead_left = a.s1 - a.s0;
    base_a = G::TA::origin(P.a, P.lda, a.m0, a.s0);
    base_b = G::TB::origin(P.b, P.ldb, a.n0, a.s0);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int b = (int)(block[f] / 1024);
      off[f] = is_a(f) ? G::TA::source(b, lane, P.lda, a.m0, P.M) : G::TB::source(b - G::TA::kBlocks, lane, P.ldb, a.n0, P.N);
    }
    // a thread's four exponents of the tile's rows, A's then B's
    const int at = 4 * (int)threadIdx.x;
    const bool of_a = at < G::BM;
    const int row = of_a ? a.m0 + at : a.n0 + at - G::BM;
    const long long le = of_a ? Q.lea : Q.leb;
    const bool in = at < G::BM + G::BN && row < le;  // (others: rows past the end, whose results are not stored)
    exps = in ? reinterpret_cast<const char*>((of_a ? Q.ea : Q.eb) + a.s0 * le + row)
              : reinterpret_cast<const char*>(&g_zero_run);
    exps_by = in ? le : 0;
  };
  // Whether there is a step to fetch, as a mask of the lanes; the tile's steps done, it is the next tile's first.
  auto ahead = [&]() __attribute__((always_inline)) {
    if (ahead_left == 0) {
      if (ahead_id + stride >= last) return (uint64_t)0;
      ahead_id += stride;
      aim();
    }
    return ~(uint64_t)0;
  };
  // that step's fetch f (NF: the exponents'), and what follows the last of them
  auto issue_one = [&](uint64_t mask, auto fc) __attribute__((always_inline)) {
    constexpr int f = decltype(fc)::value;
    if constexpr (f < NF)
      fetch_if(mask, is_a(f) ? base_a : base_b, off[f], ahead_stage, block[f]);
    else
      fetch_words_if(mask, exps, ahead_stage + (uint32_t)G::kScales + 256u * (uint32_t)wave);
  };
  // (no branch: the compiler would move the products behind it)
  auto issued = [&](uint64_t mask) __attribute__((always_inline)) {
    const int by = (int)mask & BK;
    exps += exps_by & (long long)mask;
    base_a += by;
    base_b += by;
    ahead_stage ^= (uint32_t)mask & (uint32_t)G::kStage;
    ahead_left += (int)mask;
  };
  auto issue = [&]() __attribute__((always_inline)) {
    const uint64_t mask = ahead();
    if (!mask) return;
    wave::static_for<NF + 1>([&](auto fc) __attribute__((always_inline)) { issue_one(mask, fc); });
    issued(mask);
  };

  constexpr int kParts = 2 * TM, kHeld = kParts < 4 ? kParts : 4, kAhead = kHeld / 2;
  uint32_t stage = 0;
  u32x4 fm[kHeld][2], fn[2][TN][2];
  uint32_t sm[TM], sn[TN], next_m[TM], next_n[TN];
  // the fragments of part u of the step at `at`
  auto read = [&](uint32_t at, auto u) __attribute__((always_inline)) {
    constexpr int U = decltype(u)::value, h = U / TM, i = U % TM;
    const char *la = lds + at, *lb = la + G::TA::kBytes;
    if constexpr (U == 0) {
      const char* le = lds + at + G::kScales;
#pragma unroll
      for (int k = 0; k < TM; ++k) next_m[k] = (uint8_t)le[wm + 32 * k + (lane & 31)];
#pragma unroll
      for (int k = 0; k < TN; ++k) next_n[k] = (uint8_t)le[G::BM + wn + 32 * k + (lane & 31)];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if constexpr (i == 0) {
#pragma unroll
        for (int k = 0; k < TN; ++k) fn[h][k][j] = G::TB::frag(lb, wn + 32 * k, 2 * h + j).p[0];
      }
      fm[U % kHeld][j] = G::TA::frag(la, wm + 32 * i, 2 * h + j).p[0];
    }
  };

  aim();
  issue();
  wait_loads<0>();
  step_barrier();
  issue();
  for (; id < last; id += stride) {
    const At at = tile_of(id);
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int k = 0; k < TN; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][k][e] = 0.f;
    wave::static_for<kAhead>([&](auto u) __attribute__((always_inline)) { read(stage, u); });
    for (int s = at.s0; s < at.s1; ++s) {
      // (the last step's stage is the epilogue's: nothing is fetched to it before)
      const uint64_t mask = s + 1 < at.s1 ? ahead() : 0;
#pragma unroll
      for (int i = 0; i < TM; ++i) sm[i] = next_m[i];
#pragma unroll
      for (int i = 0; i < TN; ++i) sn[i] = next_n[i];
      wave::static_for<kParts>([&](auto part) __attribute__((always_inline)) {
        constexpr int t = decltype(part)::value, u = t + kAhead;
        if constexpr (u < kParts) {
          read(stage, std::integral_constant<int, u>{});
        } else {
          if constexpr (u == kParts) {
            wait_loads<0>();
            step_barrier();
            stage ^= (uint32_t)G::kStage;
          }
          read(stage, std::integral_constant<int, u - kParts>{});
        }
        __builtin_amdgcn_sched_barrier(0);
        // (a load between two products, not all of them before)
        auto between = [&](auto kc) __attribute__((always_inline)) {
          constexpr int slots = kAhead * TN, slot = (t - (kParts - kAhead)) * TN + decltype(kc)::value;
          if constexpr (slot >= 0) {
            constexpr int from = slot * (NF + 1) / slots, to = (slot + 1) * (NF + 1) / slots;
            wave::static_for<to - from>([&](auto i) __attribute__((always_inline)) {
              issue_one(mask, std::integral_constant<int, from + decltype(i)::value>{});
            });
            __builtin_amdgcn_sched_barrier(0);
          }
        };
        if constexpr (sizeof(T) == 4)
          wide_products<ATYPE>(fn[t / TM], fm[t % kHeld], sn, sm[t % TM], acc[t % TM], between);
        else
          f8_products<ATYPE>(fn[t / TM], fm[t % kHeld], sn, sm[t % TM], acc[t % TM], between);
        __builtin_amdgcn_sched_barrier(0);
      });
      issued(mask);
    }
    // The next tile's first step has landed (the tile's last step waited for it); the stage of this tile's last step
    // is free for the sums.  Its loads are the next tile's second step's, behind the epilogue.
    f8_epilogue<T, KIND>(P, at.m0 + G::BM <= P.M && at.n0 + G::BN <= P.N, at.m0 + wm, at.n0 + wn, at.split, acc,
                         lds + (stage ^ (uint32_t)G::kStage) + G::kMine * wave);
    step_barrier();
    issue();
  }
  wait_loads<0>();  // nothing is on its way to LDS when the workgroup ends
}

template <typename T, int KIND, int SHAPE, int ATYPE>
hipError_t launch_f8_shape(const F8Plan& pl, hipStream_t stream) {
  using G = F8Geo<SHAPE>;
  static std::atomic<int> allowed{0};
  static std::atomic<int> resident{0};
  if (!allowed.load(std::memory_order_acquire)) {
    const void* f = reinterpret_cast<const void*>(f8mm<T, KIND, SHAPE, ATYPE>);
    hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds);
    if (e != hipSuccess) return e;
    int per_cu = 0;
    e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, f, G::kThreads, G::kLds);
    if (e != hipSuccess) return e;
    resident.store(per_cu > 0 ? per_cu : 1);
    allowed.store(1, std::memory_order_release);
  }
  const int most = 256 * resident.load(), blocks = (pl.p.mm.nblocks + 7) / 8 * 8;
  hipLaunchKernelGGL((f8mm<T, KIND, SHAPE, ATYPE>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(G::kThreads),
                     G::kLds, stream, pl.p);
  return hipGetLastError();
}

// Few tiles: 32 x 32 results in a workgroup, whose waves take steps of their own, one behind the other, straight from memory to
// the fragments' registers, DEPTH steps ahead of the products; the waves' sums are joined in LDS.  No step waits for another wave's,
// and four times the workgroups share them, at twice the reads of 64 x 64.  Measured with its launch, bfloat16 results, against
// 64 x 64: 16 x 768 -> 1000 3.8 us against 4.8, 5 x 5671 -> 568 10.2 against 15.4, 512 x 2048 -> 512 6.6 against 7.6, but
// 1000 x 768 -> 768 7.1 against 5.4; float32 results 3.9, 10.2 and 6.8 against 6.0, 21.9 and 10.3.  Sixteen waves of one step
// each: 44 x 1418 -> 1884 5.5, in eight waves 6.4; four steps ahead 10.0 (more loads than the first products need).
template <typename T, int KIND, int ATYPE, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void f8mm_few(F8MmParams Q) {
  const MmParams& P = Q.mm;
  __shared__ __align__(16) float sums[WAVES][32 * 32];  // runs of four in an order of their row's own: no bank conflicts
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = (int)blockDim.x / 64;
  const int per_xcd = (P.nblocks + 7) / 8, id = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (id >= P.nblocks || (int)(blockIdx.x / 8) >= per_xcd) return;
  const int m0 = id % P.tm * 32, n0 = id / P.tm * 32;
  // a thread's run of eight results and what the epilogue reads for it
  const int m = m0 + (int)threadIdx.x / 4, n = n0 + (int)threadIdx.x % 4 * 8;
  const bool mine = threadIdx.x < 128 && m < P.M && n < P.N;
  Ahead<T, KIND, false> ahead;
  float bias[8] = {};
  if (mine) {
    if constexpr (KIND != kWgrad) ahead.load(P, m, n);
    if (KIND == kFwd && P.bias) {
#pragma unroll
      for (int e = 0; e < 8; ++e) bias[e] = n + e < P.N ? to_f32(static_cast<const T*>(P.bias)[n + e]) : 0.f;
    }
  }
  // rows past the end are the last one's: their results are not stored
  const int rm = min(m0 + (lane & 31), P.M - 1), rn = min(n0 + (lane & 31), P.N - 1);
  const char* const a = static_cast<const char*>(P.a) + (long long)rm * P.lda + 32 * half;
  const char* const b = static_cast<const char*>(P.b) + (long long)rn * P.ldb + 32 * half;
  const uint8_t *const ea = Q.ea + rm, *const eb = Q.eb + rn;
  u32x4 fm[DEPTH][2][2], fn[DEPTH][2][1][2];
  uint32_t sm[DEPTH], sn[DEPTH][1];
  auto load = [&](auto dc, int s) __attribute__((always_inline)) {
    constexpr int d = decltype(dc)::value;
    s = min(s, P.steps - 1);  // (no branch: loads are waited for one by one)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const long long at = (long long)s * kF8Group + 64 * h + 16 * j;
        fm[d][h][j] = *reinterpret_cast<const u32x4*>(a + at);
        fn[d][h][0][j] = *reinterpret_cast<const u32x4*>(b + at);
      }
    sm[d] = ea[s * Q.lea];
    sn[d][0] = eb[s * Q.leb];
  };
  f32x16 acc[1];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[0][e] = 0.f;
  wave::static_for<DEPTH>([&](auto d) __attribute__((always_inline)) { load(d, wave + waves * decltype(d)::value); });
  // (steps past the end are multiplied as zeros: a branch would take their loads with it, and wait there)
  auto multiply = [&](auto dc, int s) __attribute__((always_inline)) {
    constexpr int d = decltype(dc)::value;
    const uint32_t in = s < P.steps ? ~0u : 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        fm[d][h][j] &= in;
        fn[d][h][0][j] &= in;
      }
      auto nothing = [](auto) {};
      if constexpr (sizeof(T) == 4)
        wide_products<ATYPE>(fn[d][h], fm[d][h], sn[d], sm[d], acc, nothing);
      else
        f8_products<ATYPE>(fn[d][h], fm[d][h], sn[d], sm[d], acc, nothing);
    }
  };
  int s0 = wave;
  for (; s0 + waves * DEPTH < P.steps; s0 += waves * DEPTH)
    wave::static_for<DEPTH>([&](auto dc) __attribute__((always_inline)) {
      const int s = s0 + waves * decltype(dc)::value;
      multiply(dc, s);
      load(dc, s + waves * DEPTH);
      __builtin_amdgcn_sched_barrier(0);
    });
  wave::static_for<DEPTH>([&](auto dc) __attribute__((always_inline)) { multiply(dc, s0 + waves * decltype(dc)::value); });
  float* const to = &sums[wave][(lane & 31) * 32];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const float v[4] = {acc[0][4 * g], acc[0][4 * g + 1], acc[0][4 * g + 2], acc[0][4 * g + 3]};
    __builtin_memcpy(__builtin_assume_aligned(to + 4 * ((2 * g + half) ^ (lane & 7)), 16), v, 16);
  }
  __syncthreads();
  if (!mine) return;
  float v[8] = {};
  for (int w = 0; w < waves; ++w) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = (int)threadIdx.x / 4, run = (int)threadIdx.x % 4 * 2 + j;
      float k[4];
      __builtin_memcpy(k, __builtin_assume_aligned(&sums[w][row * 32 + 4 * (run ^ (row & 7))], 16), 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] += k[e];
    }
  }
  if constexpr (KIND == kWgrad) {
    put<T, false>(static_cast<T*>(P.out) + (long long)m * P.N + n, P.N - n, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += bias[e];
    finish<T, KIND, false>(P, m, n, ahead, v);
  }
}

template <typename T, int KIND, int ATYPE>
hipError_t launch_f8_few(const F8Plan& pl, hipStream_t stream) {
  const int steps = pl.p.mm.steps, waves = steps < 2 ? 2 : (steps <= 16 ? steps : 8);  // (two have the epilogue's threads)
  const dim3 grid((unsigned)((pl.p.mm.nblocks + 7) / 8 * 8)), threads((unsigned)(64 * waves));
  if (steps <= 8)
    hipLaunchKernelGGL((f8mm_few<T, KIND, ATYPE, 8, 1>), grid, threads, 0, stream, pl.p);
  else if (steps <= 16)
    hipLaunchKernelGGL((f8mm_few<T, KIND, ATYPE, 16, 1>), grid, threads, 0, stream, pl.p);
  else
    hipLaunchKernelGGL((f8mm_few<T, KIND, ATYPE, 8, 2>), grid, threads, 0, stream, pl.p);
  return hipGetLastError();
}

template <typename T, int KIND, int SHAPE>
hipError_t launch_f8_type(const F8Plan& pl, hipStream_t stream) {
  return pl.atype == kE4M3 ? launch_f8_shape<T, KIND, SHAPE, kE4M3>(pl, stream)
                           : launch_f8_shape<T, KIND, SHAPE, kE5M2>(pl, stream);
}

template <typename T, int KIND>
hipError_t launch_f8_kind(const F8Plan& pl, hipStream_t stream) {
  switch (pl.shape) {
    case kF8_128x128: return launch_f8_type<T, KIND, kF8_128x128>(pl, stream);
    case kF8_256x256:
      if constexpr (sizeof(T) == 2 && KIND != kWgrad) return launch_f8_type<T, KIND, kF8_256x256>(pl, stream);
      return hipErrorInvalidValue;  // (no plan has it)
    case kF8_64x64: return launch_f8_type<T, KIND, kF8_64x64>(pl, stream);
    case kF8_32x32:
      return pl.atype == kE4M3 ? launch_f8_few<T, KIND, kE4M3>(pl, stream) : launch_f8_few<T, KIND, kE5M2>(pl, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace
}  // namespace rows
}  // namespace o1d
