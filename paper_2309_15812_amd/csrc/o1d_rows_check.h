// Argument checks that the row operators' entry points share (included by the units that define them).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdio.h>

#include <initializer_list>

#include "o1d.h"
#include "o1d_rows.h"
#include "o1d_status.h"

namespace {

using o1d::Dtype;
using o1d::elem_size;
using o1d::fail;
using o1d::ok;
using o1d::overlaps;
namespace rows = o1d::rows;

// Rows and features below 2^31 with room for a tile; row strides such that a
// tile's offsets stay below 2^31 bytes.
constexpr int kMaxRows = 0x7fffffff - 1024;
constexpr int kMaxFeatures = 1 << 20;
constexpr long long kMaxStride = 1 << 21;

// What a call that needs no workspace asks for all the same, so that callers need not know which do.  One that
// writes to its workspace asks for more, however little that is: callers may share
// a workspace of kNoSpace bytes between calls that run at the same time.
constexpr size_t kNoSpace = 256, kLeastSpace = 2 * kNoSpace;
[[maybe_unused]] size_t space_for(size_t bytes) { return bytes < kLeastSpace ? kLeastSpace : bytes; }

[[maybe_unused]] size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// One tensor of a call: where it lies and how far it reaches.
struct Span {
  const char* what;
  const void* p;
  size_t bytes;
  bool out;
};

[[maybe_unused]] size_t reach(long long M, long long ld, long long C, size_t es) {
  return M > 0 && C > 0 ? ((size_t)(M - 1) * (size_t)ld + (size_t)C) * es : 0;
}
[[maybe_unused]] size_t held_q_bytes(int M, int C) { return (size_t)M * (size_t)rows::held_ld(C); }
[[maybe_unused]] size_t held_scale_bytes(int M, int C) { return (size_t)M * (size_t)rows::held_groups(C) * sizeof(float); }

// No output overlaps an input or another output.
template <int N>
o1d_status_t apart(const char* fn, const Span (&s)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N; ++j)
      if (i != j && s[i].out && s[i].p && s[j].p && s[i].bytes && s[j].bytes &&
          overlaps(s[i].p, s[i].bytes, s[j].p, s[j].bytes))
        return fail(O1D_ERR_INVALID, "%s: %s overlaps %s", fn, s[i].what, s[j].what);
  return O1D_OK;
}

[[maybe_unused]] o1d_status_t check_dims(const char* fn, int M, int C, const char* feature, o1d_dtype_t dt) {
  if (dt != O1D_F32 && dt != O1D_BF16) return fail(O1D_ERR_INVALID, "%s: unknown dtype %d", fn, (int)dt);
  if (M < 0) return fail(O1D_ERR_INVALID, "%s: negative rows M=%d", fn, M);
  if (C < 1) return fail(O1D_ERR_INVALID, "%s: %s=%d must be positive", fn, feature, C);
  if (M > kMaxRows) return fail(O1D_ERR_UNSUPPORTED, "%s: M=%d rows exceed %d", fn, M, kMaxRows);
  if (C > kMaxFeatures) return fail(O1D_ERR_UNSUPPORTED, "%s: %s=%d exceeds %d", fn, feature, C, kMaxFeatures);
  return O1D_OK;
}

[[maybe_unused]] o1d_status_t check_ld(const char* fn, const char* what, long long ld, int C) {
  if (ld < C) return fail(O1D_ERR_INVALID, "%s: row stride %lld of %s is below its %d features", fn, ld, what, C);
  if (ld >= kMaxStride) return fail(O1D_ERR_UNSUPPORTED, "%s: row stride %lld of %s exceeds %lld", fn, ld, what, kMaxStride);
  return O1D_OK;
}

[[maybe_unused]] o1d_status_t check_act(const char* fn, o1d_act_t act) {
  return (int)act >= 0 && (int)act < rows::kActs ? O1D_OK
                                                 : fail(O1D_ERR_INVALID, "%s: unknown activation %d", fn, (int)act);
}

// The integers are accessed eight at a time.
[[maybe_unused]] o1d_status_t check_held(const char* fn, const signed char* q, const float* scale) {
  if (!q || !scale) return fail(O1D_ERR_INVALID, "%s: a checkpoint needs its integers and its scales", fn);
  if ((uintptr_t)q % 16) return fail(O1D_ERR_INVALID, "%s: a checkpoint's integers must be 16-byte aligned", fn);
  return O1D_OK;
}

// A tensor (p) or a checkpoint (q), one of the two.
[[maybe_unused]] o1d_status_t check_either(const char* fn, const char* what, const void* p, long long ld, int C, const signed char* q,
                          const float* scale) {
  if (!p == !q) return fail(O1D_ERR_INVALID, "%s: %s is given as a tensor or as a checkpoint, one of the two", fn, what);
  return p ? check_ld(fn, what, ld, C) : check_held(fn, q, scale);
}

[[maybe_unused]] o1d_status_t check_elem_aligned(const char* fn, const void* p, const char* what, size_t es) {
  return (uintptr_t)p % es ? fail(O1D_ERR_INVALID, "%s: %s is not aligned to its elements", fn, what) : O1D_OK;
}

[[maybe_unused]] o1d_status_t hip_status(const char* fn, hipError_t e) {
  if (e != hipSuccess) return fail(O1D_ERR_HIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return ok();
}

#define O1D_TRY(expr)                         \
  do {                                        \
    const o1d_status_t st_ = (expr);          \
    if (st_ != O1D_OK) return st_;            \
  } while (0)

[[maybe_unused]] o1d_status_t check_null(const char* fn, std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!p) return fail(O1D_ERR_INVALID, "%s: NULL tensor pointer", fn);
  return O1D_OK;
}

[[maybe_unused]] o1d_status_t check_workspace(const char* fn, const void* workspace, size_t bytes, size_t need) {
  if (need && (bytes < need || !workspace))
    return fail(O1D_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", fn, bytes, need);
  if ((uintptr_t)workspace % 16) return fail(O1D_ERR_INVALID, "%s: workspace must be 16-byte aligned", fn);
  return O1D_OK;
}

}  // namespace
