// Status codes and argument checks shared by the C ABI's translation units.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "o1d.h"

namespace o1d {

// Sets the calling thread's error text and returns st; ok() clears it.
o1d_status_t fail(o1d_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
o1d_status_t ok();

inline size_t elem_size(o1d_dtype_t dt) { return dt == O1D_BF16 ? 2u : 4u; }

inline bool overlaps(const void* a, size_t abytes, const void* b, size_t bbytes) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + bbytes && b0 < a0 + abytes;
}

}  // namespace o1d
