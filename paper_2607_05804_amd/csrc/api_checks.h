// Host-side argument checks that the C entry points of the operators around the logits
// and at the token boundary share.
#pragma once

#include "turnkl_internal.h"

namespace turnkl {
namespace {

inline bool misaligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

// Whether any of the outputs overlaps an input or another output.
inline bool any_overlap(std::initializer_list<Region> in, std::initializer_list<Region> out) {
  for (const Region* a = out.begin(); a != out.end(); ++a) {
    if (!a->p || !a->n) continue;
    if (overlaps_any(a->p, a->n, in)) return true;
    for (const Region* b = a + 1; b != out.end(); ++b)
      if (b->p && b->n && overlaps(a->p, a->n, b->p, b->n)) return true;
  }
  return false;
}

inline bool known_dtype(int dtype) { return dtype == TURNKL_BF16 || dtype == TURNKL_F32; }
inline size_t elem_size(int dtype) { return dtype == TURNKL_BF16 ? 2 : 4; }

inline bool rows_ok(const void* p, int64_t ld, int64_t width, size_t es) {
  return p && ld >= width && ld <= 0x7FFFFFFFll && !misaligned(p, es);
}

// Whether every row of the matrix is whole 16-byte packs.
inline bool whole_packs(const void* p, int64_t ld, int64_t n_rows, int64_t width, size_t es) {
  return !misaligned(p, 16) && (width * es) % 16 == 0 && (n_rows <= 1 || (ld * es) % 16 == 0);
}

}  // namespace
}  // namespace turnkl
