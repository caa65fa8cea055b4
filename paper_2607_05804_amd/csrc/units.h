// Units of a few elements of a row, bf16 or fp32, for the kernels over hidden rows: rows of
// any start, stride and width, addressed by plain pointers, so that the lanes of a wave
// may work on rows of their own.  A unit is 16 bytes, or 8 where its row goes with one of
// the wider type: then the lanes' units of either lie side by side without gaps.  (Two
// 16-byte stores of a lane side by side, which leave a gap in every line of each, wrote
// table rows at 3 TB/s.)
#pragma once

#include <hip/hip_bf16.h>

#include "row_ops.h"

namespace turnkl {
namespace {

// Computed here, before the stores that follow.
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
__device__ inline void settle_words(u32x4& x) { asm volatile("" : "+v"(x)); }
__device__ inline void settle_words(u32x2& x) { asm volatile("" : "+v"(x)); }
__device__ inline void keep_alive(const u32x2& x) { asm volatile("" ::"v"(x)); }

// Words at any address that a bf16 may have.  (The memory pipeline takes vector accesses
// off their alignment.)
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(2), may_alias));
template <int kWords>
struct Words;
template <>
struct Words<4> {
  using T = u32x4;
  using Any = u32x4_any;
};
template <>
struct Words<2> {
  using T = u32x2;
  using Any = u32x2_any;
};

// Elements of a unit where rows of these types go together.
constexpr int unit_elements(bool a_bf16, bool b_bf16) { return a_bf16 && b_bf16 ? 8 : 4; }

// kKeep: loads of rows that other waves read too, or that are read again, stay in the caches.
template <bool kBf16, int kEl, bool kKeep = false>
struct Unit {
  static constexpr int kEs = kBf16 ? 2 : 4;
  static constexpr int kWords = kEl * kEs / 4;
  using W = typename Words<kWords>::T;
  using Any = typename Words<kWords>::Any;
  W w;

  __device__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  // the unit that starts at element `at` of a row
  __device__ void load(const char* row, int at) {
    const Any* const a = reinterpret_cast<const Any*>(row + (long long)at * kEs);
    if constexpr (kKeep) w = *a;
    else w = __builtin_nontemporal_load(a);
  }
  __device__ void store(char* row, int at) const {
    __builtin_nontemporal_store(Any(w), reinterpret_cast<Any*>(row + (long long)at * kEs));
  }
  // the same for the elements of `bits` alone, one by one
  __device__ void load_some(const char* row, int at, unsigned bits) {
    clear();
#pragma unroll
    for (int j = 0; j < kEl; ++j)
      if ((bits >> j) & 1u) {
        if constexpr (kBf16)
          w[j >> 1] |= (unsigned)reinterpret_cast<const unsigned short*>(row)[at + j] << (16 * (j & 1));
        else
          w[j] = reinterpret_cast<const unsigned*>(row)[at + j];
      }
  }
  __device__ void store_some(char* row, int at, unsigned bits) const {
#pragma unroll
    for (int j = 0; j < kEl; ++j)
      if ((bits >> j) & 1u) {
        if constexpr (kBf16)
          reinterpret_cast<unsigned short*>(row)[at + j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
        else
          reinterpret_cast<unsigned*>(row)[at + j] = w[j];
      }
  }
  __device__ float get(int j) const {
    if constexpr (kBf16) return __uint_as_float((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16));
    else return __uint_as_float(w[j]);
  }
  // rounds to nearest even
  __device__ void set(const float (&v)[kEl]) {
    if constexpr (kBf16) {
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        const f32x2 x = {v[2 * k], v[2 * k + 1]};
        w[k] = __builtin_bit_cast(unsigned, __builtin_convertvector(x, bf16x2));
      }
    } else {
#pragma unroll
      for (int j = 0; j < kEl; ++j) w[j] = __float_as_uint(v[j]);
    }
  }
  // Unpacked again after it, rather than kept; and for a store's data: complete here,
  // before any of the stores that follow (the data of a wide store must not be rewritten
  // closely behind it, nor that of the next one closely behind this one).
  __device__ void fence() { settle_words(w); }
  __device__ void keep() const { keep_alive(w); }
};

// Between a wide store and what may rewrite its data, where that is not kept otherwise:
// two dozen idle instructions, an order of magnitude less than waiting for the store.
__device__ inline void store_gap() {
#pragma unroll
  for (int i = 0; i < 24; ++i) asm volatile("s_nop 7" ::: "memory");
}

// Where unit `u` of a row lies: its first element, moved inside the row where it sticks
// out, and which of the elements there are its own (none beyond the row).
template <int kEl>
struct Place {
  int at;
  unsigned bits;
  __device__ bool whole() const { return bits == (1u << kEl) - 1u; }
};
template <int kEl>
__device__ inline Place<kEl> place_unit(int u, int width) {
  const int e = u * kEl;
  Place<kEl> p;
  p.at = inside_row(e, width > kEl ? width - kEl : 0);
  p.bits = e < width ? own_bits<kEl>(e - p.at) : 0u;
  if (width < kEl) p.bits &= (1u << width) - 1u;
  return p;
}

// Loads a unit whole (elements that are not its own among them) where the row is as
// long, else its own elements.  Nothing is loaded where it has none.
template <bool kBf16, int kEl, bool kKeep>
__device__ inline void load_unit(Unit<kBf16, kEl, kKeep>& x, const char* row, const Place<kEl>& p, int width) {
  if (width >= kEl) {
    if (p.bits) x.load(row, p.at);
    else x.clear();
  } else {
    x.load_some(row, p.at, p.bits);
  }
}
// Stores of units that are not their lane's entirely, at the ends of a row, and of whole
// ones.  Of several units the first kind goes first: its code shifts the data, which must
// not follow the wide stores closely.
template <bool kBf16, int kEl, bool kKeep>
__device__ inline void store_edge(const Unit<kBf16, kEl, kKeep>& x, char* row, const Place<kEl>& p) {
  if (!p.whole() && p.bits) x.store_some(row, p.at, p.bits);
}
template <bool kBf16, int kEl, bool kKeep>
__device__ inline void store_whole(const Unit<kBf16, kEl, kKeep>& x, char* row, const Place<kEl>& p) {
  if (p.whole()) x.store(row, p.at);
}

}  // namespace
}  // namespace turnkl
