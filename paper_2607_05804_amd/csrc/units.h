// Eight elements of a row at a time, bf16 or fp32, for the kernels over hidden rows: rows
// of any start, stride and width, addressed by plain pointers, so that the lanes of a wave
// may work on rows of their own.
#pragma once

#include <hip/hip_bf16.h>

#include "row_ops.h"

namespace turnkl {
namespace {

constexpr int kUnit = 8;  // elements

// Four words at any address that a bf16 may have.  (The memory pipeline takes vector
// accesses off their alignment; those that lie on 16 bytes run at full speed.)
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2), may_alias));

__device__ inline float half_of(unsigned w, int j) {
  return __uint_as_float((j & 1) ? (w & 0xFFFF0000u) : (w << 16));
}

// kKeep: rows that other waves read too stay in the caches.
template <bool kBf16, bool kKeep = false>
struct Unit {
  static constexpr int kEs = kBf16 ? 2 : 4;
  static constexpr int kQuads = kBf16 ? 1 : 2;
  u32x4 q[kQuads];

  __device__ void clear() {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) q[i] = u32x4{0u, 0u, 0u, 0u};
  }
  // the unit that starts at element `at` of a row
  __device__ void load(const char* row, int at) {
    const char* const p = row + (long long)at * kEs;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const u32x4_any* const a = reinterpret_cast<const u32x4_any*>(p + 16 * i);
      if constexpr (kKeep) q[i] = *a;
      else q[i] = __builtin_nontemporal_load(a);
    }
  }
  __device__ void store(char* row, int at) const {
    char* const p = row + (long long)at * kEs;
#pragma unroll
    for (int i = 0; i < kQuads; ++i)
      __builtin_nontemporal_store(u32x4_any(q[i]), reinterpret_cast<u32x4_any*>(p + 16 * i));
  }
  // the same for the elements of `bits` alone, one by one
  __device__ void load_some(const char* row, int at, unsigned bits) {
    clear();
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if ((bits >> j) & 1u) {
        if constexpr (kBf16)
          q[0][j >> 1] |= (unsigned)reinterpret_cast<const unsigned short*>(row)[at + j] << (16 * (j & 1));
        else
          q[j >> 2][j & 3] = reinterpret_cast<const unsigned*>(row)[at + j];
      }
  }
  __device__ void store_some(char* row, int at, unsigned bits) const {
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if ((bits >> j) & 1u) {
        if constexpr (kBf16)
          reinterpret_cast<unsigned short*>(row)[at + j] = (unsigned short)(q[0][j >> 1] >> (16 * (j & 1)));
        else
          reinterpret_cast<unsigned*>(row)[at + j] = q[j >> 2][j & 3];
      }
  }
  __device__ float get(int j) const {
    if constexpr (kBf16) return half_of(q[0][j >> 1], j);
    else return __uint_as_float(q[j >> 2][j & 3]);
  }
  // rounds to nearest even
  __device__ void set(const float (&v)[kUnit]) {
    if constexpr (kBf16) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x2 x = {v[2 * k], v[2 * k + 1]};
        q[0][k] = __builtin_bit_cast(unsigned, __builtin_convertvector(x, bf16x2));
      }
    } else {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) q[j >> 2][j & 3] = __float_as_uint(v[j]);
    }
  }
  // Unpacked again after it, rather than kept.
  __device__ void fence() {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) asm volatile("" : "+v"(q[i]));
  }
  // Complete here, before any of the stores that follow: the data of a wide store must
  // not be rewritten closely behind it, nor that of the next one closely behind this one.
  __device__ void settle() { fence(); }
  __device__ void keep() const {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) keep_alive(q[i]);
  }
};

// Between a wide store and what may rewrite its data, where that is not kept otherwise:
// two dozen idle instructions, an order of magnitude less than waiting for the store.
__device__ inline void store_gap() {
#pragma unroll
  for (int i = 0; i < 24; ++i) asm volatile("s_nop 7" ::: "memory");
}

// Where unit `u` of a row lies: its first element, moved inside the row where it sticks
// out, and which of the eight elements there are its own (none beyond the row).
struct Place {
  int at;
  unsigned bits;
  __device__ bool whole() const { return bits == (1u << kUnit) - 1u; }
};
__device__ inline Place place_unit(int u, int width) {
  const int e = u * kUnit;
  Place p;
  p.at = inside_row(e, width > kUnit ? width - kUnit : 0);
  p.bits = e < width ? own_bits<kUnit>(e - p.at) : 0u;
  if (width < kUnit) p.bits &= (1u << width) - 1u;
  return p;
}

// Loads a unit whole (elements that are not its own among them) where the row is as
// long, else its own elements.  Nothing is loaded where it has none.
template <bool kBf16, bool kKeep>
__device__ inline void load_unit(Unit<kBf16, kKeep>& x, const char* row, const Place& p, int width) {
  if (width >= kUnit) {
    if (p.bits) x.load(row, p.at);
    else x.clear();
  } else {
    x.load_some(row, p.at, p.bits);
  }
}
// Stores of units that are not their lane's entirely, at the ends of a row, and of whole
// ones.  Of several units the first kind goes first: its code shifts the data, which must
// not follow the wide stores closely.
template <bool kBf16, bool kKeep>
__device__ inline void store_edge(const Unit<kBf16, kKeep>& x, char* row, const Place& p) {
  if (!p.whole() && p.bits) x.store_some(row, p.at, p.bits);
}
template <bool kBf16, bool kKeep>
__device__ inline void store_whole(const Unit<kBf16, kKeep>& x, char* row, const Place& p) {
  if (p.whole()) x.store(row, p.at);
}
template <bool kBf16, bool kKeep>
__device__ inline void store_unit(const Unit<kBf16, kKeep>& x, char* row, const Place& p) {
  store_edge(x, row, p);
  store_whole(x, row, p);
}

}  // namespace
}  // namespace turnkl
