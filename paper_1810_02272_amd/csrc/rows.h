// Rows of logits as vectors of 16 bytes, in the order of their values, for a team of threads that takes a row each.
#pragma once

#include <hip/hip_runtime.h>

#include "device_utils.h"
#include "elements.h"

namespace mi355conv {

// Logits in descending order, as unsigned numbers: -0 is 0, NaN the greatest.  With the index below it, each once.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xFFFFFFFEu;
  const uint32_t u = x == 0.f ? 0u : __builtin_bit_cast(uint32_t, x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

__device__ __forceinline__ uint64_t entry_of(float x, int index) { return (uint64_t)order_key(x) << 32 | (0xFFFFFFFFu - (uint32_t)index); }

// Vector v of a row holds its elements v VEC and on.  A partial one at the end, the tail, is thread 0's: it is loaded so that it ends
// with the row, and what an earlier vector holds as well is taken out (-inf): every access is inside the row.
template <class E>
struct Slot {
  int base;  // of element 0, negative in rows shorter than a vector
  int lo;    // elements from here on are this vector's
};

template <class E>
__device__ __forceinline__ Slot<E> slot_of(int v, int n) {
  const int b = v * E::VEC, over = b + E::VEC - n;
  return over <= 0 ? Slot<E>{b, 0} : Slot<E>{b - over, over};
}

template <class E>
__device__ __forceinline__ u32x4 lowest_vec() {
  return u32x4{E::kLowest, E::kLowest, E::kLowest, E::kLowest};
}

template <class E>
__device__ __forceinline__ u32x4 without_first(const u32x4& v, int lo) {
  u32x4 r = v;
  constexpr int PER = E::VEC / 4;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (PER == 1) {
      if (w < lo) r[w] = E::kLowest;
    } else {
      if (2 * w < lo) r[w] = (r[w] & 0xffff0000u) | (E::kLowest & 0xffffu);
      if (2 * w + 1 < lo) r[w] = (r[w] & 0xffffu) | (E::kLowest & 0xffff0000u);
    }
  }
  return r;
}

// Vector v (v VEC < n), wherever it lies.
template <class E, bool STREAM = false>
__device__ __forceinline__ u32x4 row_vec(const typename E::T* row, int v, int n) {
  const Slot<E> at = slot_of<E>(v, n);
  if (at.base >= 0) {
    const u32x4 r = get_vec<E, STREAM>(row + at.base);
    return at.lo ? without_first<E>(r, at.lo) : r;
  }
  float x[E::VEC];
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) x[i] = i >= at.lo ? E::to_float(row[at.base + i]) : -INFINITY;
  return E::pack(x);
}

// The same of a row of at least a vector, and -inf throughout beyond its last one: one load, whatever v is; and apart, for those who do something
// else while it is on its way.
template <class E>
__device__ __forceinline__ u32x4 begin_row_vec(const typename E::T* row, int v, int nv, int n) {
  return load_vec<E>(row + slot_of<E>(min(v, nv - 1), n).base);
}

template <class E>
__device__ __forceinline__ u32x4 end_row_vec(const u32x4& r, int v, int nv, int n) {
  const int lo = slot_of<E>(v, n).lo;
  return v >= nv ? lowest_vec<E>() : lo ? without_first<E>(r, lo) : r;
}

template <class E>
__device__ __forceinline__ u32x4 long_row_vec(const typename E::T* row, int v, int nv, int n) {
  return end_row_vec<E>(begin_row_vec<E>(row, v, nv, n), v, nv, n);
}

template <int THREADS>
__device__ __forceinline__ void team_sync() {
  if constexpr (THREADS == 64)
    wave_sync();
  else
    __syncthreads();
}

}  // namespace mi355conv
