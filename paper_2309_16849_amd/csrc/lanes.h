// lanes.h -- runs of consecutive floats that a lane loads and stores at once
// (device side), at any 4-byte address.
#pragma once

#include "layer.h"

#ifdef __HIPCC__

namespace snls {

template <int V>
using Run = float __attribute__((ext_vector_type(V), aligned(4)));

// The first cnt of V floats at `from`, 0 for the others.
template <int V>
SNLS_DEV void load_run(const float* from, int cnt, float* to) {
  if (cnt >= V) {
    const Run<V> r = *reinterpret_cast<const Run<V>*>(from);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = r[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = i < cnt ? from[i] : 0.f;
  }
}

template <int V>
SNLS_DEV void store_run(float* to, int cnt, const float* from) {
  if (cnt >= V) {
    Run<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = from[i];
    *reinterpret_cast<Run<V>*>(to) = r;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < cnt) to[i] = from[i];
  }
}

// Where every store of a wave fills whole cache lines (WHOLE: rows of 32 floats,
// or a multiple, at their multiple) outputs go past the caches (non-temporal),
// so that they do not push inputs out of them: frames of 192 channels at 152x152
// to 576 take 75 us so and 88 with ordinary stores, the norm of a residual sum at
// 5x64x480x854 404 and 422, its gradients at 5x512x128x128 171 and 177 (every
// call on inputs that no cache holds; at 4x48x272x480 ordinary stores are the
// faster, 43 us and 47).  Where lines are shared by two waves ordinary stores let
// the L2 join the parts: the norm at 4x64x270x483 126 us, past the caches 138.
template <bool WHOLE, int V>
SNLS_DEV void put_run(float* to, int cnt, const float* from) {
  if constexpr (WHOLE) {
    if (cnt >= V) {
      Run<V> r;
#pragma unroll
      for (int i = 0; i < V; ++i) r[i] = from[i];
      __builtin_nontemporal_store(r, reinterpret_cast<Run<V>*>(to));
      return;
    }
  }
  store_run<V>(to, cnt, from);
}

// The float at `base` (the same for the wave: two scalar registers) and a lane's
// offset in bytes.
SNLS_DEV float load_at(const float* base, unsigned bytes) {
  return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(base) + bytes);
}
template <bool WHOLE>
SNLS_DEV void store_at(float* base, unsigned bytes, float v) {
  float* const to = reinterpret_cast<float*>(reinterpret_cast<char*>(base) + bytes);
  if constexpr (WHOLE)
    __builtin_nontemporal_store(v, to);
  else
    *to = v;
}

// The items this workgroup takes of `items`.  By the 8 XCDs, which take
// workgroups in turn, neighbours lie on one of them: what two workgroups write of
// one cache line meets in one L2.  Every XCD has its eighth of the items, and its
// workgroups walk it together.
struct Walk {
  long long first, end, step;
};
template <bool BY_XCD>
SNLS_DEV Walk walk(long long items) {
  const unsigned b = blockIdx.x, n = gridDim.x, x = b & 7;
  if (!BY_XCD || n < 8) return {b, items, n};
  if (n % 8 == 0) return {items * x / 8 + b / 8, items * (x + 1) / 8, n / 8};
  const unsigned per = n / 8;  // (as many workgroups as items, or nearly)
  return {b < per * 8 ? x * per + b / 8 : b, items, n};
}

}  // namespace snls

#endif  // __HIPCC__
